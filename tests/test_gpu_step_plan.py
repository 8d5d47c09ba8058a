"""The bookkeeping of a step against the oracle: whole numbers, equal to the last."""
import numpy as np
import pytest

from oracle import mquant_oracle as orc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mq():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2502_00425_amd import binding
    return binding


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def make(rng, n_seq, page, most, rows_up_to, end=0.2, spare=4, extra_table=1, idle=0.1):
    """Sequences of up to `most` tokens that ask for up to rows_up_to rows, some of them ended or idle; pages dealt from a pool."""
    length = rng.integers(0, most + 1, n_seq).astype(np.int32)
    rows = rng.integers(1, rows_up_to + 1, n_seq).astype(np.int32)
    rows[rng.random(n_seq) < end] = -1
    rows[rng.random(n_seq) < idle] = 0
    have = -(-length // page)
    width = -(-(most + rows_up_to) // page) + extra_table
    need = int((-(-(length + np.maximum(rows, 0)) // page) - have).sum())
    n_pages = max(1, int(have.sum()) + need + spare)
    ids = rng.permutation(n_pages).astype(np.int32)
    table = np.full((n_seq, width), -5, dtype=np.int32)
    at = 0
    for s in range(n_seq):
        table[s, :have[s]] = ids[at:at + have[s]]
        at += have[s]
    ring = np.full(n_pages, -9, dtype=np.int32)
    head = int(rng.integers(0, n_pages))
    ring[(head + np.arange(n_pages - at)) % n_pages] = ids[at:]
    return {"length": length, "rows": rows, "table": table, "ring": ring, "state": np.array([head, n_pages - at], dtype=np.int32),
            "shared": np.minimum(have, rng.integers(0, 3, n_seq)).astype(np.int32), "T": int(np.maximum(rows, 0).sum())}


def check(mq, st, page, T, shared=True, order=None, in_place=False, slots=True):
    shared = st["shared"] if shared else None
    table, ring = st["table"].copy(), st["ring"].copy()
    want = orc.step_plan(st["length"], st["rows"], table, page, ring, st["state"], T, shared, order)
    length, state, t, r = dev(st["length"]), dev(st["state"]), dev(st["table"]), dev(st["ring"])
    new_length, new_state = (length, state) if in_place else (torch.full_like(length, 77), torch.full_like(state, 77))
    out = mq.step_plan(length, dev(st["rows"]), t, page, r, state, T, shared_dev=None if shared is None else dev(shared),
                       order_dev=None if order is None else dev(order), length_out=new_length, state_out=new_state)
    for got, ref, what in zip((*out, new_length, new_state, t, r), (*want, table, ring),
                              ("row_start", "pos", "slots", "length", "state", "table", "ring")):
        assert np.array_equal(got.cpu().numpy(), ref), what
    if not in_place:
        assert np.array_equal(length.cpu().numpy(), st["length"]) and np.array_equal(state.cpu().numpy(), st["state"])


@pytest.mark.parametrize("n_seq", [1, 2, 63, 64, 65, 700, 1023, 1024, 1025, 2500])
@pytest.mark.parametrize("page", [16, 128])
def test_plan(mq, n_seq, page):
    rng = np.random.default_rng(n_seq + page)
    st = make(rng, n_seq, page, 500, 9)
    check(mq, st, page, st["T"])
    check(mq, st, page, st["T"] + 37, shared=False, in_place=True)


@pytest.mark.parametrize("n_seq,rows", [(1, 1), (1, 5000), (3, 2000), (40, 900), (4095, 3), (4097, 3)])
def test_rows_by_the_second_kernel(mq, n_seq, rows):
    rng = np.random.default_rng(rows)
    st = make(rng, n_seq, 64, 300, rows, end=0.1 if n_seq > 1 else 0, idle=0)
    order = rng.integers(-1, rows + 1, st["T"]).astype(np.int32)             # some outside
    check(mq, st, 64, st["T"], order=order)


def test_rows_and_pages_run_out(mq):
    rng = np.random.default_rng(3)
    for n_seq in (1, 5, 1500):
        st = make(rng, n_seq, 16, 100, 40)
        for T in (0, 1, st["T"] // 3, max(st["T"] - 1, 0)):
            check(mq, st, 16, T)
        for pages in (0, 1, 7, int(st["state"][1]) // 2):
            check(mq, {**st, "state": np.array([st["state"][0], pages], dtype=np.int32)}, 16, st["T"])


def test_states_lengths_and_requests_out_of_range(mq):
    rng = np.random.default_rng(4)
    st = make(rng, 30, 16, 100, 20)
    n = len(st["ring"])
    for head, count in ((-1, 5), (n, 5), (3 * n + 2, n + 4), (-2 ** 31, 2 ** 31 - 1), (2, -7)):
        check(mq, {**st, "state": np.array([head, count], dtype=np.int32)}, 16, st["T"])
    odd = {**st, "length": st["length"].copy(), "rows": st["rows"].copy(), "shared": st["shared"].copy()}
    odd["length"][:4], odd["rows"][:8] = [-3, -2 ** 31, 2 ** 31 - 1, 10 ** 6], [2, 1, 5, -2 ** 31, 2 ** 31 - 1, 130, 5, -1]
    odd["shared"][5:9] = [-4, 2 ** 31 - 1, 2 ** 31 - 1, -2 ** 31]
    check(mq, odd, 16, st["T"])
    check(mq, odd, 16, 2 ** 16, in_place=True)


def test_pages_out_of_range_have_no_slot(mq):
    st = {"length": np.array([5], dtype=np.int32), "rows": np.array([30], dtype=np.int32), "table": np.array([[99, -1, -1, -1]], dtype=np.int32),
          "ring": np.array([2, -4, 0], dtype=np.int32), "state": np.array([0, 3], dtype=np.int32), "shared": np.zeros(1, np.int32)}
    check(mq, st, 16, 32)


def test_nothing_to_do(mq):
    e = torch.empty(0, dtype=torch.int32, device="cuda")
    ring, state = dev(np.arange(4, dtype=np.int32)), dev(np.array([1, 2], dtype=np.int32))
    start, pos, slots = mq.step_plan(e, e, e.view(0, 1), 16, ring, state, 5, state_out=state)
    assert start.tolist() == [0] and pos.tolist() == [-1] * 5 and slots.tolist() == [-1] * 5 and state.tolist() == [1, 2]


def test_a_loop_in_a_graph(mq):
    """Steps replayed from one graph, lengths and free pages in place: sequences grow, end and begin again, as the oracle says."""
    rng = np.random.default_rng(6)
    n_seq, page, T = 9, 16, 40
    table, ring = np.full((n_seq, 8), -1, dtype=np.int32), rng.permutation(60).astype(np.int32)
    length, state = np.zeros(n_seq, dtype=np.int32), np.array([11, 60], dtype=np.int32)
    d = {k: dev(v) for k, v in dict(length=length, state=state, table=table, ring=ring, rows=np.zeros(n_seq, np.int32)).items()}
    out = {"row_start": torch.empty(n_seq + 1, dtype=torch.int32, device="cuda"), "pos": torch.empty(T, dtype=torch.int32, device="cuda"),
           "slots": torch.empty(T, dtype=torch.int64, device="cuda")}
    call = lambda: mq.step_plan(d["length"], d["rows"], d["table"], page, d["ring"], d["state"], T, length_out=d["length"], state_out=d["state"], **out)
    call()                                                              # no rows: nothing changes
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(40):
        rows = rng.integers(0, 7, n_seq).astype(np.int32)
        rows[rng.random(n_seq) < 0.15] = -1
        d["rows"].copy_(dev(rows))
        graph.replay()
        start, pos, slots, length, state = orc.step_plan(length, rows, table, page, ring, state, T)
        for got, ref in ((out["row_start"], start), (out["pos"], pos), (out["slots"], slots), (d["length"], length), (d["state"], state),
                         (d["table"], table), (d["ring"], ring)):
            assert np.array_equal(got.cpu().numpy(), ref), step
