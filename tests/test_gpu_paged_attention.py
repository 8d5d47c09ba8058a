"""Attention of a step's rows over a paged cache against the fp64 oracle.  Slots that no row may look at hold NaN and
infinity, table entries behind a sequence's last page are out of range.  Tolerance: serving.attention_bound."""
import numpy as np
import pytest

from oracle import mquant_oracle as orc
from serving import D, attention_bound, make_step

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


def device_step(mq, st):
    return (dev(st["q"]), mq.PagedCache(dev(st["kp"]), dev(st["vp"]), dev(st["table"])), dev(st["start"]), dev(st["pos"]), st["hq"])


def check(st, got, rows=None, what=""):
    ref = orc.paged_attention_f64(st["q"], st["kp"], st["vp"], st["table"], st["start"], st["pos"], st["hq"], rows=rows)
    tol = attention_bound(st, ref, rows=rows)
    mine = ~np.isnan(ref[:, 0])
    got = got.cpu().numpy().astype(np.float64)
    assert np.isfinite(got[mine]).all(), what
    err = np.abs(got[mine] - ref[mine]) - tol[mine]
    worst = np.unravel_index(err.argmax(), err.shape)
    assert (err <= 0).all(), f"{what}: {np.abs(got[mine] - ref[mine])[worst]:.3e} > {tol[mine][worst]:.3e} at {worst}"
    return mine


def bounds_of(st):
    return int(np.diff(st["start"]).max(initial=0)), int(st["pos"].max(initial=0)) + 1


STEPS = {
    "one token": ([(1, 1)], 28, 4, 16),
    "two tokens": ([(1, 2)], 4, 4, 16),
    "page borders": ([(1, n) for n in (15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129)], 8, 2, 16),
    "one long": ([(1, 2500)], 28, 4, 16),
    "mixed lengths": ([(1, 700), (1, 3), (1, 1500), (1, 64), (1, 65)], 16, 2, 64),
    "large pages": ([(1, 300), (1, 1000)], 64, 8, 256),
    "every head its own": ([(1, 333), (2, 90)], 5, 5, 32),
    "one kv head": ([(1, 200), (1, 77)], 71, 1, 16),
    "drafts": ([(5, 300), (3, 90), (1, 17), (9, 9)], 28, 4, 16),
    "drafts, long": ([(5, 2100), (4, 1111)], 7, 1, 64),
    "drafts of 17 to 32 queries": ([(3, 300), (4, 1111), (1, 40), (2, 2)], 28, 4, 16),
    "24 heads on one": ([(1, 900), (1, 3), (1, 31)], 24, 1, 16),
    "a prompt": ([(130, 130)], 4, 2, 16),
    "a ragged prompt": ([(77, 77)], 28, 4, 64),
    "a chunk": ([(100, 700)], 8, 2, 16),
    "a chunk on a long cache": ([(65, 3000)], 7, 1, 32),
    "chunks": ([(33, 500), (200, 201), (17, 1000)], 12, 4, 128),
    "chunks and tokens": ([(1, 900), (150, 400), (1, 1), (0, 0), (3, 650), (64, 64)], 14, 2, 16),
    "many short": ([(1, 1 + 7 * i % 90) for i in range(150)], 4, 1, 16),
    "empty ones": ([(0, 0), (0, 40), (1, 9), (0, 0)], 4, 2, 16),
}


@pytest.mark.parametrize("name", list(STEPS))
@pytest.mark.parametrize("known", [True, False])
def test_steps(mq, name, known):
    seqs, hq, hkv, page = STEPS[name]
    rng = np.random.default_rng(sum(map(ord, name)))
    st = make_step(rng, seqs, hq, hkv, page, before=1, behind=2, spans=[(3, 20), (40, 9)] if "prompt" in name or "chunk" in name else ())
    out = torch.full((st["T"], hq * D), 7.0, dtype=torch.float16, device="cuda")
    mq.paged_attention(*device_step(mq, st), *(bounds_of(st) if known else (0, 0)), out=out)
    mine = check(st, out, what=name)
    assert (out.cpu().numpy()[~mine] == 7).all()            # rows of no sequence stay as they were


def test_seeded_sweep(mq):
    """Random steps: rows, lengths, heads, page sizes, right, low and missing bounds."""
    rng = np.random.default_rng(77)
    heads = [(1, 1), (28, 4), (8, 8), (12, 2), (9, 3), (40, 1), (16, 8), (33, 11)]
    for case in range(24):
        hq, hkv = heads[case % len(heads)]
        page = int(rng.choice([16, 32, 64, 128]))
        seqs = []
        for _ in range(int(rng.integers(1, 6))):
            n = int(rng.choice([1, 1, 2, 7, int(rng.integers(10, 160))]))
            seqs.append((n, n + int(rng.choice([0, 1, int(rng.integers(0, 60)), int(rng.integers(0, 900))]))))
        st = make_step(rng, seqs, hq, hkv, page, before=int(rng.integers(0, 3)), behind=int(rng.integers(0, 3)),
                       spans=[(1, int(rng.integers(1, 7)))])
        bounds = [bounds_of(st), (0, 0), (1, 1), (3, 200)][int(rng.integers(0, 4))]
        check(st, mq.paged_attention(*device_step(mq, st), *bounds), what=f"{case}: {seqs} {hq}/{hkv} page {page} bounds {bounds}")


def test_rows_that_see_nothing(mq):
    """Negative positions, alone and among others, with every slot of the cache NaN."""
    rng = np.random.default_rng(4)
    for rows, length in ((1, 200), (6, 200), (150, 400)):
        st = make_step(rng, [(rows, length), (rows, length)], 8, 2, 16)
        st["pos"][:rows] = -1 - np.arange(rows)
        st["pos"][rows] = -2 ** 31
        st["kp"][st["table"][0, :-1]] = np.nan                         # the first sequence's pages
        st["vp"][st["table"][0, :-1]] = np.nan
        for bounds in ((rows, length), (0, 0)):
            got = mq.paged_attention(*device_step(mq, st), *bounds)
            check(st, got, what=f"{rows} rows")
            assert (got[:rows + 1] == 0).all()


def test_positions_in_any_order_and_holes(mq):
    """Rows of a chunk in random order, some far back, equal ones among them."""
    rng = np.random.default_rng(5)
    for rows in (4, 40, 200):
        st = make_step(rng, [(rows, 600)], 7, 1, 32, poison=False)
        st["pos"][:] = rng.integers(-3, 600, rows)
        check(st, mq.paged_attention(*device_step(mq, st), rows, 600), what=f"{rows}")


def test_positions_beyond_the_table_and_pages_out_of_range(mq):
    rng = np.random.default_rng(6)
    for rows in (1, 90):
        st = make_step(rng, [(rows, 100)], 4, 2, 16, poison=False)
        st["table"] = st["table"][:, :7].copy()                         # 112 slots; the tokens take all seven pages
        st["table"][0, 2], st["table"][0, 4] = -1, 1 << 30              # page 0 is read in their place
        st["pos"][0] = 5000
        st["pos"][-1] = 2 ** 31 - 1
        check(st, mq.paged_attention(*device_step(mq, st), rows, 112), what=f"{rows} rows")


@pytest.mark.parametrize("rows", [1, 4, 130])
def test_peaked_and_flat(mq, rows):
    """Large logits of both signs (one slot takes all), equal logits, maxima that come late and early."""
    rng = np.random.default_rng(7)
    st = make_step(rng, [(rows, 1000)], 4, 2, 64, poison=False)
    for gain in (0.0, 5.0, 30.0):
        st2 = {**st, "q": (st["q"] * gain).astype(np.float16)}
        check(st2, mq.paged_attention(*device_step(mq, st2), rows, 1000), what=f"gain {gain}")
    up = st["kp"].copy()
    for s in range(1000):                                               # logits that rise along the cache
        page, r = orc.cache_slot(st["table"], 64, 0, s, len(up))
        up[page, :, r] = 0.004 * s
    st3 = {**st, "kp": up, "q": np.ones_like(st["q"])}
    check(st3, mq.paged_attention(*device_step(mq, st3), rows, 1000), what="rising")


def test_every_slot_counts(mq):
    """Values one-hot in the slot's number: output channel c is the mass of the slots c, c + 128, ..., and a slot
    skipped or taken twice shows, for single rows, drafts and chunks."""
    rng = np.random.default_rng(8)
    for rows, length, page in ((1, 128, 16), (1, 4000, 16), (6, 1500, 64), (140, 1200, 32)):
        st = make_step(rng, [(rows, length)], 8, 2, page, poison=False)
        st["q"] *= np.float16(0.2)
        for s in range(length):
            pg, r = orc.cache_slot(st["table"], page, 0, s, len(st["vp"]))
            st["vp"][pg, :, r] = np.eye(D, dtype=np.float16)[s % D]
        check(st, mq.paged_attention(*device_step(mq, st), rows, length), what=f"{rows} {length}")


def test_strides_and_streams(mq):
    """q and o as column slices with other strides, on a stream of its own."""
    rng = np.random.default_rng(9)
    for seqs in ([(1, 700), (1, 90)], [(70, 300)]):
        st = make_step(rng, seqs, 6, 2, 16)
        q, cache, start, pos, hq = device_step(mq, st)
        wide = torch.full((st["T"], 6 * D + 40), 3.0, dtype=torch.float16, device="cuda")
        wide[:, 16:16 + 6 * D] = q
        out = torch.full((st["T"], 6 * D + 20), 3.0, dtype=torch.float16, device="cuda")
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            mq.paged_attention(wide[:, 16:16 + 6 * D], cache, start, pos, hq, out=out[:, 4:4 + 6 * D])
        s.synchronize()
        check(st, out[:, 4:4 + 6 * D], what="strides")
        assert bool((out[:, :4] == 3).all()) and bool((out[:, 4 + 6 * D:] == 3).all())


def test_long_cache_sampled(mq):
    """A batch over caches of up to 12000 tokens on the 7B-class heads; every row."""
    rng = np.random.default_rng(10)
    st = make_step(rng, [(1, 12000), (1, 5), (2, 7001)], 28, 4, 64)
    check(st, mq.paged_attention(*device_step(mq, st), 2, 12000), what="long")
    st = make_step(rng, [(300, 9000)], 28, 4, 64, spans=[(20, 200)])
    rows = [0, 1, 127, 128, 199, 200, 201, 298, 299]
    check(st, mq.paged_attention(*device_step(mq, st), 300, 9000), rows=rows, what="long chunk")


def test_captured_step_follows_its_lengths(mq):
    """A captured call replayed while positions, rows per sequence and pages change under it: bounds that hold for all of
    them are enough.  Eager work runs between the replays."""
    rng = np.random.default_rng(11)
    hq, hkv, page, S, T = 14, 2, 16, 3, 3
    first = make_step(rng, [(1, 600), (1, 600), (1, 600)], hq, hkv, page, poison=False)
    q, cache, start, pos, _ = device_step(mq, first)
    ws = torch.empty(max(256, mq.paged_attention_workspace_bytes(T, cache, hq, 3, 600)), dtype=torch.uint8, device="cuda")
    out = torch.zeros((T, hq * D), dtype=torch.float16, device="cuda")
    call = lambda: mq.paged_attention(q, cache, start, pos, hq, 3, 600, out=out, workspace=ws)
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for starts, positions in (([0, 1, 2, 3], [599, 10, 300]), ([0, 3, 3, 3], [0, 1, 2]), ([0, 0, 1, 3], [64, 500, 501]),
                              ([0, 1, 1, 2], [599, 15, 7])):
        st = {**first, "start": np.array(starts, dtype=np.int32), "pos": np.array(positions, dtype=np.int32)}
        start.copy_(dev(st["start"])), pos.copy_(dev(st["pos"]))
        ws.fill_(0xff)
        out.fill_(5.0)
        g.replay()
        torch.cuda.synchronize()
        mine = check(st, out, what=f"{starts} {positions}")
        assert (out.cpu().numpy()[~mine] == 5).all()
        eager = torch.full_like(out, 5.0)
        mq.paged_attention(q, cache, start, pos, hq, 3, 600, out=eager)
        assert torch.equal(eager, out)


@pytest.mark.parametrize("seqs,hq,hkv", [([(1, 150)], 8, 8), ([(3, 40), (1, 161)], 8, 8), ([(100, 170)], 8, 8)])
def test_pages_beyond_32_bits(mq, seqs, hq, hkv):
    """Pages whose offset passes 2^31 halves (4.3 GB of pages each): the same bits as from a small cache."""
    rng = np.random.default_rng(12)
    st = make_step(rng, seqs, hq, hkv, 128, poison=False)
    q, cache, start, pos, _ = device_step(mq, st)
    small = mq.paged_attention(q, cache, start, pos, hq)
    check(st, small, what="small")
    n = (1 << 31) // (hkv * 128 * D) + len(st["kp"]) + 1
    up = n - len(st["kp"])
    big = []
    for p in (cache.k_pages, cache.v_pages):
        b = torch.zeros((n, hkv, 128, D), dtype=torch.float16, device="cuda")
        b[up:] = p
        big.append(b)
    table = torch.where(cache.page_table >= 0, cache.page_table + up, cache.page_table)
    assert torch.equal(mq.paged_attention(q, mq.PagedCache(*big, table), start, pos, hq), small)


def test_results_repeat_and_two_streams_run_at_once(mq):
    """The same bits every time, also with other calls on another stream beside them (each with a workspace of its own)."""
    rng = np.random.default_rng(13)
    for seqs in ([(1, 1500), (1, 200)], [(4, 900)], [(90, 1100), (1, 700)]):
        st = make_step(rng, seqs, 14, 2, 16)
        t = device_step(mq, st)
        want = mq.paged_attention(*t, *bounds_of(st))
        check(st, want, what="alone")
        streams = [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        outs = []
        for _ in range(10):
            for s in streams:
                with torch.cuda.stream(s):
                    outs.append(mq.paged_attention(*t, *bounds_of(st)))
        torch.cuda.synchronize()
        mine = torch.from_numpy(np.concatenate([np.arange(a, b) for a, b in zip(st["start"], st["start"][1:])])).cuda()
        assert all(torch.equal(o[mine], want[mine]) for o in outs)


def test_two_graphs_that_share_a_workspace(mq):
    """A decode step and a chunk captured with the same scratch memory and replayed in turn, eager work between."""
    rng = np.random.default_rng(14)
    steps = [make_step(rng, seqs, 14, 2, 16, poison=False) for seqs in ([(1, 1500), (1, 900)], [(60, 1500)])]
    args = [(*device_step(mq, st), *bounds_of(st)) for st in steps]
    need = max(mq.paged_attention_workspace_bytes(a[0].shape[0], a[1], 14, *a[5:]) for a in args)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    outs, graphs = [torch.zeros_like(a[0]) for a in args], []
    for a, o in zip(args, outs):
        mq.paged_attention(*a, out=o, workspace=ws)
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            mq.paged_attention(*a, out=o, workspace=ws)
    for rep in range(3):
        for st, a, o, g in zip(steps, args, outs, graphs):
            o.zero_()
            g.replay()
            check(st, o, what=f"replay {rep}")
            assert torch.equal(mq.paged_attention(*a), o)


@pytest.mark.parametrize("seqs,hq,hkv,page", [
    ([(13 + i % 5, 13 + 11 * i % 300) if i % 7 else (0, 9) for i in range(70)], 4, 1, 16), ([(1, 5000), (1, 4096), (3, 4097)], 4, 2, 4096),
    ([(40, 2500), (1, 2048)], 7, 1, 2048), ([(1, 30)] * 130 + [(20, 90)] + [(2, 8)] * 5, 6, 2, 16)])
def test_many_chunks_and_large_pages(mq, seqs, hq, hkv, page):
    """More sequences than a wave sorts, some without rows, and the largest pages."""
    seqs = [(n, max(n, length)) for n, length in seqs]
    st = make_step(np.random.default_rng(len(seqs)), seqs, hq, hkv, page, behind=1)
    for bounds in (bounds_of(st), (0, 0), (1, 1)):
        check(st, mq.paged_attention(*device_step(mq, st), *bounds), what=f"{len(seqs)} {bounds}")


def test_sequences_that_share_pages(mq):
    """Two sequences with the same first pages: a prompt that both continue."""
    st = make_step(np.random.default_rng(18), [(1, 700), (5, 600), (60, 640)], 14, 2, 16)
    st["table"][1, :20], st["table"][2, :30] = st["table"][0, :20], st["table"][0, :30]
    check(st, mq.paged_attention(*device_step(mq, st), *bounds_of(st)))


def test_queries_of_rows_that_see_nothing_may_be_anything(mq):
    for seqs in ([(6, 300)], [(1, 40), (90, 700)]):
        st = make_step(np.random.default_rng(19), seqs, 7, 1, 16, behind=2)
        blind = np.arange(0, st["T"] - 2, 5)
        st["pos"][blind] = -1
        clean = {**st, "q": st["q"].copy()}
        st["q"][blind], st["q"][-2:] = np.nan, np.inf
        out = mq.paged_attention(*device_step(mq, st), *bounds_of(st))
        check(clean, out, what=f"{seqs}")
        assert (out[torch.from_numpy(blind).cuda()] == 0).all()


def test_nothing_to_do(mq):
    """No rows, and no sequences."""
    st = make_step(np.random.default_rng(20), [(0, 40), (0, 3)], 4, 2, 16)
    q, cache, start, pos, hq = device_step(mq, st)
    assert mq.paged_attention(q, cache, start, pos, hq).shape == (0, 4 * D)
    none = mq.PagedCache(cache.k_pages, cache.v_pages, cache.page_table[:0])
    x = torch.ones((3, 4 * D), dtype=torch.float16, device="cuda")
    at = torch.zeros(3, dtype=torch.int32, device="cuda")
    out = torch.full_like(x, 5)
    assert (mq.paged_attention(x, none, start[:1], at, 4, out=out) == 5).all()
    assert (mq.kv_append(x, x[:, :2 * D], x[:, :2 * D], none, start[:1], at, 4, q_out=out) == 5).all()
    before = cache.k_pages.clone()
    assert mq.kv_append(q, q[:, :2 * D], q[:, :2 * D], cache, start, pos, 4).shape == (0, 4 * D)
    assert torch.equal(cache.k_pages.view(torch.int16), before.view(torch.int16))


def test_large_logits(mq):
    """Logits up to 2.96e6 (sums that are exact in fp32, 2896 apart where they differ): the mean over the slots of the largest one.  Their
    probabilities are equal, so the sum over them is off by the fp32 accumulation (1024 slots of 2^-24 of the largest value) and by the
    rounding of the output."""
    rng = np.random.default_rng(17)
    for seqs, hq, hkv in ([(1, 700), (1, 64)], 28, 4), ([(4, 500)], 7, 1), ([(130, 900)], 4, 2):
        st = make_step(rng, seqs, hq, hkv, 16)
        sign = rng.choice([-1.0, 1.0], D)
        st["q"][:] = np.tile(256 * sign, hq)
        steps = rng.integers(-1024, 1025, st["kp"].shape[:3]).astype(np.float64)
        steps[rng.random(steps.shape) < 0.05] = 1024
        st["kp"][:] = np.where(np.isnan(st["kp"]) | np.isinf(st["kp"]), st["kp"], (steps[..., None] * sign).astype(np.float16))
        ref = orc.paged_attention_f64(st["q"], st["kp"], st["vp"], st["table"], st["start"], st["pos"], hq)
        got = mq.paged_attention(*device_step(mq, st), *bounds_of(st)).cpu().numpy().astype(np.float64)
        top = np.abs(np.nan_to_num(st["vp"].astype(np.float64), nan=0, posinf=0)).max()
        assert (np.abs(got - ref) <= 2.0 ** -11 * np.abs(ref) + 2.0 ** -25 + 2.0 ** -14 * top).all()


@pytest.mark.parametrize("n,spans", [(77, [(5, 30)]), (300, [(0, 64), (100, 130)]), (1, []), (640, [])])
def test_a_prompt_as_the_attention_without_a_cache_sees_it(mq, n, spans):
    """One whole prompt in AIFS order: the unified mask over its rows and the slots by position are the same sum.  Each side is off by its
    own bound: this one's, and 1.5 * 2^-11 (sum p |v| + |o|) + 1e-6 of the other."""
    st = make_step(np.random.default_rng(n), [(n, n)], 14, 2, 16, spans=spans, poison=False)
    q, cache, start, pos, hq = device_step(mq, st)
    at = st["table"][0, st["pos"] // 16], st["pos"] % 16
    k, v = (dev(st[p][at[0], :, at[1]].reshape(n, -1)) for p in ("kp", "vp"))       # rows in AIFS order
    ref = orc.paged_attention_f64(st["q"], st["kp"], st["vp"], st["table"], st["start"], st["pos"], hq)
    mass = orc.paged_attention_f64(st["q"], st["kp"], np.abs(st["vp"]), st["table"], st["start"], st["pos"], hq)
    tol = attention_bound(st, ref) + 1.5 * 2.0 ** -11 * (mass + np.abs(ref)) + 1e-6
    a, b = (o.cpu().numpy().astype(np.float64) for o in (mq.paged_attention(q, cache, start, pos, hq, n, n), mq.aifs_attention(q, k, v, pos, hq, 2)))
    assert (np.abs(a - b) <= tol).all()


@pytest.mark.parametrize("fill", [float("nan"), float("inf"), float("-inf"), 3e38])
def test_scratch_holds_anything(mq, fill):
    """What a workspace held before the call leaves no trace: sequences with fewer pieces than the longest one among them."""
    rng = np.random.default_rng(16)
    for seqs, hq, hkv in ([(1, 3000), (1, 130), (1, 900)], 28, 4), ([(5, 2500), (4, 300), (3, 129)], 28, 4), ([(3, 2500), (3, 257)], 28, 4), \
            ([(60, 2600), (50, 90), (40, 1200)], 7, 1), ([(60, 2600), (1, 1200), (2, 5)], 8, 2):
        st = make_step(rng, seqs, hq, hkv, 16)
        need = mq.paged_attention_workspace_bytes(st["T"], device_step(mq, st)[1], hq, *bounds_of(st))
        assert need > 0
        ws = torch.full((need // 4,), fill, dtype=torch.float32, device="cuda")
        check(st, mq.paged_attention(*device_step(mq, st), *bounds_of(st), workspace=ws), what=f"{seqs} {fill}")


def test_routes(mq):
    """Which kernels a step's bounds choose: few queries, chunks, both, and the join of pieces where slots are split."""
    from kernel_trace import kernels
    rng = np.random.default_rng(15)
    for seqs, hq, hkv, bounds, want in [
            ([(1, 100)], 28, 4, True, ["paged_few_kernel<1>"]), ([(1, 1281)], 28, 4, True, ["paged_few_kernel<1>", "paged_combine_kernel<false>"]),
            ([(5, 300)], 28, 4, True, ["paged_few_kernel<3>", "paged_combine_kernel<false>"]),
            ([(7, 60)], 28, 4, True, ["paged_chunk_kernel<2>"]), ([(1300, 1300)], 28, 4, True, ["paged_chunk_kernel<1>"]),
            ([(20, 3000)], 28, 4, True, ["paged_chunk_kernel<2>", "paged_combine_kernel<true>"]),
            ([(100, 200), (1, 100)], 4, 2, False, ["paged_chunk_kernel<2>", "paged_few_kernel<3>", "paged_combine_kernel<false>"])]:
        st = make_step(rng, seqs, hq, hkv, 16, poison=False)
        args = (*device_step(mq, st), *(bounds_of(st) if bounds else (0, 0)))
        names = kernels(lambda: mq.paged_attention(*args))
        assert [n for n in names if "paged" in n] == want, (seqs, names)


@pytest.mark.parametrize("seqs,hq,hkv,slope,rows", [
    ([(1, 200), (1, 70)], 28, 4, 400, None), ([(1, 1281)], 28, 4, 400, None), ([(5, 2500), (4, 300)], 28, 4, 30, None),
    ([(60, 256)], 7, 1, 400, None), ([(40, 2000), (1, 700)], 8, 2, 30, None), ([(1300, 1300)], 28, 4, 4, [0, 700, 1023, 1024, 1298, 1299])])
def test_large_logits_that_differ_by_single_steps(mq, seqs, hq, hkv, slope, rows):
    """Scores are whole numbers of about 8e6 and exact in fp32 (logits 6.8e5 to 7.4e5): what waves, key groups, pieces and tiles have seen last
    differs by a few of them, and what each adds to the sum has to be scaled alike.  Values are one-hot in the slot's number, so that the
    channels of a result are the shares of the parts: in its lowest bits, then in its highest ones.  Probabilities are off by half a
    step each (2^-11, 2^-25 in the subnormal range), in the numerator and in the denominator, the output by another, the fp32 sums by 2^-14."""
    rng = np.random.default_rng(len(seqs) + slope)
    st = make_step(rng, seqs, hq, hkv, 16, poison=False)
    q = np.ones((st["T"], hq, D), dtype=np.float16)
    q[:, :, :127] = (256 - np.arange(hq) % 20)[None, :, None]           # a head's scores: (256 - h) * 256 * 127 + the slot's step
    st["q"] = q.reshape(st["T"], hq * D)
    st["kp"][..., :127] = 256
    longest = max(n for _, n in seqs)
    for high in (False, True):
        for s, (_, length) in enumerate(seqs):
            for i in range(length):
                page, r = orc.cache_slot(st["table"], 16, s, i, len(st["vp"]))
                st["kp"][page, :, r, 127] = i // slope + 2 * (i // 32 % 4) + rng.integers(0, 3)
                st["vp"][page, :, r] = np.eye(D, dtype=np.float16)[i * D // longest if high else i % D]
        ref = orc.paged_attention_f64(st["q"], st["kp"], st["vp"], st["table"], st["start"], st["pos"], hq, rows=rows)
        got = mq.paged_attention(*device_step(mq, st), *bounds_of(st)).cpu().numpy().astype(np.float64)
        mine = ~np.isnan(ref[:, 0])
        tol = (3 * 2.0 ** -11 + 2.0 ** -14) * ref + 2.0 ** -25 * (1 + 2 * longest)
        err = np.abs(got - ref)[mine] - tol[mine]
        worst = np.unravel_index(err.argmax(), err.shape)
        assert (err <= 0).all(), f"high {high}: {(err + tol[mine])[worst]:.3e} > {tol[mine][worst]:.3e} at {worst}"


@pytest.mark.parametrize("seqs,hq,hkv", [([(1, 1 + 5 * i % 60) for i in range(128)], 8, 8), ([(1, 300), (3, 40)], 28, 4), ([(40, 300), (1, 9)], 8, 8)])
def test_bounds_beyond_the_table(mq, seqs, hq, hkv):
    """Bounds up to the largest number: the same bits as with the table's own slots."""
    st = make_step(np.random.default_rng(len(seqs)), seqs, hq, hkv, 16)
    t = device_step(mq, st)
    want = mq.paged_attention(*t, 0, t[1].slots)
    check(st, want, what="the table's slots")
    mine = torch.from_numpy(np.concatenate([np.arange(a, b) for a, b in zip(st["start"], st["start"][1:])])).cuda()
    for max_kv in (0, t[1].slots + 1, 2 ** 31 - 128, 2 ** 31 - 1, 2 ** 33):
        assert torch.equal(mq.paged_attention(*t, 0, max_kv)[mine], want[mine])
