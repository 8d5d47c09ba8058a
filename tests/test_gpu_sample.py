"""The next token of rows of logits against the definition in fp64: tokens equal, log-probabilities within what is rounded.

A log-probability is (l - m) / t - ln S: the result rounded to fp32 (2^-24 of it), S a sum of V whole multiples of 2^-43 (V * 2^-44 off, of at
least 1) of weights that are off by 2^-38.7 of themselves, twice where a part of the row is summed against its own largest logit first: less
than 2^-37 of S, so 2^-37 of ln S; (l - m) / t and the logarithm in double (2^-43 covers them)."""
import numpy as np
import pytest

from oracle import mquant_oracle as orc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
NEXT = np.nextafter(np.float32(1), np.float32(0))


@pytest.fixture(scope="module")
def mq():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2502_00425_amd import binding
    return binding


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def check(mq, logits, t, k, p, m, u, dtype=torch.float16, what=""):
    """logits [rows, V] as numpy of the type; settings a row."""
    rows, V = logits.shape
    full = lambda x, d: np.broadcast_to(np.asarray(x, dtype=d), (rows,)).copy()
    t, k, p, m, u = full(t, np.float32), full(k, np.int32), full(p, np.float32), full(m, np.float32), full(u, np.float32)
    token, logprob = (x.cpu().numpy() for x in mq.sample(dev(logits), dev(t), dev(k), dev(p), dev(m), dev(u)))
    for r in range(rows):
        want, lp = orc.sample_f64(logits[r].astype(np.float64), float(t[r]), int(k[r]), float(p[r]), float(m[r]), float(u[r]))
        assert token[r] == want, f"{what} row {r}: {token[r]}, not {want} ({t[r]} {k[r]} {p[r]} {m[r]} {u[r]})"
        if want < 0:
            assert logprob[r] == -np.inf
        else:
            assert abs(float(logprob[r]) - lp) <= 2.0 ** -24 * abs(lp) + V * 2.0 ** -44 + 2.0 ** -37, f"{what} row {r}: {logprob[r]} {lp}"


def logits_of(rng, rows, V, dtype, kind="model"):
    x = {"model": lambda: 3 - 1.1 * np.log(1e-9 + rng.random((rows, V))) + 0.5 * rng.standard_normal((rows, V)),
         "flat": lambda: 0.3 * rng.standard_normal((rows, V)), "equal": lambda: np.full((rows, V), 2.5),
         "two": lambda: rng.choice([1.0, 1.5], (rows, V)), "wide": lambda: 300 * rng.standard_normal((rows, V)),
         "normal": lambda: 2.5 * rng.standard_normal((rows, V))}[kind]()
    return x.astype(np.float16 if dtype == torch.float16 else np.float32)


SETTINGS = [(0.0, 0, 1.0, 0.0), (1.0, 0, 1.0, 0.0), (0.7, 0, 0.9, 0.0), (1.3, 50, 1.0, 0.0), (1.0, 0, 1.0, 0.05), (0.8, 40, 0.95, 0.02),
            (1.0, 1, 1.0, 0.0), (1.0, 0, 1e-6, 0.0), (1.0, 0, 0.0, 0.0), (1.0, 0, 1.0, 1.0), (1.0, 0, 1.0, 3.0), (1.0, 10 ** 9, 1.5, -1.0),
            (1.0, -5, float("nan"), float("nan")), (float("nan"), 3, 0.5, 0.0), (-1.0, 0, 1.0, 0.0), (100.0, 0, 0.5, 0.0), (100.0, 1500, 0.7, 0.1),
            (100.0, 5000, 0.7, 0.0), (0.01, 0, 0.99, 0.0), (1e-30, 0, 1.0, 0.0), (1e30, 7, 0.5, 0.0), (float("inf"), 0, 1.0, 0.0),
            (2.0, 2048, 1.0, 0.0), (2.0, 2049, 0.999, 0.0), (1.0, 0, float(NEXT), 1e-30)]


@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 63, 64, 65, 511, 513, 1000, 2048, 2049, 8191, 32000, 50001])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_settings(mq, V, dtype):
    rng = np.random.default_rng(V)
    rows = len(SETTINGS)
    x = logits_of(rng, rows, V, dtype)
    check(mq, x, *zip(*SETTINGS), rng.random(rows, dtype=np.float32), dtype, f"V={V}")


@pytest.mark.parametrize("kind", ["flat", "equal", "two", "wide", "normal"])
@pytest.mark.parametrize("V", [100, 5000, 40001])
@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_distributions(mq, kind, V, dtype):
    rng = np.random.default_rng(V + len(kind))
    x = logits_of(rng, len(SETTINGS), V, dtype, kind)
    check(mq, x, *zip(*SETTINGS), rng.random(len(SETTINGS), dtype=np.float32), dtype, kind)


@pytest.mark.parametrize("args", [(1.0, 0, 1.0, 0.0), (1.0, 30, 1.0, 0.0), (2.0, 0, 0.8, 0.0), (1.0, 0, 1.0, 0.01), (50.0, 6000, 0.9, 0.0)])
def test_every_part_of_the_interval(mq, args):
    """Random numbers from 0 to the one below 1, and those outside."""
    rng = np.random.default_rng(2)
    u = np.concatenate([[0.0, 1e-30, 2.0 ** -24, 0.5, 1 - 2.0 ** -24, NEXT, 1.0, 7.0, -0.5, np.nan], rng.random(54)]).astype(np.float32)
    x = np.repeat(logits_of(rng, 1, 9001, torch.float16), len(u), axis=0)
    check(mq, x, *args, u)


def test_probabilities_that_fill_top_p_exactly(mq):
    """Equal probabilities 1/8: those that end exactly at top_p are kept and no more; ties at the end of top-k and top-p go to the lowest."""
    x = np.full((9, 3000), -np.inf, dtype=np.float16)
    x[:, 5:2805:350] = 1.0
    u = np.full(9, NEXT)
    for p, want in ((0.125, 0), (0.25, 1), (0.5, 3), (0.625, 4), (0.875, 6), (1.0, 7)):
        token, _ = mq.sample(dev(x), None, None, dev(np.full(9, p, np.float32)), None, dev(u.astype(np.float32)))
        assert (token.cpu().numpy() == 5 + 350 * want).all(), p
        check(mq, x, 1.0, 0, p, 0.0, u)
    for k in range(1, 10):
        check(mq, x, 1.0, k, 1.0, 0.0, u)
        check(mq, x, 1.0, k, 0.5, 0.0, u)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_masked_and_infinite_logits(mq, dtype):
    rng = np.random.default_rng(5)
    n = len(SETTINGS)
    x = logits_of(rng, n, 3001, dtype)
    low = np.finfo(x.dtype).min
    cases = {}
    y = x.copy()
    y[:, rng.random(3001) < 0.5] = -np.inf
    y[:, ::7] = np.nan
    cases["masked"] = y
    y = np.full_like(x, -np.inf)
    y[:, 1234] = -3.0
    cases["one is left"] = y
    cases["none is left"] = np.full_like(x, -np.inf)
    cases["nothing but NaN"] = np.full_like(x, np.nan)
    y = x.copy()
    y[:, 50:90:3] = np.inf
    cases["infinite"] = y
    y = np.full_like(x, low)
    y[:, 77], y[:, 99] = 0.0, -0.0
    cases["lowest values and both zeros"] = y
    cases["lowest values only"] = np.full_like(x, low)
    y = x.copy()
    y[:, 10], y[:, 20], y[:, 30] = -low, low, 6e-8
    cases["largest values"] = y
    for what, y in cases.items():
        with np.errstate(all="ignore"):
            check(mq, y, *zip(*SETTINGS), rng.random(n, dtype=np.float32), dtype, what)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_rows_at_any_address(mq, dtype):
    """Rows of an odd width, views into wider rows that hold infinities on both sides."""
    rng = np.random.default_rng(6)
    n = len(SETTINGS)
    for off in range(9):
        buf = np.full((n, 1000 + 21), np.inf, dtype=np.float16 if dtype == torch.float16 else np.float32)
        x = logits_of(rng, n, 997, dtype)
        buf[:, off:off + 997] = x
        view = dev(buf)[:, off:off + 997]
        u = rng.random(n, dtype=np.float32)
        cols = [dev(np.asarray(c, d)) for c, d in zip(zip(*SETTINGS), (np.float32, np.int32, np.float32, np.float32))]
        a = mq.sample(view, *cols, dev(u))
        b = mq.sample(dev(x), *cols, dev(u))
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    check(mq, x, *zip(*SETTINGS), u, dtype)


def test_long_vocabularies(mq):
    rng = np.random.default_rng(7)
    some = [SETTINGS[i] for i in (1, 2, 3, 5, 15, 17, 24)]
    for V, dtype in ((150001, torch.float16), (1 << 20, torch.float16), (1 << 20, torch.float32), ((1 << 20) - 3, torch.float32)):
        for kind in ("model", "equal", "normal"):
            check(mq, logits_of(rng, len(some), V, dtype, kind), *zip(*some), rng.random(len(some), dtype=np.float32), dtype, f"{V} {kind}")


def test_many_rows(mq):
    rng = np.random.default_rng(8)
    x = logits_of(rng, 700, 1201, torch.float16)
    some = [SETTINGS[i % len(SETTINGS)] for i in range(700)]
    check(mq, x, *zip(*some), rng.random(700, dtype=np.float32))


def test_defaults_and_no_rows(mq):
    x = dev(np.zeros((3, 10), np.float16))
    u = dev(np.array([0.0, 0.55, 0.95], np.float32))
    token, logprob = mq.sample(x, None, None, None, None, u)
    assert token.tolist() == [0, 5, 9] and torch.allclose(logprob, torch.full((3,), -float(np.log(10.0)), device="cuda"))
    token, _ = mq.sample(x[:0], None, None, None, None, u[:0])
    assert token.shape == (0,)
    t = torch.full((3,), 9, dtype=torch.int32, device="cuda")
    assert mq.lib.mquant_sample(x.data_ptr(), mq.F16, 10, None, None, None, None, u.data_ptr(), t.data_ptr(), None, 3, 10, None, 0,
                                None) in (mq.OK, mq.ERR_WORKSPACE)
    torch.cuda.synchronize()


def test_how_often_tokens_come(mq):
    """20000 rows of the same five logits with evenly spread random numbers: each token as often as its probability says, to a row."""
    n = 20000
    x = np.repeat(np.log([[0.4, 0.05, 0.3, 0.2, 0.05]]), n, axis=0).astype(np.float32)
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    token, _ = mq.sample(dev(x), None, None, None, None, dev(u))
    count = np.bincount(token.cpu().numpy(), minlength=5)
    assert (np.abs(count - n * np.array([0.4, 0.05, 0.3, 0.2, 0.05])) <= 1).all()


def test_replays_and_streams(mq):
    rng = np.random.default_rng(10)
    n, V = len(SETTINGS), 30001
    x, u = dev(logits_of(rng, n, V, torch.float16)), dev(rng.random(n, dtype=np.float32))
    cols = [dev(np.asarray(c, d)) for c, d in zip(zip(*SETTINGS), (np.float32, np.int32, np.float32, np.float32))]
    out, lp = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.float32, device="cuda")
    need = mq.sample_workspace_bytes(n, V)
    ws = torch.full((max(need, 256),), 255, dtype=torch.uint8, device="cuda")
    call = lambda **kw: mq.sample(x, *cols, u, **kw)
    call(out=out, logprob=lp, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out=out, logprob=lp, workspace=ws)
    for step in range(4):
        x.copy_(dev(logits_of(rng, n, V, torch.float16, ["model", "flat", "equal", "normal"][step])))
        u.copy_(dev(rng.random(n, dtype=np.float32)))
        graph.replay()
        got = out.clone(), lp.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            want = call()
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_lists_of_every_length(mq, dtype):
    """As many kept tokens as a way of drawing takes at most, one less and one more: by their number, by their weight and as equals."""
    rng = np.random.default_rng(11)
    V = 9000
    lengths = [1, 2, 15, 16, 17, 63, 64, 65, 127, 129, 255, 256, 257, 511, 513, 1023, 1024, 1025, 2047, 2048, 2049, 4095, 4097]
    for kind in ("steps", "equal ahead", "near"):
        x = np.full((len(lengths), V), -12.0)
        for r, n in enumerate(lengths):
            ahead = rng.permutation(V)[:n]
            x[r, ahead] = {"steps": 4 - 0.002 * np.arange(n), "equal ahead": np.full(n, 2.0), "near": rng.uniform(1.9, 2.1, n)}[kind]
            x[r] += {"steps": 1, "equal ahead": 0, "near": 0}[kind] * rng.uniform(0, 1e-3, V)
        x = x.astype(np.float16 if dtype == torch.float16 else np.float32)
        n, u = np.array(lengths), rng.random(len(lengths), dtype=np.float32)
        check(mq, x, 1.0, n, 1.0, 0.0, u, dtype, kind)
        check(mq, x, 1.0, n, 0.9, 0.0, u, dtype, kind + " top-p")
        check(mq, x, 1.0, n + 5, 1.0, 0.01, u, dtype, kind + " min-p")
        check(mq, x, 1.0, 0, 1.0, 0.0001, u, dtype, kind + " min-p alone")
        check(mq, x, 0.5, 0, 0.97, 0.0, u, dtype, kind + " top-p alone")
        check(mq, x, 0.5, 0, 0.99, 0.2, u, dtype, kind + " top-p and min-p")
        check(mq, x, 1.0, n, 0.99, 0.0, NEXT, dtype, kind + " the last")


def test_kept_tokens_without_weight(mq):
    """Top-k keeps tokens whose weight is nothing beside the first ones: they hold no part of the interval, wherever they lie."""
    x = np.full((8, 700), -60000.0, dtype=np.float16)
    x[:, 300], x[:, 500], x[:, 20] = 5.0, 4.0, 4.5
    u = np.array([0, 0.1, 0.3, 0.4, 0.5, 0.9, 0.99, NEXT], dtype=np.float32)
    for k in (2, 3, 4, 50, 200, 600):
        check(mq, x, 1.0, k, 1.0, 0.0, u)
        check(mq, x, 1.0, k, 0.9999, 0.0, u)


def test_scratch_of_a_larger_call_with_anything_in_it(mq):
    rng = np.random.default_rng(12)
    n = len(SETTINGS)
    ws = torch.empty(mq.sample_workspace_bytes(64, 70000), dtype=torch.uint8, device="cuda")
    cols = [dev(np.asarray(c, d)) for c, d in zip(zip(*SETTINGS), (np.float32, np.int32, np.float32, np.float32))]
    for V in (5, 3000, 50000):
        x, u = dev(logits_of(rng, n, V, torch.float32)), dev(rng.random(n, dtype=np.float32))
        want = mq.sample(x, *cols, u)
        for fill in (0, 0x7f, 0xff):
            ws.fill_(fill)
            got = mq.sample(x, *cols, u, workspace=ws)
            assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_rows_beyond_32_bits(mq):
    """2100 rows of 2^20 logits: the last ones are drawn as they are alone; what is behind them is no row."""
    rng = np.random.default_rng(13)
    V, rows = 1 << 20, 2100
    x = torch.zeros((rows, V), dtype=torch.float16, device="cuda")
    some = dev(logits_of(rng, 3, V, torch.float16))
    x[-3:] = some
    u = dev(rng.random(rows, dtype=np.float32))
    for args in ((None, None, None, None), (None, 50, None, None), (None, None, 0.6, None)):
        full = lambda c, d, n: None if c is None else torch.full((n,), c, dtype=d, device="cuda")
        cols = lambda n: [full(c, d, n) for c, d in zip(args, (torch.float32, torch.int32, torch.float32, torch.float32))]
        token, logprob = mq.sample(x, *cols(rows), u)
        alone = mq.sample(some, *cols(3), u[-3:].contiguous())
        assert torch.equal(token[-3:], alone[0]) and torch.equal(logprob[-3:], alone[1])
        if args[1] is None and args[2] is None:
            assert token[:-3].cpu().numpy().tolist() == np.floor(u[:-3].cpu().numpy().astype(np.float64) * V).astype(int).tolist()


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_bins_of_every_length(mq, dtype):
    """As many tokens in the bin that top-p cuts as are held there, one less and one more, among long lists."""
    rng = np.random.default_rng(14)
    V = 60000
    for n in (2000, 8191, 8192, 8193, 20000):
        x = rng.uniform(-9.0, -4.0, (5, V))
        for r in range(5):
            x[r, rng.permutation(V)[:n]] = -0.01 * rng.random(n) if r < 3 else 0.25
        x = x.astype(np.float16 if dtype == torch.float16 else np.float32)
        u = np.array([0.0, 0.3, 0.7, NEXT, 0.5], dtype=np.float32)
        for p in (0.3, 0.6, 0.9, 0.99):
            check(mq, x, 1.0, 0, p, 0.0, u, dtype, f"{n} {p}")
        check(mq, x, 1.0, n - 100, 0.9, 0.0, u, dtype, f"{n} by both")
        check(mq, x, 1.0, n + 100, 0.999, 1e-3, u, dtype, f"{n} and by weight")


def test_two_graphs_that_share_a_workspace_and_two_streams_at_once(mq):
    """Steps of other sizes and settings in turn on the same scratch; then both at once on two streams, each with its own: the same bits."""
    rng = np.random.default_rng(15)
    ws = torch.full((mq.sample_workspace_bytes(70, 60000),), 255, dtype=torch.uint8, device="cuda")
    steps = []
    for rows, V, dtype, kind in ((70, 9001, torch.float16, "model"), (25, 60000, torch.float32, "normal")):
        x, u = dev(logits_of(rng, rows, V, dtype, kind)), dev(rng.random(rows, dtype=np.float32))
        cols = [dev(np.resize(np.asarray(c, d), rows)) for c, d in zip(zip(*SETTINGS), (np.float32, np.int32, np.float32, np.float32))]
        out, lp = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.zeros(rows, dtype=torch.float32, device="cuda")
        want = mq.sample(x, *cols, u)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            mq.sample(x, *cols, u, out, lp, ws)
        steps.append((graph, (x, *cols, u), out, lp, want))
    for _ in range(3):
        for graph, _, out, lp, want in steps:
            out.fill_(-5), lp.fill_(5.0)
            graph.replay()
            assert torch.equal(out, want[0]) and torch.equal(lp, want[1])
    streams = [torch.cuda.Stream() for _ in steps]
    torch.cuda.synchronize()
    got = []
    for stream, (_, args, _, _, _) in zip(streams, steps):
        with torch.cuda.stream(stream):
            got.append([mq.sample(*args) for _ in range(20)])
    torch.cuda.synchronize()
    for results, (_, _, _, _, want) in zip(got, steps):
        assert all(torch.equal(a, want[0]) and torch.equal(b, want[1]) for a, b in results)
