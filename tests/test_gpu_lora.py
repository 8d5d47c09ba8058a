"""Adapters of many requests beside a shared linear against the fp64 oracle.

Tolerance per element: the fp16 result is off by half a step, 2^-11 |y| and 2^-25 among subnormals.  The intermediate is an
fp32 sum of K exact products whose accumulator takes at least 8 of them an addition, (K / 8 + 16) * 2^-24 of the
sum of their magnitudes; carried into the second product as two fp16 parts it loses another 2^-21; that product's sum adds
(rank + 4) * 2^-24 of its magnitudes."""
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


def make(rng, T, K, N, rank, n, ids=None, gain=1.0):
    return {"x": (rng.standard_normal((T, K)) * gain).astype(np.float16),
            "a": (rng.standard_normal((n, rank, K)) / np.sqrt(K)).astype(np.float16),
            "b": (rng.standard_normal((n, N, rank)) / np.sqrt(rank)).astype(np.float16),
            "scale": rng.uniform(-2, 2, n).astype(np.float32), "base": rng.standard_normal((T, N)).astype(np.float16),
            "ids": (rng.integers(-1, n + 1, T) if ids is None else np.asarray(ids)).astype(np.int32), "perm": None}


def check(c, got, what=""):
    ref = orc.lora_f64(c["x"], c["perm"], c["ids"], c["a"], c["b"], c["scale"], c["base"])
    a, b, x = (np.abs(c[k].astype(np.float64)) for k in "abx")
    K, rank = a.shape[2], a.shape[1]
    size = orc.lora_f64(x, c["perm"], c["ids"], a, b, np.abs(c["scale"].astype(np.float64)), np.zeros_like(c["base"], dtype=np.float64))
    tol = 2.0 ** -11 * np.abs(ref) + 2.0 ** -25 + ((K / 8 + 16 + rank + 4) * 2.0 ** -24 + 2.0 ** -21) * size
    got = got.cpu().numpy().astype(np.float64)
    assert np.isfinite(got).all(), what
    err = np.abs(got - ref) - tol
    worst = np.unravel_index(err.argmax(), err.shape)
    assert (err <= 0).all(), f"{what}: {np.abs(got - ref)[worst]:.3e} > {tol[worst]:.3e} at {worst}"
    none = (c["ids"] < 0) | (c["ids"] >= len(c["scale"]))
    assert np.array_equal(got[none], c["base"].astype(np.float64)[none])


def call(mq, c, **kw):
    return mq.lora_apply(dev(c["x"]), dev(c["ids"]), dev(c["a"]), dev(c["b"]), dev(c["scale"]), dev(c["base"]),
                         perm_dev=None if c["perm"] is None else dev(c["perm"]), **kw)


@pytest.mark.parametrize("T,K,N,rank,n", [
    (1, 8, 1, 8, 1), (1, 64, 16, 16, 1), (1, 3584, 4608, 16, 3), (2, 72, 100, 24, 2), (4, 3584, 512, 8, 4), (5, 520, 333, 40, 3),
    (16, 512, 640, 16, 16), (17, 512, 640, 64, 4), (33, 1000, 130, 128, 5), (48, 4096, 264, 16, 12), (64, 640, 31, 32, 2),
    (100, 264, 257, 56, 7), (150, 2048, 512, 64, 3), (257, 136, 72, 16, 40), (300, 512, 1032, 128, 2)])
def test_sizes(mq, T, K, N, rank, n):
    c = make(np.random.default_rng(T + K + N), T, K, N, rank, n)
    check(c, call(mq, c), what=f"{T} {K} {N} r{rank}")


@pytest.mark.parametrize("ids", ["one", "none", "runs", "each its own", "alternating", "last row only"])
def test_who_has_which_adapter(mq, ids):
    T, n = 133, 20
    rows = {"one": np.full(T, 3), "none": np.where(np.arange(T) % 2, -1, n), "runs": np.arange(T) // 50, "each its own": np.arange(T) % n,
            "alternating": np.where(np.arange(T) % 2, 0, 19), "last row only": np.where(np.arange(T) == T - 1, 5, -5)}[ids]
    c = make(np.random.default_rng(1), T, 384, 272, 16, n, ids=rows)
    check(c, call(mq, c), what=ids)


@pytest.mark.parametrize("T", [6, 140])
def test_reordered_rows(mq, T):
    """x in original order, y in AIFS order; an index out of range reads row 0."""
    rng = np.random.default_rng(2)
    c = make(rng, T, 256, 320, 16, 3)
    c["perm"] = orc.aifs_build_perm(T, [(1, T // 2)])[0].copy()
    c["perm"][2], c["perm"][T - 1] = -1, T
    check(c, call(mq, c), what="perm")


def test_in_place_strides_and_streams(mq):
    rng = np.random.default_rng(3)
    for T, N in ((3, 96), (70, 96), (70, 91)):
        c = make(rng, T, 128, N, 16, 4)
        xw = torch.zeros((T, 200), dtype=torch.float16, device="cuda")
        xw[:, 8:136] = dev(c["x"])
        y = torch.full((T, N + 21), 2.0, dtype=torch.float16, device="cuda")
        y[:, 5:5 + N] = dev(c["base"])
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            mq.lora_apply(xw[:, 8:136], dev(c["ids"]), dev(c["a"]), dev(c["b"]), dev(c["scale"]), y[:, 5:5 + N], out=y[:, 5:5 + N])
        s.synchronize()
        check(c, y[:, 5:5 + N], what="in place")
        assert bool((y[:, :5] == 2).all()) and bool((y[:, 5 + N:] == 2).all())


@pytest.mark.parametrize("T", [21, 400])
def test_rows_that_are_not_finite_stay_by_themselves(mq, T):
    """NaN in x of rows without an adapter is not read; infinities in x and NaN in base show in their own rows only."""
    rng = np.random.default_rng(T)
    c = make(rng, T, 264, 200, 24, 3, ids=rng.integers(-1, 4, T))
    want = call(mq, c)
    off = np.flatnonzero((c["ids"] < 0) | (c["ids"] >= 3))
    on = np.flatnonzero((c["ids"] >= 0) & (c["ids"] < 3))
    c["x"][off] = np.nan
    c["x"][on[2], 7], c["base"][on[4]] = np.inf, np.nan
    got = call(mq, c)
    odd = torch.tensor([int(on[2]), int(on[4])]).cuda()
    assert not torch.isfinite(got[odd]).any(dim=1).all() and torch.isnan(got[odd[1]]).all()
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[odd] = False
    assert torch.equal(got[rest], want[rest])


def test_nothing_to_do(mq):
    h = lambda *s: torch.zeros(s, dtype=torch.float16, device="cuda")
    ids, scale = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.ones(2, device="cuda")
    assert mq.lora_apply(h(0, 64), ids, h(2, 8, 64), h(2, 40, 8), scale, h(0, 40)).shape == (0, 40)
    ids = torch.zeros(3, dtype=torch.int32, device="cuda")
    assert mq.lora_apply(h(3, 64), ids, h(2, 8, 64), h(2, 0, 8), scale, h(3, 0)).shape == (3, 0)
    base = h(3, 40) + 2
    assert torch.equal(mq.lora_apply(h(3, 64) + 1, ids, h(0, 8, 64), h(0, 40, 8), scale[:0], base), base)
    pos = torch.zeros(0, dtype=torch.int32, device="cuda")
    assert [tuple(t.shape) for t in mq.qk_norm_rope(h(0, 512), h(0, 128), None, None, pos, 4, 1)] == [(0, 512), (0, 128)]


def test_wide_ranges(mq):
    """Visual activations with outlier channels, an intermediate beyond fp16's range, tiny ones, no adapters at all."""
    rng = np.random.default_rng(4)
    c = make(rng, 40, 1024, 144, 16, 2, gain=20.0)
    c["x"][:, [3, 97, 200]] *= np.float16(50)
    check(c, call(mq, c), what="outliers")
    c = make(rng, 20, 1024, 144, 16, 2)
    c["x"][:] = 60000.0
    c["a"][:] = np.abs(c["a"]) * np.float16(8)
    c["b"][:] = (c["b"].astype(np.float32) * 1e-6).astype(np.float16)
    check(c, call(mq, c), what="large intermediate")
    c = make(rng, 20, 1024, 144, 16, 2, gain=1e-6)
    check(c, call(mq, c), what="small")
    c = make(rng, 20, 1024, 144, 16, 0, ids=np.zeros(20))
    check(c, call(mq, c), what="no adapters")


@pytest.mark.parametrize("T,K,N,rank,n", [(1100, 1032, 130, 72, 2), (1025, 640, 96, 128, 1), (700, 2056, 200, 104, 3), (300, 256, 1160, 128, 2),
                                          (129, 3584, 512, 80, 1)])
def test_many_rows_of_two_parts_of_ranks(mq, T, K, N, rank, n):
    """Ranks beyond 64, which many rows take in two parts; the last part nearly empty or full."""
    c = make(np.random.default_rng(T + rank), T, K, N, rank, n)
    check(c, call(mq, c), what=f"{T} {K} {N} r{rank}")


def test_stale_workspace_and_replays(mq):
    """A captured call replayed with other ids and inputs, its workspace full of NaN patterns before each replay."""
    rng = np.random.default_rng(5)
    c = make(rng, 37, 2048, 264, 32, 5)
    x, ids, base = dev(c["x"]), dev(c["ids"]), dev(c["base"])
    rest = dev(c["a"]), dev(c["b"]), dev(c["scale"])
    ws = torch.empty(mq.lora_workspace_bytes(37, 2048, 32), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(base)
    run = lambda: mq.lora_apply(x, ids, *rest, base, out=out, workspace=ws)
    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for rep in range(4):
        c["ids"] = rng.integers(-1, 6, 37).astype(np.int32)
        c["x"] = rng.standard_normal((37, 2048)).astype(np.float16)
        ids.copy_(dev(c["ids"])), x.copy_(dev(c["x"]))
        ws.fill_(0xff)
        g.replay()
        torch.cuda.synchronize()
        check(c, out, what=f"replay {rep}")
        assert torch.equal(mq.lora_apply(x, ids, *rest, base), out)


@pytest.mark.parametrize("T,K,N,rank,n", [(200, 264, 257, 24, 3), (513, 520, 333, 40, 2), (1500, 136, 72, 8, 4), (140, 128, 128, 16, 1),
                                          (256, 1000, 640, 128, 3), (700, 3584, 136, 64, 5), (1100, 8, 1, 8, 2), (300, 392, 1288, 104, 2)])
def test_many_rows(mq, T, K, N, rank, n):
    """More rows of an adapter than a tile holds, odd sizes and ranks that are no power of two."""
    c = make(np.random.default_rng(T * 3 + rank), T, K, N, rank, n)
    check(c, call(mq, c), what=f"{T} {K} {N} r{rank}")


@pytest.mark.parametrize("ids", ["one", "none", "runs", "each its own", "alternating", "last row only"])
def test_who_has_which_adapter_among_many_rows(mq, ids):
    T, n = 700, 20
    rows = {"one": np.full(T, 3), "none": np.where(np.arange(T) % 2, -1, n), "runs": np.arange(T) // 90, "each its own": np.arange(T) % n,
            "alternating": np.where(np.arange(T) % 2, 0, 19), "last row only": np.where(np.arange(T) == T - 1, 5, -5)}[ids]
    c = make(np.random.default_rng(11), T, 256, 264, 16, n, ids=rows)
    check(c, call(mq, c), what=ids)


def test_many_rows_in_place_with_strides(mq):
    rng = np.random.default_rng(12)
    for N in (96, 91):
        c = make(rng, 300, 128, N, 32, 3)
        y = torch.full((300, N + 21), 2.0, dtype=torch.float16, device="cuda")
        y[:, 5:5 + N] = dev(c["base"])
        mq.lora_apply(dev(c["x"]), dev(c["ids"]), dev(c["a"]), dev(c["b"]), dev(c["scale"]), y[:, 5:5 + N], out=y[:, 5:5 + N])
        check(c, y[:, 5:5 + N], what="in place")
        assert bool((y[:, :5] == 2).all()) and bool((y[:, 5 + N:] == 2).all())


@pytest.mark.parametrize("T", [40, 300])
def test_results_repeat_and_two_streams_run_at_once(mq, T):
    """The same bits every time, also with another call on another stream beside it."""
    rng = np.random.default_rng(13)
    c = make(rng, T, 2048, 520, 32, 4)
    t = [dev(c[k]) for k in ("x", "ids", "a", "b", "scale", "base")]
    want = mq.lora_apply(*t)
    check(c, want, what="alone")
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for _ in range(10):
        for s in streams:
            with torch.cuda.stream(s):
                outs.append(mq.lora_apply(*t))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_many_rows_replayed(mq):
    rng = np.random.default_rng(14)
    c = make(rng, 260, 1024, 136, 64, 3)
    x, ids, base = dev(c["x"]), dev(c["ids"]), dev(c["base"])
    rest = dev(c["a"]), dev(c["b"]), dev(c["scale"])
    ws = torch.empty(mq.lora_workspace_bytes(260, 1024, 64), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(base)
    run = lambda: mq.lora_apply(x, ids, *rest, base, out=out, workspace=ws)
    run()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run()
    for rep in range(3):
        c["ids"] = rng.integers(-1, 4, 260).astype(np.int32)
        ids.copy_(dev(c["ids"]))
        ws.fill_(0xff)
        g.replay()
        torch.cuda.synchronize()
        check(c, out, what=f"replay {rep}")


@pytest.mark.parametrize("T,N", [(5, 264), (256, 130), (900, 264), (900, 16392), (1300, 264)])
def test_many_more_adapters_than_rows_use(mq, T, N):
    """Five of five hundred in use."""
    rng = np.random.default_rng(T + N)
    used = np.array([0, 17, 255, 256, 499])
    c = make(rng, T, 136, N, 16, 500, ids=np.where(np.arange(T) % 7 == 6, 500, used[np.arange(T) * 3 % 5]))
    got = call(mq, c)
    five = {**c, "a": c["a"][used], "b": c["b"][used], "scale": c["scale"][used]}
    five["ids"] = np.where(c["ids"] == 500, -1, np.searchsorted(used, c["ids"])).astype(np.int32)
    check(five, got, what=f"{T} {N}")
    check(five, call(mq, five), what=f"{T} {N}, five")


@pytest.mark.parametrize("T", [21, 400])
def test_adapters_that_are_not_finite_stay_by_themselves(mq, T):
    """An infinity in A shows in every column of the rows that use it, one in B in its own column of them, and nowhere else."""
    rng = np.random.default_rng(T + 1)
    c = make(rng, T, 264, 200, 24, 4, ids=np.arange(T) % 5 - 1)
    want = call(mq, c)
    c["a"][1, 5, 263], c["b"][2, 77, 3] = np.inf, -np.inf
    got = call(mq, c)
    ids = torch.from_numpy(c["ids"]).cuda()
    odd = torch.zeros((T, 200), dtype=torch.bool, device="cuda")
    odd[:, 77] = ids == 2
    odd[ids == 1] = True
    assert not torch.isfinite(got[odd]).any() and torch.equal(got[~odd], want[~odd])
