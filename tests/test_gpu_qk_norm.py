"""Norm and rotation of queries and keys per head, and the same with the write to the cache's pages, against the
fp64 oracle.

Tolerance per element: the fp16 result is off by half a step, 2^-11 |y|, 2^-25 in the subnormal range.  Before it, all is
fp32: the sum of 128 squares (12 roundings on a path: 8 in a lane, 4 across), the mean, the reciprocal root (4), the weight and the
scaling (2), sine and cosine rounded to fp32 (1), two products and a sum (3): 24 roundings of 2^-24 of the
pair's magnitude |u_even| + |u_odd| at most, within 2^-19."""
import numpy as np
import pytest

from oracle import mquant_oracle as orc
from serving import D, make_step

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


def host(t):
    return t.cpu().numpy().astype(np.float64)


def bound(ref):
    pair = np.abs(ref).reshape(ref.shape[0], -1, 2).sum(axis=2)
    return 2.0 ** -11 * np.abs(ref) + 2.0 ** -25 + 2.0 ** -19 * np.repeat(pair, 2, axis=1) * np.sqrt(2)


def check(got, ref, what):
    assert np.isfinite(got).all(), what
    err, tol = np.abs(got - ref), bound(ref)
    worst = np.unravel_index((err - tol).argmax(), err.shape)
    assert (err <= tol).all(), f"{what}: {err[worst]:.3e} > {tol[worst]:.3e} at {worst}"


def weights(rng):
    return rng.uniform(0.3, 2.0, D).astype(np.float16), rng.uniform(-2.0, 2.0, D).astype(np.float16)


@pytest.mark.parametrize("T,hq,hkv,norm", [(1, 28, 4, True), (1, 1, 1, True), (3, 64, 8, False), (77, 28, 4, True), (130, 5, 1, True),
                                           (33, 3, 7, True), (64, 40, 40, True), (257, 12, 2, False), (5, 16, 0, True), (5, 0, 3, True)])
@pytest.mark.parametrize("in_place", [False, True])
def test_norm_rope(mq, T, hq, hkv, norm, in_place):
    rng = np.random.default_rng(T * 100 + hq)
    buf = (rng.standard_normal((T, (hq + 2 * hkv) * D + 24)) * rng.choice([0.01, 1.0, 300.0], (T, 1))).astype(np.float16)
    pos = rng.integers(0, 40000, T).astype(np.int32)
    wq, wk = weights(rng) if norm else (None, None)
    b = dev(buf)
    q, k = b[:, :hq * D], b[:, hq * D:(hq + hkv) * D]
    before = b.clone()
    qo, ko = mq.qk_norm_rope(q, k, None if wq is None else dev(wq), None if wk is None else dev(wk), dev(pos), hq, hkv,
                             q_out=q if in_place else None, k_out=k if in_place else None)
    for got, x, w, n in ((qo, buf[:, :hq * D], wq, hq), (ko, buf[:, hq * D:(hq + hkv) * D], wk, hkv)):
        if n:
            check(host(got), orc.qk_norm_rope_f64(x, w, pos, n), f"T={T} {hq}/{hkv}")
    if in_place:
        before[:, :(hq + hkv) * D] = b[:, :(hq + hkv) * D]
    assert torch.equal(b, before)                     # what is not written stays as it was


def test_rotation_alone_is_rope_apply(mq):
    rng = np.random.default_rng(5)
    x = dev(rng.standard_normal((90, 28 * D)).astype(np.float16))
    pos = dev(rng.integers(0, 16384, 90).astype(np.int32))
    y, _ = mq.qk_norm_rope(x, x[:, :0], None, None, pos, 28, 0, base=500000.0)
    ref = orc.rope_apply_f64(host(x), pos.cpu().numpy(), 28, base=500000.0)
    check(host(y), ref, "rope")
    assert (np.abs(host(mq.rope_apply(x.clone(), pos, 28, base=500000.0)) - host(y)) <= 2 * bound(ref)).all()


def test_extremes(mq):
    """Heads of zeros, of the largest and of the smallest values; negative and large positions; eps from 0 up."""
    x = np.zeros((6, 2 * D), dtype=np.float16)
    x[1], x[2] = 65504.0, 6e-8
    x[3, ::2], x[3, 1::2] = -65504.0, 65504.0
    x[4] = np.linspace(-3, 3, 2 * D)
    pos = np.array([0, 7, 2 ** 31 - 1, -5, 1 << 20, 123456789], dtype=np.int32)
    w = np.ones(D, dtype=np.float16)
    for eps in (1e-6, 1e-12, 1.0):
        y, _ = mq.qk_norm_rope(dev(x), dev(x)[:, :0], dev(w), None, dev(pos), 2, 0, eps=eps)
        check(host(y), orc.qk_norm_rope_f64(x, w, pos, 2, eps=eps), f"eps={eps}")
    y, _ = mq.qk_norm_rope(dev(x[1:5]), dev(x[1:5])[:, :0], dev(w), None, dev(pos[1:5]), 2, 0, eps=0.0)
    check(host(y), orc.qk_norm_rope_f64(x[1:5], w, pos[1:5], 2, eps=0.0), "eps=0")


@pytest.mark.parametrize("seqs,hq,hkv,page,norm,own_ids", [
    ([(1, 1)], 28, 4, 16, True, False), ([(1, 1281)], 28, 4, 16, False, False), ([(1, 16), (1, 17), (1, 300)], 64, 8, 16, True, True),
    ([(40, 40)], 5, 1, 32, True, False), ([(0, 0), (3, 3), (0, 9), (130, 200)], 12, 2, 64, True, True),
    ([(1, 5 + i) for i in range(150)], 4, 2, 16, True, False), ([(77, 77)], 0, 3, 128, True, False)])
def test_append(mq, seqs, hq, hkv, page, norm, own_ids):
    rng = np.random.default_rng(len(seqs) * 7 + hq)
    st = make_step(rng, seqs, hq, hkv, page, before=2, behind=3, spans=[(2, 5)], poison=False)
    T = st["T"]
    buf = rng.standard_normal((T, (hq + 2 * hkv) * D)).astype(np.float16)
    q, k, v = buf[:, :hq * D], buf[:, hq * D:(hq + hkv) * D], buf[:, (hq + hkv) * D:]
    wq, wk = weights(rng) if norm else (None, None)
    ids = rng.integers(0, 5000, T).astype(np.int32) if own_ids else None
    b = dev(buf)
    kp, vp = dev(st["kp"]), dev(st["vp"])
    cache = mq.PagedCache(kp, vp, dev(st["table"]))
    qo = torch.full((T, hq * D), 9.0, dtype=torch.float16, device="cuda")
    mq.kv_append(b[:, :hq * D], b[:, hq * D:(hq + hkv) * D], b[:, (hq + hkv) * D:], cache, dev(st["start"]), dev(st["pos"]), hq,
                 None if wq is None else dev(wq), None if wk is None else dev(wk),
                 rope_pos_dev=None if ids is None else dev(ids), q_out=qo)
    turn = st["pos"] if ids is None else ids
    inside = slice(2, T - 3)
    if hq:
        check(host(qo)[inside], orc.qk_norm_rope_f64(q, wq, turn, hq)[inside], "q")
        assert (host(qo)[:2] == 9).all() and (host(qo)[T - 3:] == 9).all()
    want_k, want_v = st["kp"].astype(np.float64), st["vp"].astype(np.float64)
    orc.kv_append(want_k, want_v, st["table"], st["start"], st["pos"], orc.qk_norm_rope_f64(k, wk, turn, hkv), v.astype(np.float64))
    assert np.array_equal(host(vp), want_v)
    shape = lambda a: a.reshape(-1, D)
    check(shape(host(kp)), shape(want_k), "k pages")
    untouched = (want_k == st["kp"]).reshape(-1, D).all(axis=1)
    assert np.array_equal(shape(host(kp))[untouched], shape(st["kp"].astype(np.float64))[untouched])
    assert torch.equal(b, dev(buf))


def test_append_rows_without_a_slot(mq):
    """Positions below zero and beyond the table, pages out of range: q is written, the cache is left alone."""
    rng = np.random.default_rng(3)
    hq, hkv, page, T = 4, 2, 16, 5
    table = np.array([[1, 4, -1]], dtype=np.int32)                       # 4 pages: the second and third are no pages
    kp = dev(rng.standard_normal((4, hkv, page, D)).astype(np.float16))
    vp = kp.clone() + 1
    pos = np.array([-1, 16, 32, 48, 2 ** 31 - 1], dtype=np.int32)
    x = dev(rng.standard_normal((T, (hq + 2 * hkv) * D)).astype(np.float16))
    k0, v0 = kp.clone(), vp.clone()
    qo = mq.kv_append(x[:, :hq * D], x[:, hq * D:(hq + hkv) * D], x[:, (hq + hkv) * D:], mq.PagedCache(kp, vp, dev(table)),
                      dev(np.array([0, T], dtype=np.int32)), dev(pos), hq)
    assert torch.equal(kp, k0) and torch.equal(vp, v0)
    check(host(qo), orc.qk_norm_rope_f64(host(x)[:, :hq * D], None, pos, hq), "q")


def test_append_beyond_32_bits(mq):
    """A page whose offset passes 2^31 halves (the pages take 4.3 GB each): the write lands in it."""
    hkv, page, n_pages = 8, 128, (1 << 31) // (8 * 128 * D) + 3
    kp = torch.zeros((n_pages, hkv, page, D), dtype=torch.float16, device="cuda")
    vp = torch.zeros_like(kp)
    rng = np.random.default_rng(8)
    x = dev(rng.standard_normal((1, (8 + 2 * hkv) * D)).astype(np.float16))
    cache = mq.PagedCache(kp, vp, dev(np.array([[n_pages - 1]], dtype=np.int32)))
    q = mq.kv_append(x[:, :8 * D], x[:, 8 * D:16 * D], x[:, 16 * D:], cache, dev(np.array([0, 1], dtype=np.int32)),
                     dev(np.array([77], dtype=np.int32)), 8)
    ref = orc.qk_norm_rope_f64(host(x)[:, 8 * D:16 * D], None, [77], hkv)
    check(host(kp[n_pages - 1, :, 77]).reshape(1, -1), ref, "k")
    assert torch.equal(vp[n_pages - 1, :, 77].reshape(1, -1), x[:, 16 * D:])
    assert int(torch.count_nonzero(vp[n_pages - 1])) <= hkv * D and not bool(vp[:4].any())
    o = mq.paged_attention(q, cache, dev(np.array([0, 1], dtype=np.int32)), dev(np.array([77], dtype=np.int32)), 8, max_kv=78)
    assert np.isfinite(host(o)).all()


@pytest.mark.parametrize("T", [7, 900])
def test_append_captured(mq, T):
    """A captured append replayed while rows, positions and pages change under it, eager work between."""
    rng = np.random.default_rng(T)
    hq, hkv, page, n_pages = 28, 4, 16, 140
    x = dev(rng.standard_normal((T, (hq + 2 * hkv) * D)).astype(np.float16))
    q, k, v = x[:, :hq * D], x[:, hq * D:(hq + hkv) * D], x[:, (hq + hkv) * D:]
    table = dev(rng.permutation(n_pages)[:130].reshape(2, 65).astype(np.int32))
    start, pos = dev(np.array([0, 2, T], dtype=np.int32)), dev(np.arange(T, dtype=np.int32))
    w = dev(rng.uniform(0.5, 1.5, D).astype(np.float16))
    cache = mq.PagedCache(*(torch.zeros((n_pages, hkv, page, D), dtype=torch.float16, device="cuda") for _ in range(2)), table)
    qo = torch.zeros((T, hq * D), dtype=torch.float16, device="cuda")
    run = lambda c, o: mq.kv_append(q, k, v, c, start, pos, hq, w, w, q_out=o)
    run(cache, qo)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        run(cache, qo)
    for rep in range(3):
        x.copy_(dev(rng.standard_normal(x.shape).astype(np.float16)))
        pos.copy_(dev(rng.permutation(1040)[:T].astype(np.int32)))
        start.copy_(dev(np.array([0, rep, T - rep], dtype=np.int32)))
        table.copy_(dev(rng.permutation(n_pages)[:130].reshape(2, 65).astype(np.int32)))
        cache.k_pages.zero_(), cache.v_pages.zero_(), qo.zero_()
        g.replay()
        torch.cuda.synchronize()
        kp, vp, o = cache.k_pages.clone(), cache.v_pages.clone(), qo.clone()
        cache.k_pages.zero_(), cache.v_pages.zero_()
        o2 = torch.zeros_like(o)
        run(cache, o2)
        assert torch.equal(cache.k_pages, kp) and torch.equal(cache.v_pages, vp) and torch.equal(o, o2)
        ref = orc.qk_norm_rope_f64(host(q), w.cpu().numpy(), pos.cpu().numpy(), hq)
        check(host(o)[:T - rep], ref[:T - rep], f"replay {rep}")
        assert bool(vp.any()) and not bool(o[T - rep:].any())


def test_a_single_row_in_place_whatever_its_width(mq):
    """A row alone is written where it was read from, also where the two views of it end elsewhere."""
    rng = np.random.default_rng(21)
    hq, hkv = 6, 2
    x = rng.standard_normal((1, (hq + 2 * hkv) * D)).astype(np.float16)
    pos = np.array([9], dtype=np.int32)
    want_q, want_k = orc.qk_norm_rope_f64(x[:, :hq * D], None, pos, hq), orc.qk_norm_rope_f64(x[:, hq * D:(hq + hkv) * D], None, pos, hkv)
    b = dev(x)
    mq.qk_norm_rope(b, b[:, hq * D:], None, None, dev(pos), hq, hkv, q_out=b[:, :hq * D], k_out=b[:, hq * D:(hq + hkv) * D])
    check(host(b)[:, :hq * D], want_q, "q")
    check(host(b)[:, hq * D:(hq + hkv) * D], want_k, "k")
    assert torch.equal(b[:, (hq + hkv) * D:], dev(x)[:, (hq + hkv) * D:])
    b = dev(x)
    cache = mq.PagedCache(*(torch.zeros((2, hkv, 16, D), dtype=torch.float16, device="cuda") for _ in range(2)),
                          dev(np.array([[1]], dtype=np.int32)))
    mq.kv_append(b, b[:, hq * D:], b[:, (hq + hkv) * D:], cache, dev(np.array([0, 1], dtype=np.int32)), dev(pos), hq, q_out=b[:, :hq * D])
    check(host(b)[:, :hq * D], want_q, "q")
    assert torch.equal(b[:, hq * D:], dev(x)[:, hq * D:])
    check(host(cache.k_pages[1, :, 9]).reshape(1, -1), want_k, "k page")
