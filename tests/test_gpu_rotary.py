"""Rotations of a descriptor, by themselves and with the write to the cache's pages, against the fp64 oracle.

Tolerance per element as for the norm and rotation of whole heads (24 roundings of 2^-24 of the pair's magnitude, within 2^-19, then half a
step of fp16: 2^-11 relative, 2^-25 in the subnormal range), with two roundings more for the factor of sine and cosine: the pair's
magnitude is that of the result.  Frequencies are rounded to double (2^-53) and positions reach 2^31: 2^31 * 2^-53 radians are within
2^-22 of an angle."""
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


def pairs(ref, rot, halves):
    """Magnitude of the pair that an element belongs to, of itself behind the rotated channels."""
    h = np.abs(ref).reshape(ref.shape[0], -1, D)
    m = h.copy()
    first = np.arange(rot // 2) if halves else np.arange(0, rot, 2)
    second = first + (rot // 2 if halves else 1)
    m[:, :, first] = m[:, :, second] = h[:, :, first] + h[:, :, second]
    return m.reshape(ref.shape)


def check(got, ref, rot, halves, what=""):
    assert np.isfinite(got).all(), what
    err, tol = np.abs(got - ref), 2.0 ** -11 * np.abs(ref) + 2.0 ** -25 + 2.0 ** -19 * np.sqrt(2) * pairs(ref, rot, halves)
    worst = np.unravel_index((err - tol).argmax(), err.shape)
    assert (err <= tol).all(), f"{what}: {err[worst]:.3e} > {tol[worst]:.3e} at {worst}"


def sections_of(rng, half, axes):
    cut = np.sort(rng.integers(0, half + 1, axes - 1))
    return tuple(int(n) for n in np.diff(np.concatenate([[0], cut, [half]])))


@pytest.mark.parametrize("rot", [16, 32, 48, 64, 96, 112, 128])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("axes", [1, 2, 3])
def test_layouts(mq, rot, halves, axes):
    rng = np.random.default_rng(rot * 10 + axes + halves)
    for T, hq, hkv, norm, in_place in ((1, 28, 4, True, False), (70, 5, 3, False, True), (400, 28, 4, True, True), (1100, 22, 2, False, False)):
        buf = (rng.standard_normal((T, (hq + hkv) * D + 24)) * rng.choice([0.01, 1.0, 300.0], (T, 1))).astype(np.float16)
        pos = rng.integers(0, 40000, (axes, T)).astype(np.int32)
        sec, scale = sections_of(rng, rot // 2, axes), float(np.float32(rng.choice([1.0, 1.375, 0.3])))
        wq, wk = (rng.uniform(-2.0, 2.0, D).astype(np.float16) if norm else None for _ in range(2))
        turn = mq.Rotary(rot, base=1e6, halves=halves, sections=sec, scale=scale)
        b = dev(buf)
        q, k, before = b[:, :hq * D], b[:, hq * D:(hq + hkv) * D], b.clone()
        qo, ko = mq.rotary_apply(q, k, dev(pos), turn, hq, hkv, None if wq is None else dev(wq), None if wk is None else dev(wk),
                                 q_out=q if in_place else None, k_out=k if in_place else None)
        f = orc.rotary_frequencies(rot, 1e6)
        for got, x, w, n in ((qo, buf[:, :hq * D], wq, hq), (ko, buf[:, hq * D:(hq + hkv) * D], wk, hkv)):
            check(host(got), orc.rotary_f64(x, w, pos, n, f, halves, sec, scale), rot, halves, f"T={T} {sec}")
        if in_place:
            before[:, :(hq + hkv) * D] = b[:, :(hq + hkv) * D]
        assert torch.equal(b, before)                     # what is not written stays as it was


@pytest.mark.parametrize("scaling,args", [("linear", dict(factor=8.0)), ("base", dict(factor=4.0)), ("turns", dict(factor=16.0, trained=4096.0)),
                                          ("turns", dict(factor=8.0, trained=8192.0, low=1.0, high=4.0)), ("none", {})])
def test_stretched(mq, scaling, args):
    rng = np.random.default_rng(len(scaling))
    x = rng.standard_normal((200, 4 * D)).astype(np.float16)
    pos = rng.integers(0, 1 << 20, 200).astype(np.int32)
    for rot, halves in ((128, True), (64, False)):
        turn = mq.Rotary(rot, base=5e5, halves=halves, scaling=scaling, **args)
        f = orc.rotary_frequencies(rot, 5e5, scaling, **args)
        assert np.allclose(list(turn.struct.freq)[:rot // 2], f, rtol=1e-14, atol=0)
        y, _ = mq.rotary_apply(dev(x), dev(x)[:, :0], dev(pos), turn, 4, 0)
        check(host(y), orc.rotary_f64(x, None, pos, 4, f, halves), rot, halves, scaling)


def test_whole_interleaved_heads_are_the_plain_rotation(mq):
    rng = np.random.default_rng(2)
    x, pos = dev(rng.standard_normal((300, 8 * D)).astype(np.float16)), dev(rng.integers(0, 30000, 300).astype(np.int32))
    w = dev(rng.uniform(0.5, 2, D).astype(np.float16))
    a, _ = mq.rotary_apply(x, x[:, :0], pos, mq.Rotary(), 8, 0, w)
    b, _ = mq.qk_norm_rope(x, x[:, :0], w, None, pos, 8, 0)
    ref = orc.qk_norm_rope_f64(host(x), host(w), pos.cpu().numpy(), 8)
    check(host(a), ref, 128, False)
    assert (np.abs(host(a) - host(b)) <= 2 * (2.0 ** -11 * np.abs(ref) + 2.0 ** -25 + 2.0 ** -18 * pairs(ref, 128, False))).all()


def test_extremes(mq):
    x = np.zeros((6, 2 * D), dtype=np.float16)
    x[1], x[2] = 40000.0, 6e-8
    x[3, ::2], x[3, 1::2] = -40000.0, 40000.0
    x[4] = np.linspace(-3, 3, 2 * D)
    pos = np.array([0, 7, 2 ** 31 - 1, -5, 1 << 20, -2 ** 31], dtype=np.int32)
    w = np.ones(D, dtype=np.float16)
    for halves in (False, True):
        for rot in (48, 128):
            y, _ = mq.rotary_apply(dev(x), dev(x)[:, :0], dev(pos), mq.Rotary(rot, halves=halves), 2, 0, dev(w))
            check(host(y), orc.rotary_f64(x, w, pos, 2, orc.rotary_frequencies(rot, 1e4), halves), rot, halves)
    free = np.linspace(-0.9, 0.9, 24)                     # given frequencies, in both directions and 0
    y, _ = mq.rotary_apply(dev(x), dev(x)[:, :0], dev(pos), mq.Rotary(48, freq=free, halves=True, scale=0.0), 2, 0, dev(w))
    check(host(y), orc.rotary_f64(x, w, pos, 2, free, True, scale=0.0), 48, True)


@pytest.mark.parametrize("seqs,hq,hkv,page,norm,axes", [
    ([(1, 1)], 28, 4, 16, True, 0), ([(1, 1281)], 28, 4, 16, False, 3), ([(1, 16), (1, 17), (1, 300)], 64, 8, 16, True, 3),
    ([(40, 40)], 5, 1, 32, True, 2), ([(0, 0), (3, 3), (0, 9), (130, 200)], 12, 2, 64, True, 1),
    ([(1, 5 + i) for i in range(150)], 4, 2, 16, True, 3), ([(77, 77)], 0, 3, 128, True, 0), ([(900, 900), (300, 700)], 28, 4, 16, True, 3)])
@pytest.mark.parametrize("rot,halves", [(128, True), (64, True), (96, False), (128, False)])
def test_append(mq, seqs, hq, hkv, page, norm, axes, rot, halves):
    rng = np.random.default_rng(len(seqs) * 7 + hq + rot)
    st = make_step(rng, seqs, hq, hkv, page, before=2, behind=3, spans=[(2, 5)], poison=False)
    T = st["T"]
    buf = rng.standard_normal((T, (hq + 2 * hkv) * D)).astype(np.float16)
    x = [buf[:, :hq * D], buf[:, hq * D:(hq + hkv) * D], buf[:, (hq + hkv) * D:]]
    wq, wk = (rng.uniform(0.3, 2.0, D).astype(np.float16) if norm else None for _ in range(2))
    ids = rng.integers(0, 5000, (axes, T)).astype(np.int32) if axes else None
    sec = sections_of(rng, rot // 2, axes or 2)
    b, kp, vp = dev(buf), dev(st["kp"]), dev(st["vp"])
    q, k, v = b[:, :hq * D], b[:, hq * D:(hq + hkv) * D], b[:, (hq + hkv) * D:]
    q_out = torch.full((T, hq * D + 8), 7.0, dtype=torch.float16, device="cuda")
    mq.rotary_append(q, k, v, mq.PagedCache(kp, vp, dev(st["table"])), dev(st["start"]), dev(st["pos"]), mq.Rotary(rot, halves=halves, sections=sec),
                     hq, None if wq is None else dev(wq), None if wk is None else dev(wk), rope_pos_dev=None if ids is None else dev(ids), q_out=q_out)
    f = orc.rotary_frequencies(rot, 1e4)
    at = ids if axes else np.tile(st["pos"], (2, 1))
    mine = np.concatenate([r for _, r in orc.sequence_rows(st["start"], T)])
    if hq:
        got = host(q_out)
        check(got[mine, :hq * D], orc.rotary_f64(x[0], wq, at, hq, f, halves, sec)[mine], rot, halves, "q")
        others = np.setdiff1d(np.arange(T), mine)
        assert (got[others] == 7.0).all() and (got[:, hq * D:] == 7.0).all()
    k64 = orc.rotary_f64(x[1], wk, at, hkv, f, halves, sec)
    want_k, want_v = st["kp"].astype(np.float64), st["vp"].copy()
    orc.kv_append(want_k, want_v, st["table"], st["start"], st["pos"], k64, x[2])
    assert np.array_equal(vp.cpu().numpy(), want_v)
    got_k, written = host(kp), np.zeros(want_k.shape[:3:2], dtype=bool)
    for s, rows in orc.sequence_rows(st["start"], T):
        for i in rows:
            slot = orc.cache_slot(st["table"], page, s, int(st["pos"][i]), len(st["kp"]))
            written[slot] = True
            check(got_k[slot[0], :, slot[1]].reshape(1, -1), k64[i:i + 1], rot, halves, "k")
    assert np.array_equal(got_k.transpose(0, 2, 1, 3)[~written], want_k.transpose(0, 2, 1, 3)[~written])


def test_rows_without_a_slot(mq):
    """Negative positions, positions behind the table, pages out of range: the query is written, nothing is cached."""
    rng = np.random.default_rng(8)
    T, hq, hkv = 4, 4, 2
    buf = rng.standard_normal((T, (hq + 2 * hkv) * D)).astype(np.float16)
    b = dev(buf)
    kp = torch.full((3, hkv, 16, D), 5.0, dtype=torch.float16, device="cuda")
    vp = torch.full_like(kp, 6.0)
    pos = np.array([-1, 32, 3, 16], dtype=np.int32)
    q = mq.rotary_append(b[:, :hq * D], b[:, hq * D:(hq + hkv) * D], b[:, (hq + hkv) * D:], mq.PagedCache(kp, vp, dev(np.array([[3, -1]], dtype=np.int32))),
                         dev(np.array([0, 4], dtype=np.int32)), dev(pos), mq.Rotary(halves=True), hq)
    check(host(q), orc.rotary_f64(buf[:, :hq * D], None, pos, hq, orc.rotary_frequencies(128, 1e4), True), 128, True)
    assert (kp == 5).all() and (vp == 6).all()


def test_replays_and_streams(mq):
    rng = np.random.default_rng(9)
    x = dev(rng.standard_normal((64, 32 * D)).astype(np.float16))
    pos, turn = dev(rng.integers(0, 900, (3, 64)).astype(np.int32)), mq.Rotary(halves=True, sections=(16, 24, 24))
    q, k = x[:, :28 * D], x[:, 28 * D:]
    qo, ko = torch.empty((64, 28 * D), dtype=torch.float16, device="cuda"), torch.empty((64, 4 * D), dtype=torch.float16, device="cuda")
    mq.rotary_apply(q, k, pos, turn, 28, 4, q_out=qo, k_out=ko)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mq.rotary_apply(q, k, pos, turn, 28, 4, q_out=qo, k_out=ko)
    for step in range(3):
        pos.copy_(dev(rng.integers(0, 90000, (3, 64)).astype(np.int32)))
        graph.replay()
        got = qo.clone(), ko.clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            want = mq.rotary_apply(q, k, pos, turn, 28, 4)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
