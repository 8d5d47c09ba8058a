"""Refusals of the serving loop's entry points that need no GPU: a bad call is turned down on the host, nothing is launched, and the
binding turns down tensors that the kernels cannot address."""
import ctypes

import numpy as np
import pytest

from oracle import mquant_oracle as orc
from paper_2502_00425_amd import binding as mq
from test_serving_host import BAD_CACHES, L, P, Q, cache

torch = pytest.importorskip("torch")


def test_plan_refusals():
    def call(length=P, rows=P, shared=None, order=None, n_seq=3, table=P, table_pages=4, page=16, ring=P, n_pages=9, state=P, state_out=P,
             length_out=P, start=P, pos=P, slot=P, T=5):
        return L.mquant_step_plan(length, rows, shared, order, n_seq, table, table_pages, page, ring, n_pages, state, state_out, length_out,
                                  start, pos, slot, T, None)

    for bad in (dict(n_seq=-1), dict(T=-1), dict(n_pages=0), dict(n_pages=-4), dict(table_pages=0)):
        assert call(**bad) == mq.ERR_BAD_SHAPE, bad
    for bad in (dict(page=8), dict(page=0), dict(page=24), dict(page=8192), dict(page=-16), dict(n_seq=(1 << 20) + 1), dict(table_pages=1 << 27),
                dict(page=4096, table_pages=1 << 19)):
        assert call(**bad) == mq.ERR_UNSUPPORTED, bad
    for name in ("length", "rows", "table", "ring", "state", "state_out", "length_out", "start", "pos"):
        assert call(**{name: None}) == mq.ERR_NULL, name
    for name in ("length", "rows", "shared", "order", "table", "ring", "state", "state_out", "length_out", "start", "pos"):
        assert call(**{name: P + 2}) == mq.ERR_ALIGNMENT, name
    assert call(slot=P + 4) == mq.ERR_ALIGNMENT


def rotation(**changes):
    r = mq.RotaryStruct()
    assert L.mquant_rotary_init(ctypes.addressof(r), 0, 128, 1e4, 0, 1.0, 0.0, 1.0, 32.0) == mq.OK
    for name, v in changes.items():
        if isinstance(v, dict):
            for i, x in v.items():
                getattr(r, name)[i] = x
        else:
            setattr(r, name, v)
    return r


BAD_ROTATIONS = [
    (dict(rot_dim=8), mq.ERR_UNSUPPORTED), (dict(rot_dim=0), mq.ERR_UNSUPPORTED), (dict(rot_dim=144), mq.ERR_UNSUPPORTED),
    (dict(rot_dim=40), mq.ERR_UNSUPPORTED), (dict(rot_dim=-16), mq.ERR_UNSUPPORTED), (dict(rot_dim=64), mq.ERR_BAD_SHAPE),
    (dict(layout=2), mq.ERR_BAD_SHAPE), (dict(layout=-1), mq.ERR_BAD_SHAPE), (dict(n_axes=0), mq.ERR_BAD_SHAPE), (dict(n_axes=4), mq.ERR_BAD_SHAPE),
    (dict(n_axes=2, section={0: 64, 1: 1}), mq.ERR_BAD_SHAPE), (dict(n_axes=2, section={0: 65, 1: -1}), mq.ERR_BAD_SHAPE),
    (dict(n_axes=3, section={0: 2 ** 31 - 1, 1: 2 ** 31 - 1, 2: 66}), mq.ERR_BAD_SHAPE), (dict(scale=float("nan")), mq.ERR_BAD_SHAPE),
    (dict(scale=float("inf")), mq.ERR_BAD_SHAPE), (dict(freq={63: float("inf")}), mq.ERR_BAD_SHAPE), (dict(freq={0: float("nan")}), mq.ERR_BAD_SHAPE)]


def test_rotary_refusals():
    good = rotation()

    def apply(q=P, ldq=3584, qo=Q, ldqo=3584, k=P, ldk=512, ko=Q, ldko=512, qw=P, kw=P, eps=1e-6, pos=P, T=4, hq=28, hkv=4, D=128, r=good):
        return L.mquant_rotary_apply(q, ldq, qo, ldqo, k, ldk, ko, ldko, qw, kw, eps, pos, T, hq, hkv, D, r and ctypes.addressof(r), None)

    def append(q=P, ldq=3584, qo=Q, ldqo=3584, k=P, ldk=512, v=P, ldv=512, qw=None, kw=None, eps=1e-6, start=P, pos=P, rope=None, T=4, hq=28,
               r=good, c=None):
        keep, address = c if c is not None else cache(k=Q + 65536, v=Q + 131072)
        return L.mquant_rotary_append(q, ldq, qo, ldqo, k, ldk, v, ldv, qw, kw, eps, start, pos, rope, T, hq, r and ctypes.addressof(r), address, None)

    for changes, want in BAD_ROTATIONS:
        assert apply(r=rotation(**changes)) == want and append(r=rotation(**changes)) == want, changes
    for bad in (dict(T=-1), dict(hq=-1), dict(hkv=-1), dict(hq=0, hkv=0), dict(ldq=3576), dict(ldqo=3576), dict(ldk=504), dict(ldko=504),
                dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(q=Q, ldq=3592)):
        assert apply(**bad) == mq.ERR_BAD_SHAPE, bad
    for bad in (dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(pos=None), dict(r=None)):
        assert apply(**bad) == mq.ERR_NULL, bad
    for bad in (dict(q=P + 2), dict(qo=Q + 8), dict(k=P + 4), dict(ko=Q + 2), dict(qw=P + 8), dict(kw=P + 2), dict(pos=P + 2), dict(ldq=3588),
                dict(ldko=516)):
        assert apply(**bad) == mq.ERR_ALIGNMENT, bad
    for bad in (dict(D=64), dict(D=256), dict(hq=1 << 23, ldq=1 << 30, ldqo=1 << 30), dict(T=1 << 26, hq=1, ldq=128, ldqo=128, hkv=0)):
        assert apply(**bad) == mq.ERR_UNSUPPORTED, bad
    for bad in (dict(T=-1), dict(hq=-1), dict(ldq=3576), dict(ldk=504), dict(ldv=504), dict(eps=-1.0)):
        assert append(**bad) == mq.ERR_BAD_SHAPE, bad
    for bad in (dict(q=None), dict(qo=None), dict(k=None), dict(v=None), dict(start=None), dict(pos=None), dict(r=None), dict(c=(None, None))):
        assert append(**bad) == mq.ERR_NULL, bad
    for bad in (dict(q=P + 2), dict(k=P + 8), dict(v=P + 8), dict(ldv=516), dict(start=P + 2), dict(pos=P + 1), dict(rope=P + 2), dict(qw=P + 2)):
        assert append(**bad) == mq.ERR_ALIGNMENT, bad
    for kw, want in BAD_CACHES:
        assert append(c=cache(**{**dict(k=Q + 65536, v=Q + 131072), **kw})) == want, kw
    assert append(T=1 << 26, hq=1, ldq=128, ldqo=128) == mq.ERR_UNSUPPORTED
    assert apply(T=0, q=None, k=None, qo=None, ko=None, pos=None) == mq.OK and append(T=0, q=None) == mq.OK
    assert append(c=cache(k=None, v=None, table=None, n_seq=0), q=None) == mq.OK


def test_descriptor_refusals_and_contents():
    r = mq.RotaryStruct()

    def init(layout=0, rot=128, base=1e4, scaling=0, factor=1.0, trained=4096.0, low=1.0, high=32.0, to=ctypes.addressof(r)):
        return L.mquant_rotary_init(to, layout, rot, base, scaling, factor, trained, low, high)

    assert init(to=None) == mq.ERR_NULL
    for bad in (dict(rot=0), dict(rot=8), dict(rot=24), dict(rot=144), dict(rot=-16)):
        assert init(**bad) == mq.ERR_UNSUPPORTED, bad
    for bad in (dict(layout=2), dict(layout=-1), dict(scaling=4), dict(scaling=-1), dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")),
                dict(factor=0.5), dict(factor=float("nan")), dict(factor=float("inf")), dict(scaling=2, base=1e300, factor=1e300),
                *(dict(scaling=3, **x) for x in (dict(trained=0.0), dict(trained=float("nan")), dict(trained=float("inf")), dict(low=32.0),
                                                 dict(high=float("nan")), dict(high=float("inf")), dict(low=-float("inf"))))):
        assert init(**bad) == mq.ERR_BAD_SHAPE, bad
    for scaling, number in mq.Rotary.SCALINGS.items():
        for rot in (16, 48, 128):
            assert init(rot=rot, scaling=number, factor=8.0, base=5e5) == mq.OK
            want = orc.rotary_frequencies(rot, 5e5, scaling, 8.0, 4096.0, 1.0, 32.0)
            assert np.allclose(r.freq[:rot // 2], want, rtol=1e-14, atol=0) and list(r.freq[rot // 2:]) == [0.0] * (64 - rot // 2)
            assert (r.layout, r.rot_dim, r.n_axes, list(r.section), r.scale) == (0, rot, 1, [rot // 2, 0, 0], 1.0)
    for bad in (dict(scaling="stretch"), dict(sections=[]), dict(sections=[16, 16, 16, 16]), dict(freq=[1.0] * 63), dict(base=0.5)):
        with pytest.raises(mq.MQuantError) as e:
            mq.Rotary(128, **bad)
        assert e.value.status == mq.ERR_BAD_SHAPE
    a = mq.Rotary(32, sections=[4, 6, 6], scale=0.5, freq=range(16), halves=True)
    assert (a.n_axes, list(a.struct.section), list(a.struct.freq[:16]), a.struct.layout) == (3, [4, 6, 6], list(range(16)), 1)
    a.struct.n_axes = 2
    assert a.n_axes == 2 and a.fast == (a.address, 2)


def test_shared_attention_refusals():
    size = L.mquant_paged_attention_shared_workspace_bytes

    def call(q=P, ldq=3584, start=P, pos=P, groups=P, prefix=P, n_groups=1, o=Q, ldo=3584, T=2, hq=28, rows=0, longest=0, behind=0, ws=P,
             ws_bytes=1 << 40, c=None):
        keep, address = c if c is not None else cache()
        return L.mquant_paged_attention_shared(q, ldq, address, start, pos, groups, prefix, n_groups, o, ldo, T, hq, rows, longest, behind, ws,
                                               ws_bytes, None)

    for n_groups in (0, 1):
        for bad in (dict(T=-1), dict(hq=0), dict(hq=30), dict(ldq=3576), dict(ldo=3580), dict(rows=-1), dict(longest=-1), dict(behind=-1),
                    dict(n_groups=-1)):
            assert call(**{"n_groups": n_groups, **bad}) == mq.ERR_BAD_SHAPE, bad
        for bad in (dict(q=None), dict(o=None), dict(start=None), dict(pos=None), dict(c=(None, None))):
            assert call(n_groups=n_groups, **bad) == mq.ERR_NULL, bad
        for bad in (dict(q=P + 8), dict(o=Q + 4), dict(ldq=3588), dict(ldo=3586), dict(start=P + 2), dict(pos=P + 2)):
            assert call(n_groups=n_groups, **bad) == mq.ERR_ALIGNMENT, bad
        for kw, want in BAD_CACHES:
            assert call(n_groups=n_groups, c=cache(**kw)) == want, kw
        assert call(n_groups=n_groups, T=0, q=None) == mq.OK
        assert call(n_groups=n_groups, c=cache(k=None, v=None, table=None, n_seq=0), q=None) == mq.OK
        assert call(n_groups=n_groups, T=1 << 30, hq=4) == mq.ERR_UNSUPPORTED
    assert call(groups=None) == call(prefix=None) == mq.ERR_NULL
    for page, table_pages in ((16, (1 << 26) + 1), (64, 33554431), (4096, (1 << 18) + 1)):
        assert call(c=cache(page=page, table_pages=table_pages), ws=None) == mq.ERR_UNSUPPORTED
        assert call(c=cache(page=page, table_pages=table_pages - 1), ws=None) == (mq.ERR_UNSUPPORTED if page == 64 else mq.ERR_WORKSPACE)
    assert call(groups=P + 2) == call(prefix=P + 1) == mq.ERR_ALIGNMENT
    big = dict(T=2, rows=1, longest=100000, behind=100, c=cache(page=64, table_pages=2000, n_pages=4000))
    need = size(2, 2, 1, 28, 4, 128, 1, 100000, 100)
    assert need > 0
    assert call(**big, ws=None) == call(**big, ws_bytes=need - 1) == mq.ERR_WORKSPACE and call(**big, ws=P + 16) == mq.ERR_ALIGNMENT
    assert size(-1, 2, 1, 28, 4, 128, 0, 9, 9) == size(2, 2, -1, 28, 4, 128, 0, 9, 9) == size(2, 2, 1, 28, 3, 128, 0, 9, 9) == mq.ERR_BAD_SHAPE
    assert size(2, 2, 1, 28, 4, 128, 0, -9, 9) == size(2, 2, 1, 28, 4, 128, 0, 9, -9) == mq.ERR_BAD_SHAPE
    assert size(2, 2, 1, 28, 4, 96, 0, 9, 9) == size((1 << 24) + 1, 1, 1, 64, 8, 128, 0, 9, 9) == mq.ERR_UNSUPPORTED
    assert size(0, 0, 0, 28, 4, 128, 0, 0, 0) == 0


def test_sample_refusals():
    size = L.mquant_sample_workspace_bytes
    need = size(3, 1000)
    assert need > 0

    def call(x=P, kind=mq.F16, ld=1000, t=P, k=P, p=P, m=P, u=P, token=P, logprob=P, rows=3, V=1000, ws=P, ws_bytes=need):
        return L.mquant_sample(x, kind, ld, t, k, p, m, u, token, logprob, rows, V, ws, ws_bytes, None)

    for bad in (dict(rows=-1), dict(V=0), dict(V=-5), dict(ld=999), dict(ld=-1000), dict(kind=2), dict(kind=-1)):
        assert call(**bad) == mq.ERR_BAD_SHAPE, bad
    for bad in (dict(V=(1 << 20) + 1, ld=1 << 21), dict(rows=1 << 22, ws_bytes=1 << 50), dict(rows=1 << 17, V=1 << 20, ld=1 << 20, ws_bytes=1 << 50)):
        assert call(**bad) == mq.ERR_UNSUPPORTED, bad
    for bad in (dict(x=None), dict(u=None), dict(token=None)):
        assert call(**bad) == mq.ERR_NULL, bad
    for bad in (dict(x=P + 1), dict(x=P + 2, kind=mq.F32), dict(t=P + 2), dict(k=P + 2), dict(p=P + 2), dict(m=P + 2), dict(u=P + 2),
                dict(token=P + 2), dict(logprob=P + 2), dict(ws=P + 16)):
        assert call(**bad) == mq.ERR_ALIGNMENT, bad
    for bad in (dict(ws=None), dict(ws_bytes=need - 1)):
        assert call(**bad) == mq.ERR_WORKSPACE, bad
    assert call(rows=0, x=None, u=None, token=None, ws=None, ws_bytes=0) == mq.OK
    assert size(-1, 10) == size(1, 0) == size(1, -1) == mq.ERR_BAD_SHAPE and size(1, (1 << 20) + 1) == mq.ERR_UNSUPPORTED


def test_scratch_of_sampling_grows_with_rows_and_vocabulary():
    size = L.mquant_sample_workspace_bytes
    lengths = sorted({*range(1, 70), *(n + d for n in (1024, 2048, 4096, 8192, 16384, 32768, 150000) for d in range(-8, 9)), (1 << 20) - 1, 1 << 20})
    for rows in (0, 1, 2, 7, 64, 1000):
        by_length = [size(rows, V) for V in lengths]
        assert by_length == sorted(by_length)
        assert all(size(rows, V) <= size(rows + 1, V) for V in lengths)


def test_binding_refuses_tensors_it_cannot_hand_on():
    h, i, f = torch.zeros((4, 512), dtype=torch.float16), torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    table, two = torch.zeros((4, 2), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: mq.rotary_apply(h, h, i, mq.Rotary(), 4, 4), lambda: mq.step_plan(i, i, table, 16, i, two, 4),
                 lambda: mq.sample(h, f, i, f, f, f), lambda: mq.sample(h.double(), f, i, f, f, f)):
        with pytest.raises(mq.MQuantError) as e:
            call()
        assert e.value.status == mq.ERR_UNSUPPORTED
    with pytest.raises(mq.MQuantError) as e:
        mq.sample(h.view(-1), f, i, f, f, f)
    assert e.value.status == mq.ERR_BAD_SHAPE
