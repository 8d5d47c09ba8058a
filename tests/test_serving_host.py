"""Refusals of the serving-step entry points that need no GPU: a bad call is turned down on the host, nothing is
launched, and the binding turns down tensors that the kernels cannot address."""
import ctypes

import pytest

from paper_2502_00425_amd import binding as mq

torch = pytest.importorskip("torch")
P, Q = 0x10000, 0x20000
L = mq.lib


def cache(k=P, v=P, table=P, n_seq=2, n_pages=8, page=16, table_pages=4, hkv=4, D=128):
    c = mq.PagedCacheStruct(k, v, table, n_seq, n_pages, page, table_pages, hkv, D)
    return c, ctypes.addressof(c)


BAD_CACHES = [
    (dict(k=None), mq.ERR_NULL), (dict(v=None), mq.ERR_NULL), (dict(table=None), mq.ERR_NULL),
    (dict(k=P + 8), mq.ERR_ALIGNMENT), (dict(v=P + 2), mq.ERR_ALIGNMENT), (dict(table=P + 2), mq.ERR_ALIGNMENT),
    (dict(n_seq=-1), mq.ERR_BAD_SHAPE), (dict(n_pages=0), mq.ERR_BAD_SHAPE), (dict(table_pages=0), mq.ERR_BAD_SHAPE),
    (dict(hkv=0), mq.ERR_BAD_SHAPE), (dict(D=64), mq.ERR_UNSUPPORTED), (dict(page=8), mq.ERR_UNSUPPORTED),
    (dict(page=48), mq.ERR_UNSUPPORTED), (dict(page=8192), mq.ERR_UNSUPPORTED),
    (dict(page=4096, table_pages=1 << 20), mq.ERR_UNSUPPORTED),
]


def test_norm_refusals():
    f = L.mquant_qk_norm_rope

    def call(q=P, ldq=3584, qo=Q, ldqo=3584, k=P, ldk=512, ko=Q, ldko=512, qw=P, kw=P, eps=1e-6, pos=P, T=4, hq=28, hkv=4, D=128,
             base=10000.0):
        return f(q, ldq, qo, ldqo, k, ldk, ko, ldko, qw, kw, eps, pos, T, hq, hkv, D, base, None)

    for bad in (dict(T=-1), dict(hq=-1), dict(hkv=-1), dict(hq=0, hkv=0), dict(ldq=3576), dict(ldqo=3576), dict(ldk=504),
                dict(ldko=504), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(base=1.0),
                dict(base=float("nan")), dict(q=Q, ldq=3592)):
        assert call(**bad) == mq.ERR_BAD_SHAPE, bad
    for bad in (dict(q=None), dict(qo=None), dict(k=None), dict(ko=None), dict(pos=None)):
        assert call(**bad) == mq.ERR_NULL, bad
    for bad in (dict(q=P + 2), dict(qo=Q + 8), dict(k=P + 4), dict(ko=Q + 2), dict(qw=P + 8), dict(kw=P + 2), dict(pos=P + 2),
                dict(ldq=3588), dict(ldko=516)):
        assert call(**bad) == mq.ERR_ALIGNMENT, bad
    for bad in (dict(D=64), dict(D=256), dict(hq=1 << 23, ldq=1 << 30, ldqo=1 << 30)):
        assert call(**bad) == mq.ERR_UNSUPPORTED, bad
    assert call(T=0, q=None, k=None, qo=None, ko=None, pos=None) == mq.OK


def test_append_refusals():
    f = L.mquant_kv_append

    def call(q=P, ldq=3584, qo=Q, ldqo=3584, k=P, ldk=512, v=P, ldv=512, qw=None, kw=None, eps=1e-6, start=P, pos=P, rope=None, T=4,
             hq=28, base=10000.0, c=None):
        keep, address = c if c is not None else cache(k=Q + 65536, v=Q + 131072)
        return f(q, ldq, qo, ldqo, k, ldk, v, ldv, qw, kw, eps, start, pos, rope, T, hq, base, address, None)

    for bad in (dict(T=-1), dict(hq=-1), dict(ldq=3576), dict(ldk=504), dict(ldv=504), dict(eps=-1.0), dict(base=0.5)):
        assert call(**bad) == mq.ERR_BAD_SHAPE, bad
    for bad in (dict(q=None), dict(qo=None), dict(k=None), dict(v=None), dict(start=None), dict(pos=None), dict(c=(None, None))):
        assert call(**bad) == mq.ERR_NULL, bad
    for bad in (dict(q=P + 2), dict(k=P + 8), dict(v=P + 8), dict(ldv=516), dict(start=P + 2), dict(pos=P + 1), dict(rope=P + 2),
                dict(qw=P + 2), dict(kw=P + 8)):
        assert call(**bad) == mq.ERR_ALIGNMENT, bad
    for kw, want in BAD_CACHES:
        assert call(c=cache(**{**dict(k=Q + 65536, v=Q + 131072), **kw})) == want, kw
    assert call(T=0, q=None) == mq.OK and call(c=cache(k=None, v=None, table=None, n_seq=0), q=None) == mq.OK


def test_attention_refusals():
    f = L.mquant_paged_attention
    size = L.mquant_paged_attention_workspace_bytes

    def call(q=P, ldq=3584, start=P, pos=P, o=Q, ldo=3584, T=2, hq=28, max_rows=0, max_kv=0, ws=P, ws_bytes=1 << 40, c=None):
        keep, address = c if c is not None else cache()
        return f(q, ldq, address, start, pos, o, ldo, T, hq, max_rows, max_kv, ws, ws_bytes, None)

    for bad in (dict(T=-1), dict(hq=0), dict(hq=30), dict(ldq=3576), dict(ldo=3580), dict(max_rows=-1), dict(max_kv=-1)):
        assert call(**bad) == mq.ERR_BAD_SHAPE, bad
    for bad in (dict(q=None), dict(o=None), dict(start=None), dict(pos=None), dict(c=(None, None))):
        assert call(**bad) == mq.ERR_NULL, bad
    for bad in (dict(q=P + 8), dict(o=Q + 4), dict(ldq=3588), dict(ldo=3586), dict(start=P + 2), dict(pos=P + 2)):
        assert call(**bad) == mq.ERR_ALIGNMENT, bad
    for kw, want in BAD_CACHES:
        assert call(c=cache(**kw)) == want, kw
    assert call(T=0, q=None) == mq.OK and call(c=cache(k=None, v=None, table=None, n_seq=0), q=None) == mq.OK
    # keys split over work-groups: the workspace is asked for, and has to be there
    big = dict(T=2, max_rows=1, max_kv=100000, c=cache(page=64, table_pages=2000, n_pages=4000))
    need = size(2, 2, 28, 4, 128, 1, 100000)
    if need > 0:
        assert call(**big, ws=None) == mq.ERR_WORKSPACE
        assert call(**big, ws_bytes=need - 1) == mq.ERR_WORKSPACE
        assert call(**big, ws=P + 16) == mq.ERR_ALIGNMENT
    assert size(-1, 2, 28, 4, 128, 0, 100) == mq.ERR_BAD_SHAPE and size(2, 2, 28, 3, 128, 0, 100) == mq.ERR_BAD_SHAPE
    assert size(2, 2, 28, 4, 96, 0, 100) == mq.ERR_UNSUPPORTED
    assert size(1 << 24, 1, 64, 8, 128, 0, 100) >= 0 and size((1 << 24) + 1, 1, 64, 8, 128, 0, 100) == mq.ERR_UNSUPPORTED
    assert call(T=1 << 30, hq=4) == mq.ERR_UNSUPPORTED
    assert size(0, 0, 28, 4, 128, 0, 0) == 0


def test_adapter_refusals():
    f = L.mquant_lora_apply
    need = L.mquant_lora_workspace_bytes(4, 512, 16)
    assert need >= 4 * 16 * 4

    def call(x=P, ldx=512, perm=None, ids=P, a=P, b=P, scale=P, base=P, ldb=640, y=Q, ldy=640, T=4, N=640, K=512, rank=16, n=3, ws=P,
             ws_bytes=need):
        return f(x, ldx, perm, ids, a, b, scale, base, ldb, y, ldy, T, N, K, rank, n, ws, ws_bytes, None)

    for bad in (dict(T=-1), dict(N=-1), dict(K=-8), dict(n=-1), dict(rank=0), dict(ldx=504), dict(ldb=639), dict(ldy=632),
                dict(y=P, ldy=648)):
        assert call(**bad) == mq.ERR_BAD_SHAPE, bad
    for bad in (dict(x=None), dict(ids=None), dict(a=None), dict(b=None), dict(scale=None), dict(base=None), dict(y=None)):
        assert call(**bad) == mq.ERR_NULL, bad
    for bad in (dict(rank=12), dict(rank=136), dict(K=516, ldx=520), dict(K=0), dict(K=(1 << 30) + 8, ldx=1 << 31, ws_bytes=1 << 50),
                dict(N=(1 << 30) + 1, ldb=1 << 31, ldy=1 << 31), dict(T=65536 * 256, ws_bytes=1 << 50)):
        assert call(**bad) == mq.ERR_UNSUPPORTED, bad
    for bad in (dict(x=P + 8), dict(ldx=516), dict(a=P + 2), dict(b=P + 8), dict(base=P + 1), dict(y=Q + 1), dict(ids=P + 2),
                dict(perm=P + 2), dict(scale=P + 2), dict(ws=P + 16)):
        assert call(**bad) == mq.ERR_ALIGNMENT, bad
    for bad in (dict(ws=None), dict(ws_bytes=need - 1)):
        assert call(**bad) == mq.ERR_WORKSPACE, bad
    assert call(T=0, x=None) == mq.OK and call(N=0, base=None, y=None) == mq.OK
    assert L.mquant_lora_workspace_bytes(-1, 512, 16) == mq.ERR_BAD_SHAPE
    assert L.mquant_lora_workspace_bytes(4, 512, 20) == mq.ERR_UNSUPPORTED


def test_binding_refuses_host_tensors():
    """What is not on the current device would be an address the GPU cannot read."""
    h = torch.zeros((4, 512), dtype=torch.float16)
    i = torch.zeros(4, dtype=torch.int32)
    pages, table = torch.zeros((3, 4, 16, 128), dtype=torch.float16), torch.zeros((2, 2), dtype=torch.int32)
    for call in (lambda: mq.qk_norm_rope(h, h, None, None, i, 4, 4), lambda: mq.PagedCache(pages, pages, table),
                 lambda: mq.lora_apply(h, i, h.view(1, 4, 512), h.view(1, 512, 4), torch.ones(1), h)):
        with pytest.raises(mq.MQuantError) as e:
            call()
        assert e.value.status == mq.ERR_UNSUPPORTED
    with pytest.raises(mq.MQuantError) as e:
        mq.PagedCache(pages[0], pages[0], table)
    assert e.value.status == mq.ERR_BAD_SHAPE


@pytest.mark.parametrize("K", [8, 512, 3584, 18944, 29568, 1 << 20])
def test_scratch_of_the_adapters_grows_with_rows_channels_and_rank(K):
    """Scratch for the largest step does for every smaller one."""
    size = L.mquant_lora_workspace_bytes
    rows = sorted({*range(1, 300), *range(300, 5000, 61), *(64 * i + d for i in range(1, 80) for d in (0, 1)), 16384, 16385, 100000, 1 << 24})
    for rank in (8, 16, 64, 72, 128):
        sizes = [size(T, K, rank) for T in rows]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])), rank
        assert all(s >= T * rank * 4 for s, T in zip(sizes, rows))
    for T in rows[::7]:
        by_rank = [size(T, K, r) for r in range(8, 129, 8)]
        assert by_rank == sorted(by_rank) and size(T, K, 64) <= size(T, K + 8, 64) and size(T, K, 128) <= size(T, K + 512, 128)


def test_rows_beyond_a_grid_are_refused():
    """2^32 threads are more than a launch takes: a wave of 64 to a row of up to 16 heads."""
    keep, address = cache(k=Q + 65536, v=Q + 131072)
    for T, heads in ((1 << 26, 1), (1 << 26, 16), (1 << 25, 17), (2 ** 31 - 1, 1)):
        w = heads * 128
        assert L.mquant_qk_norm_rope(P, w, Q, w, None, 0, None, 0, None, None, 1e-6, P, T, heads, 0, 128, 1e4, None) == mq.ERR_UNSUPPORTED
        assert L.mquant_kv_append(P, w, Q, w, P, 512, P, 512, None, None, 1e-6, P, P, None, T, heads, 1e4, address, None) == mq.ERR_UNSUPPORTED
