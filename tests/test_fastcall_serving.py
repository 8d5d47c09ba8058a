"""The call module's way of the serving entries: it hands the library the same arguments as the way through ctypes, and what
it does not take (types, devices, layouts, sizes that do not fit together) calls nothing on either way.  Recording C functions stand in
for the library's entries, and objects with a tensor's methods for device tensors."""
import ctypes

import pytest
import torch

from paper_2502_00425_amd import binding as mq

P, I32, I64, F32, F64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_double
TYPES = {
    "qk_norm_rope": [P, I64, P, I64, P, I64, P, I64, P, P, F32, P, I32, I32, I32, I32, F64, P],
    "kv_append": [P, I64, P, I64, P, I64, P, I64, P, P, F32, P, P, P, I32, I32, F64, P, P],
    "paged_attention": [P, I64, P, P, P, P, I64, I32, I32, I32, I32, P, I64, P],
    "lora_apply": [P, I64, P, P, P, P, P, P, I64, P, I64, I32, I32, I32, I32, I32, P, I64, P],
}
STREAM, DEVICE = 0x1230, 1


class Tensor:
    """A device tensor as far as the binding asks."""
    is_cuda, count = True, 0

    def __init__(self, *shape, dtype=torch.float16, ld=None, device=DEVICE):
        Tensor.count += 1
        self.shape, self.dtype, self._ld, self._device, self._at = shape, dtype, ld, device, 0x10000 * Tensor.count
        self.device = torch.device("cuda", device)

    def stride(self, i=None):
        st, n = [], 1
        for s in reversed(self.shape):
            st.insert(0, n)
            n *= s
        if self._ld:
            st[0] = self._ld
        return tuple(st) if i is None else st[i]

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return self._ld is None

    def data_ptr(self):
        return self._at

    def get_device(self):
        return self._device

    def numel(self):
        return int(torch.Size(self.shape).numel())

    def element_size(self):
        return torch.tensor([], dtype=self.dtype).element_size()


@pytest.fixture
def both(monkeypatch):
    seen, keep = [], []

    def recorder(name):
        f = ctypes.CFUNCTYPE(ctypes.c_int, *TYPES[name])(lambda *a: seen.append((name, a)) or 0)
        keep.append(f)
        return f

    entries = {n: recorder(n) for n in TYPES}
    loader = mq.importlib.machinery.ExtensionFileLoader("mquant_fastcall", mq.FAST_PATH)
    mod = mq.importlib.util.module_from_spec(mq.importlib.util.spec_from_file_location("mquant_fastcall", mq.FAST_PATH, loader=loader))
    loader.exec_module(mod)
    mod.setup(lambda: True, lambda: DEVICE, lambda d: STREAM, *[1] * 7)
    assert mod.attention(*[None] * 10) is NotImplemented                                # before setup_serving
    mod.setup_serving(torch.float16, torch.float32, torch.int32, *(ctypes.cast(entries[n], P).value for n in TYPES))

    class Lib:
        mquant_status_string = staticmethod(lambda st: b"")
    for n in TYPES:
        setattr(Lib, "mquant_" + n, staticmethod(entries[n]))
    monkeypatch.setattr(mq, "lib", Lib)
    monkeypatch.setattr(mq, "_stream", lambda: STREAM)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: DEVICE)
    slow = type("Slow", (), {"__getattr__": lambda s, _: lambda *a: NotImplemented})()
    yield mod, slow, seen, monkeypatch, keep


def i32(*shape, **k):
    return Tensor(*shape, dtype=torch.int32, **k)


def calls(rows=3):
    """name -> (operands by name, the call on them)"""
    D = 128
    cache = mq.PagedCache(Tensor(9, 2, 16, D), Tensor(9, 2, 16, D), i32(4, 5))
    w = dict(q=Tensor(rows, 6 * D, ld=1600), k=Tensor(rows, 2 * D, ld=1600), v=Tensor(rows, 2 * D), wq=Tensor(D), wk=None, pos=i32(rows),
             qo=Tensor(rows, 6 * D), ko=Tensor(rows, 2 * D), start=i32(5), rope=i32(rows), ws=Tensor(4096, dtype=torch.uint8))
    lo = dict(x=Tensor(rows, 64, ld=80), ids=i32(rows), a=Tensor(3, 16, 64), b=Tensor(3, 40, 16), scale=Tensor(3, dtype=torch.float32),
              base=Tensor(rows, 40), perm=None, out=Tensor(rows, 40, ld=48), ws=Tensor(4096, dtype=torch.uint8))
    pick = lambda *names: {n: w[n] for n in names}
    return {
        "qk_norm_rope": (pick("q", "k", "wq", "wk", "pos", "qo", "ko"), lambda q, k, wq, wk, pos, qo, ko:
                         mq.qk_norm_rope(q, k, wq, wk, pos, 6, 2, eps=1e-5, base=5e5, q_out=qo, k_out=ko)),
        "kv_append": (pick("q", "k", "v", "start", "pos", "wq", "wk", "rope", "qo"), lambda q, k, v, start, pos, wq, wk, rope, qo:
                      mq.kv_append(q, k, v, cache, start, pos, 6, wq, wk, rope_pos_dev=rope, q_out=qo)),
        "paged_attention": (pick("q", "start", "pos", "qo", "ws"), lambda q, start, pos, qo, ws:
                            mq.paged_attention(q, cache, start, pos, 6, 2, 70, out=qo, workspace=ws)),
        "lora_apply": (lo, lambda x, ids, a, b, scale, base, perm, out, ws:
                       mq.lora_apply(x, ids, a, b, scale, base, perm_dev=perm, out=out, workspace=ws)),
    }


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("rows", [1, 3])
def test_the_same_arguments_either_way(both, name, rows):
    mod, slow, seen, mp, _ = both
    operands, call = calls(rows)[name]
    for way in (mod, slow):
        mp.setattr(mq, "_fast", way)
        call(**operands)
    assert len(seen) == 2 and seen[0] == seen[1] and seen[0][0] == name and seen[0][1][-1] == STREAM
    fast = {"qk_norm_rope": "norm", "kv_append": "append", "paged_attention": "attention", "lora_apply": "lora"}[name]
    mp.setattr(mq, "_fast", type("Counting", (), {"__getattr__": lambda s, n: lambda *a: calls_made.append(n) or getattr(mod, n)(*a)})())
    calls_made = []
    call(**operands)
    assert calls_made == [fast] and len(seen) == 3                     # the module took the call


@pytest.mark.parametrize("name", list(TYPES))
def test_operands_that_do_not_fit_call_nothing(both, name):
    """Each operand in turn of another type, on another device, of a row more, of columns that are not next to each other."""
    mod, slow, seen, mp, _ = both
    operands, call = calls()[name]
    for what, t in operands.items():
        if t is None:
            continue
        wrong = [Tensor(*t.shape, dtype=torch.bfloat16, ld=t._ld), Tensor(*t.shape, dtype=t.dtype, ld=t._ld, device=DEVICE + 1)]
        if what == "ws":
            wrong = wrong[1:]
        else:
            wrong.append(Tensor(t.shape[0] + 1, *t.shape[1:], dtype=t.dtype, ld=t._ld))
        if len(t.shape) != 2:
            wrong.append(Tensor(*t.shape, dtype=t.dtype, ld=77))
        for bad in wrong:
            for way in (mod, slow):
                mp.setattr(mq, "_fast", way)
                with pytest.raises(mq.MQuantError):
                    call(**{**operands, what: bad})
    assert not seen


def test_errors_and_interrupts(both):
    mod, slow, seen, mp, keep = both
    mp.setattr(mq, "_fast", mod)
    bad = ctypes.CFUNCTYPE(ctypes.c_int, *TYPES["lora_apply"])(lambda *a: mq.ERR_WORKSPACE)
    keep.append(bad)
    mod.setup_serving(torch.float16, torch.float32, torch.int32, 1, 1, 1, ctypes.cast(bad, P).value)
    operands, call = calls()["lora_apply"]
    with pytest.raises(mq.MQuantError) as e:
        call(**operands)
    assert e.value.status == mq.ERR_WORKSPACE
    for where in ("get_device", "data_ptr", "is_contiguous"):
        for error in (KeyboardInterrupt, MemoryError, SystemExit):
            def fail(*a):
                raise error
            t = i32(3)
            setattr(t, where, fail)
            with pytest.raises(error):
                call(**{**operands, "ids": t})
    assert not seen


@pytest.mark.parametrize("bound", [70, 80, 81, 2 ** 31 - 1, 2 ** 32 + 3, 2 ** 40])
def test_a_bound_beyond_the_table_is_the_tables(both, bound):
    """5 pages of 16 slots: the scratch that is asked for and the call go by 80 slots at most."""
    mod, slow, seen, mp, _ = both
    asked = []
    mq.lib.mquant_paged_attention_workspace_bytes = staticmethod(lambda *a: asked.append(a) or 0)
    operands, _ = calls()["paged_attention"]
    cache = mq.PagedCache(Tensor(9, 2, 16, 128), Tensor(9, 2, 16, 128), i32(4, 5))
    for way in (mod, slow):
        mp.setattr(mq, "_fast", way)
        mq.paged_attention(operands["q"], cache, operands["start"], operands["pos"], 6, 2, bound, out=operands["qo"])
    assert [a[-1] for a in asked] == [min(bound, 80)] * 2 and [s[1][10] for s in seen] == [min(bound, 80)] * 2


def test_sizes_beyond_32_bits_call_nothing(both):
    """Rows, channels, columns, sequences and pages whose lowest 32 bits would make sense."""
    mod, slow, seen, mp, _ = both
    far = 1 << 32
    mq.lib.mquant_lora_workspace_bytes = mq.lib.mquant_paged_attention_workspace_bytes = staticmethod(lambda *a: 256)
    for way in (mod, slow):
        mp.setattr(mq, "_fast", way)
        for name in TYPES:                                                    # rows
            operands, call = calls(rows=far + 3)[name]
            with pytest.raises(mq.MQuantError) as e:
                call(**operands)
            assert e.value.status == mq.ERR_UNSUPPORTED
        operands, call = calls()["lora_apply"]
        for other in (dict(x=Tensor(3, far + 64), a=Tensor(3, 16, far + 64)),
                      dict(base=Tensor(3, far + 40), b=Tensor(3, far + 40, 16), out=Tensor(3, far + 40)),
                      dict(a=Tensor(far + 3, 16, 64), b=Tensor(far + 3, 40, 16), scale=Tensor(far + 3, dtype=torch.float32))):
            with pytest.raises(mq.MQuantError) as e:
                call(**{**operands, **other})
            assert e.value.status == mq.ERR_UNSUPPORTED
        for pages, table in (((far + 9, 2, 16, 128), (4, 5)), ((9, 2, 16, 128), (far + 4, 5)), ((9, 2, 16, 128), (4, far + 5))):
            with pytest.raises(mq.MQuantError) as e:
                mq.PagedCache(Tensor(*pages), Tensor(*pages), i32(*table))
            assert e.value.status == mq.ERR_UNSUPPORTED
    assert not seen
    operands, call = calls()["lora_apply"]                                    # scratch may be as large as it likes
    for way in (mod, slow):
        mp.setattr(mq, "_fast", way)
        call(**{**operands, "ws": Tensor(far + 4096, dtype=torch.uint8)})
    assert [s[1][-2] for s in seen] == [far + 4096] * 2
