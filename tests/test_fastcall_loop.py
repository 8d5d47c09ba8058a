"""The call module's way of the serving loop's entries: it hands the library the same arguments as the way through ctypes, and what it does
not take calls nothing on either way.  Recording C functions stand in for the library's entries."""
import ctypes

import pytest
import torch

from paper_2502_00425_amd import binding as mq
from test_fastcall_serving import DEVICE, F32, I32, I64, P, STREAM, Tensor, i32

TYPES = {
    "step_plan": [P, P, P, P, I32, P, I32, I32, P, I32, P, P, P, P, P, P, I32, P],
    "rotary_apply": [P, I64, P, I64, P, I64, P, I64, P, P, F32, P, I32, I32, I32, I32, P, P],
    "rotary_append": [P, I64, P, I64, P, I64, P, I64, P, P, F32, P, P, P, I32, I32, P, P, P],
    "paged_attention_shared": [P, I64, P, P, P, P, P, I32, P, I64, I32, I32, I32, I32, I32, P, I64, P],
    "sample": [P, I32, I64, P, P, P, P, P, P, P, I32, I32, P, I64, P],
}
FAST = {"step_plan": "plan", "rotary_apply": "rotary", "rotary_append": "rotary_append", "paged_attention_shared": "shared", "sample": "sample"}


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
    mod.setup_serving(torch.float16, torch.float32, torch.int32, *[1] * 4)
    for n, count in (("plan", 14), ("rotary", 12), ("rotary_append", 13), ("shared", 13), ("sample", 11)):
        assert getattr(mod, n)(*[None] * count) is NotImplemented                       # before setup_loop
    mod.setup_loop(torch.int64, *(ctypes.cast(entries[n], P).value for n in TYPES))
    rotary_init = mq.lib.mquant_rotary_init

    class Lib:
        mquant_status_string = staticmethod(lambda st: b"")
        mquant_rotary_init = staticmethod(rotary_init)
        mquant_sample_workspace_bytes = staticmethod(lambda rows, V: 512)
    for n in TYPES:
        setattr(Lib, "mquant_" + n, staticmethod(entries[n]))
    monkeypatch.setattr(mq, "lib", Lib)
    monkeypatch.setattr(mq, "_stream", lambda: STREAM)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: DEVICE)
    slow = type("Slow", (), {"__getattr__": lambda s, _: lambda *a: NotImplemented})()
    yield mod, slow, seen, monkeypatch, keep


def calls(rows=3, V=500):
    """name -> (operands by name, the call on them)"""
    D = 128
    f32 = lambda *s: Tensor(*s, dtype=torch.float32)
    cache = mq.PagedCache(Tensor(9, 2, 16, D), Tensor(9, 2, 16, D), i32(4, 5))
    three, one = mq.Rotary(sections=[16, 24, 24]), mq.Rotary(64, halves=True)
    ws = Tensor(4096, dtype=torch.uint8)
    plan = dict(length=i32(4), rows=i32(4), table=i32(4, 5), ring=i32(9), state=i32(2), shared=i32(4), order=i32(rows), length_out=i32(4),
                state_out=i32(2), start=i32(5), pos=i32(rows), slots=Tensor(rows, dtype=torch.int64))
    norm = dict(q=Tensor(rows, 6 * D, ld=1600), k=Tensor(rows, 2 * D, ld=1600), pos=i32(3, rows), wq=Tensor(D), wk=None, qo=Tensor(rows, 6 * D),
                ko=Tensor(rows, 2 * D))
    append = dict(q=norm["q"], k=norm["k"], v=Tensor(rows, 2 * D), start=i32(5), pos=i32(rows), wq=None, wk=Tensor(D), rope=i32(rows), qo=norm["qo"])
    att = dict(q=norm["q"], start=i32(5), pos=i32(rows), groups=i32(3), prefix=i32(2), out=norm["qo"], ws=ws)
    smp = dict(logits=Tensor(rows, V, ld=V + 12), t=f32(rows), k=i32(rows), p=None, m=f32(rows), u=f32(rows), out=i32(rows), lp=f32(rows), ws=ws)
    return {
        "step_plan": (plan, lambda length, rows_, table, ring, state, shared, order, length_out, state_out, start, pos, slots:
                      mq.step_plan(length, rows_, table, 16, ring, state, rows, shared, order, length_out, state_out, start, pos, slots)),
        "rotary_apply": (norm, lambda q, k, pos, wq, wk, qo, ko: mq.rotary_apply(q, k, pos, three, 6, 2, wq, wk, eps=1e-5, q_out=qo, k_out=ko)),
        "rotary_append": (append, lambda q, k, v, start, pos, wq, wk, rope, qo:
                          mq.rotary_append(q, k, v, cache, start, pos, one, 6, wq, wk, rope_pos_dev=rope, q_out=qo)),
        "paged_attention_shared": (att, lambda q, start, pos, groups, prefix, out, ws:
                                   mq.paged_attention_shared(q, cache, start, pos, groups, prefix, 6, 2, 70, 33, out=out, workspace=ws)),
        "sample": (smp, lambda logits, t, k, p, m, u, out, lp, ws: mq.sample(logits, t, k, p, m, u, out, lp, ws)),
    }


def run(call, operands):
    call(*operands.values())


@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("rows", [1, 3])
def test_the_same_arguments_either_way(both, name, rows):
    mod, slow, seen, mp, _ = both
    operands, call = calls(rows)[name]
    for way in (mod, slow):
        mp.setattr(mq, "_fast", way)
        run(call, operands)
    assert len(seen) == 2 and seen[0][0] == name and seen[0][1][-1] == STREAM
    a, b = (list(s[1]) for s in seen)
    if name == "sample" and rows == 1:                                 # the stride of a single row says nothing
        a[2] = b[2] = None
    assert a == b
    mp.setattr(mq, "_fast", type("Counting", (), {"__getattr__": lambda s, n: lambda *a: calls_made.append(n) or getattr(mod, n)(*a)})())
    calls_made = []
    run(call, operands)
    assert calls_made == [FAST[name]] and len(seen) == 3               # the module took the call


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
        elif what != "ring":                                           # as many pages as there are
            wrong.append(Tensor(t.shape[0] + 1, *t.shape[1:], dtype=t.dtype, ld=t._ld))
        if len(t.shape) != 2:
            wrong.append(Tensor(*t.shape, dtype=t.dtype, ld=77))
        for bad in wrong:
            for way in (mod, slow):
                mp.setattr(mq, "_fast", way)
                with pytest.raises(mq.MQuantError):
                    run(call, {**operands, what: bad})
    assert not seen


def test_positions_go_by_the_axes(both):
    mod, slow, seen, mp, _ = both
    norm, apply = calls()["rotary_apply"]
    step, append = calls()["rotary_append"]
    for way in (mod, slow):
        mp.setattr(mq, "_fast", way)
        for bad in (i32(3), i32(1, 3), i32(2, 3), i32(9), i32(3, 3, ld=8)):
            with pytest.raises(mq.MQuantError):
                run(apply, {**norm, "pos": bad})
        for bad in (i32(2, 3), i32(3, 1), i32(4)):
            with pytest.raises(mq.MQuantError):
                run(append, {**step, "rope": bad})
        assert not seen
    for way in (mod, slow):
        mp.setattr(mq, "_fast", way)
        run(append, {**step, "rope": i32(1, 3)}), run(append, {**step, "rope": None})
    assert [s[1][13] is None for s in seen] == [False, True] * 2


def test_logits_whose_rows_overlap_call_nothing(both):
    mod, slow, seen, mp, _ = both
    operands, call = calls()["sample"]
    for ld in (0, 1, 499):
        logits = Tensor(3, 500, ld=500)
        logits.stride = lambda i=None, ld=ld: (ld, 1) if i is None else (ld, 1)[i]
        logits.is_contiguous = lambda: False
        for way in (mod, slow):
            mp.setattr(mq, "_fast", way)
            with pytest.raises(mq.MQuantError):
                run(call, {**operands, "logits": logits})
    assert not seen


def test_errors_and_interrupts(both):
    mod, slow, seen, mp, keep = both
    mp.setattr(mq, "_fast", mod)
    bad = ctypes.CFUNCTYPE(ctypes.c_int, *TYPES["sample"])(lambda *a: mq.ERR_WORKSPACE)
    keep.append(bad)
    mod.setup_loop(torch.int64, 1, 1, 1, 1, ctypes.cast(bad, P).value)
    operands, call = calls()["sample"]
    with pytest.raises(mq.MQuantError) as e:
        run(call, operands)
    assert e.value.status == mq.ERR_WORKSPACE
    for where in ("get_device", "data_ptr", "is_contiguous"):
        for error in (KeyboardInterrupt, MemoryError, SystemExit):
            def fail(*a):
                raise error
            t = i32(3)
            setattr(t, where, fail)
            with pytest.raises(error):
                run(call, {**operands, "k": t})
    assert not seen


@pytest.mark.parametrize("bound", [70, 80, 81, 2 ** 31 - 1, 2 ** 32 + 3, 2 ** 40])
def test_bounds_beyond_the_table_are_the_tables(both, bound):
    """5 pages of 16 slots: the scratch that is asked for and the call go by 80 slots at most."""
    mod, slow, seen, mp, _ = both
    asked = []
    mq.lib.mquant_paged_attention_shared_workspace_bytes = staticmethod(lambda *a: asked.append(a) or 0)
    o, _ = calls()["paged_attention_shared"]
    cache = mq.PagedCache(Tensor(9, 2, 16, 128), Tensor(9, 2, 16, 128), i32(4, 5))
    mp.setattr(torch, "empty", lambda *a, **k: Tensor(256, dtype=torch.uint8))
    for way in (mod, slow):
        mp.setattr(mq, "_fast", way)
        mq.paged_attention_shared(o["q"], cache, o["start"], o["pos"], o["groups"], o["prefix"], 6, 2, bound, bound, out=o["out"])
    assert [a[-2:] for a in asked] == [(min(bound, 80),) * 2] * 2 and [s[1][13:15] for s in seen] == [(min(bound, 80),) * 2] * 2


def test_sizes_beyond_32_bits_call_nothing(both):
    """Rows, tokens, pages and sequences whose lowest 32 bits would make sense."""
    mod, slow, seen, mp, _ = both
    far = 1 << 32
    mq.lib.mquant_paged_attention_shared_workspace_bytes = staticmethod(lambda *a: 256)
    for way in (mod, slow):
        mp.setattr(mq, "_fast", way)
        for name in ("rotary_apply", "rotary_append", "paged_attention_shared", "sample"):
            operands, call = calls(rows=far + 3)[name]
            with pytest.raises(mq.MQuantError) as e:
                run(call, operands)
            assert e.value.status == mq.ERR_UNSUPPORTED
        operands, call = calls(V=far + 500)["sample"]
        with pytest.raises(mq.MQuantError) as e:
            run(call, operands)
        assert e.value.status == mq.ERR_UNSUPPORTED
        operands, call = calls()["step_plan"]
        for other in (dict(ring=i32(far + 9)), dict(table=i32(4, far + 5))):
            with pytest.raises(mq.MQuantError) as e:
                run(call, {**operands, **other})
            assert e.value.status == mq.ERR_UNSUPPORTED
    assert not seen
