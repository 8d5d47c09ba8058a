"""Thin ctypes binding of libmquant.so: argument marshalling only.

Every function has the name of the C entry point it calls (without the
``mquant_`` prefix) and does no arithmetic of the method: tensors are handed
over as device pointers, the stream is torch's current HIP stream.  PyTorch is
used for device memory and streams only.  There is no CPU fallback: if the HIP
library is missing or cannot be loaded the import of this module raises.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import operator
import os
import struct
import sysconfig
from typing import Optional, Sequence, Tuple

import numpy as np
# torch before libmquant.so: the ROCm wheel of torch carries its own HIP runtime under the
# same soname.  Loaded second, libmquant binds to that copy and shares torch's streams and
# memory; loaded first, it would pull in the system runtime as a second one in the process,
# and a second runtime may find no device to open.
import torch  # noqa: F401

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "lib", "libmquant.so")
FAST_PATH = os.path.join(_HERE, "lib", "mquant_fastcall" + sysconfig.get_config_var("EXT_SUFFIX"))

EXPORTS = (
    "mquant_version", "mquant_status_string", "mquant_aifs_build_perm", "mquant_aifs_permute",
    "mquant_aifs_remap_mask", "mquant_hadamard_quant_act", "mquant_hadamard_absmax",
    "mquant_w4_prepacked_bytes", "mquant_w4_prepack", "mquant_w4a8_workspace_bytes",
    "mquant_w4a8_gemm", "mquant_w4a8_linear_prefill_workspace_bytes", "mquant_w4a8_linear_prefill",
    "mquant_hadamard_dynquant_act", "mquant_w4a8_gemm_rowscale", "mquant_w4a8_gemm_rms",
    "mquant_rope_apply", "mquant_aifs_attention_workspace_bytes", "mquant_aifs_attention",
    "mquant_hadamard_quant_act_bits", "mquant_static_scale_from_absmax", "mquant_tune_set",
    "mquant_build_id",
    "mquant_w4a8_linear_decode", "mquant_w4a8_linear_prefill_static", "mquant_w4a8_gemv_grouped",
    "mquant_w4a8_linear_decode_grouped",
    "mquant_w4g128_prepacked_bytes", "mquant_w4g128_prepack", "mquant_w4g128_gemm",
    "mquant_qk_norm_rope", "mquant_kv_append", "mquant_paged_attention_workspace_bytes", "mquant_paged_attention",
    "mquant_lora_workspace_bytes", "mquant_lora_apply",
)

OK, ERR_NULL, ERR_BAD_SHAPE, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_HIP, ERR_ALIGNMENT = 0, -1, -2, -3, -4, -5, -6


class MQuantError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


class Span(ctypes.Structure):
    _fields_ = [("start", ctypes.c_int32), ("len", ctypes.c_int32)]


class PagedCacheStruct(ctypes.Structure):
    _fields_ = [("k_pages_dev", ctypes.c_void_p), ("v_pages_dev", ctypes.c_void_p), ("page_table_dev", ctypes.c_void_p),
                ("n_seq", ctypes.c_int32), ("n_pages", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("table_pages", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32)]


class Linear(ctypes.Structure):
    _fields_ = [("w_prepacked_dev", ctypes.c_void_p), ("w_scale_dev", ctypes.c_void_p),
                ("y_dev", ctypes.c_void_p), ("ldy", ctypes.c_int64), ("N", ctypes.c_int32)]


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2502_00425_amd.build` "
            "(there is no CPU fallback)")
    lib = ctypes.CDLL(LIB_PATH)
    i32, i64, f32, p = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p
    lib.mquant_version.restype = ctypes.c_int
    lib.mquant_status_string.restype = ctypes.c_char_p
    lib.mquant_status_string.argtypes = [ctypes.c_int]
    lib.mquant_build_id.restype = ctypes.c_char_p
    lib.mquant_build_id.argtypes = []
    lib.mquant_static_scale_from_absmax.argtypes = [f32, i32, i32, p]
    lib.mquant_tune_set.argtypes = [i32, i32]
    lib.mquant_aifs_build_perm.argtypes = [i32, p, i32, p, p, p]
    lib.mquant_aifs_permute.argtypes = [p, i64, p, i64, p, i32, i32, p]
    lib.mquant_aifs_remap_mask.argtypes = [p, p, p, i32, p]
    lib.mquant_hadamard_quant_act.argtypes = [p, i64, p, p, i32, i32, i32, f32, f32, i32, p]
    lib.mquant_hadamard_absmax.argtypes = [p, i64, i32, i32, i32, p, p]
    lib.mquant_hadamard_quant_act_bits.argtypes = [p, i64, p, p, i32, i32, i32, f32, f32, i32, i32, p]
    lib.mquant_hadamard_dynquant_act.argtypes = [p, i64, p, p, p, i32, i32, i32, p]
    lib.mquant_w4a8_gemm_rowscale.argtypes = [p, p, p, p, p, i64, p, i32, i32, i32, p, i64, p]
    lib.mquant_w4a8_gemm_rms.argtypes = [p, p, p, p, i64, p, i32, i32, i32, i32, f32, f32, p, p, p, i32,
                                         p, i64, p]
    lib.mquant_w4_prepacked_bytes.restype = i64
    lib.mquant_w4_prepacked_bytes.argtypes = [i32, i32]
    lib.mquant_w4_prepack.argtypes = [p, p, i32, i32, p]
    lib.mquant_w4a8_workspace_bytes.restype = i64
    lib.mquant_w4a8_workspace_bytes.argtypes = [i32, i32, i32]
    lib.mquant_w4a8_gemm.argtypes = [p, p, p, p, i64, p, i32, i32, i32, i32, f32, f32, p, i64, p]
    lib.mquant_w4a8_linear_prefill_workspace_bytes.restype = i64
    lib.mquant_w4a8_linear_prefill_workspace_bytes.argtypes = [i32, i32, i32]
    lib.mquant_w4a8_linear_prefill.argtypes = [p, i64, p, p, p, p, i64, i32, i32, i32, i32, f32, f32,
                                               i32, p, i64, p]
    lib.mquant_w4a8_linear_prefill_static.argtypes = [p, i64, p, p, p, p, i64, i32, i32, i32, i32, f32, f32,
                                                      i32, p]
    lib.mquant_w4a8_gemv_grouped.argtypes = [p, i32, i32, i32, f32, f32, p, i32, p]
    lib.mquant_w4a8_linear_decode_grouped.argtypes = [p, i64, i32, i32, i32, f32, f32, i32, p, i32, p]
    lib.mquant_rope_apply.argtypes = [p, i64, p, i32, i32, i32, ctypes.c_double, p]
    lib.mquant_aifs_attention_workspace_bytes.restype = i64
    lib.mquant_aifs_attention_workspace_bytes.argtypes = [i32, i32, i32]
    lib.mquant_aifs_attention.argtypes = [p, i64, p, i64, p, i64, p, i64, p, i32, i32, i32, i32, p, i64, p]
    lib.mquant_w4a8_linear_decode.argtypes = [p, i64, p, p, p, i64, i32, i32, i32, i32, f32, f32, i32, p]
    lib.mquant_w4g128_prepacked_bytes.restype = i64
    lib.mquant_w4g128_prepacked_bytes.argtypes = [i32, i32]
    lib.mquant_w4g128_prepack.argtypes = [p, p, p, i32, i32, p]
    lib.mquant_w4g128_gemm.argtypes = [p, i64, p, p, i64, i32, i32, i32, p]
    f64 = ctypes.c_double
    lib.mquant_qk_norm_rope.argtypes = [p, i64, p, i64, p, i64, p, i64, p, p, f32, p, i32, i32, i32, i32, f64, p]
    lib.mquant_kv_append.argtypes = [p, i64, p, i64, p, i64, p, i64, p, p, f32, p, p, p, i32, i32, f64, p, p]
    lib.mquant_paged_attention_workspace_bytes.restype = i64
    lib.mquant_paged_attention_workspace_bytes.argtypes = [i32] * 7
    lib.mquant_paged_attention.argtypes = [p, i64, p, p, p, p, i64, i32, i32, i32, i32, p, i64, p]
    lib.mquant_lora_workspace_bytes.restype = i64
    lib.mquant_lora_workspace_bytes.argtypes = [i32, i32, i32]
    lib.mquant_lora_apply.argtypes = [p, i64, p, p, p, p, p, p, i64, p, i64, i32, i32, i32, i32, i32, p, i64, p]
    for name in EXPORTS:
        if name not in ("mquant_status_string", "mquant_w4_prepacked_bytes", "mquant_aifs_attention_workspace_bytes",
                        "mquant_build_id", "mquant_w4g128_prepacked_bytes",
                        "mquant_paged_attention_workspace_bytes", "mquant_lora_workspace_bytes",
                        "mquant_w4a8_workspace_bytes", "mquant_w4a8_linear_prefill_workspace_bytes",
                        "mquant_version"):
            getattr(lib, name).restype = ctypes.c_int
    return lib


lib = _load()


def status_string(status: int) -> str:
    return lib.mquant_status_string(int(status)).decode()


def version() -> int:
    return int(lib.mquant_version())


def build_id() -> str:
    return lib.mquant_build_id().decode()


TUNE_GEMM_TILE, TUNE_GEMM_NOSPLIT, TUNE_G128_TILE, TUNE_GEMV_VARIANT, TUNE_G128_SHAPE = 0, 1, 2, 3, 4
TUNE_GEMM_SHAPE = 5


def tune_set(key: int, value: int) -> None:
    _check(lib.mquant_tune_set(int(key), int(value)), "mquant_tune_set")


def static_scale_from_absmax(absmax_u: float, had_block: int, act_bits: int = 8) -> float:
    """Eq. (2)'s static scale from the statistic of ``hadamard_absmax`` (computed by the library)."""
    out = ctypes.c_float(0.0)
    _check(lib.mquant_static_scale_from_absmax(float(absmax_u), int(had_block), int(act_bits),
                                               ctypes.cast(ctypes.byref(out), ctypes.c_void_p)),
           "mquant_static_scale_from_absmax")
    return float(out.value)


def _check(status: int, where: str) -> None:
    if status != OK:
        raise MQuantError(int(status), where)


def _dp(t) -> Optional[int]:
    """Device (or host) address of a torch tensor; None stays NULL."""
    return None if t is None else t.data_ptr()


def _rows(t, what: str) -> int:
    """A 2-D operand the ABI addresses through a leading dimension, which is returned: unit
    stride along a row."""
    st = t.stride()
    if len(st) == 2:
        rows, cols = t.shape
        if (st[1] == 1 or cols <= 1) and (st[0] >= cols or rows <= 1):
            return st[0]
    raise MQuantError(ERR_BAD_SHAPE, f"{what}: expected a 2-D tensor with unit column stride")


def _dense(t, what: str) -> None:
    """An operand the ABI takes without a leading dimension."""
    if t is not None and not t.is_contiguous():
        raise MQuantError(ERR_BAD_SHAPE, f"{what}: expected a contiguous tensor")


# torch.cuda.current_stream() builds a stream object around the handle (2.8 us a call against 0.2 us
# for the handle, of about 8 us that a launch through this module costs the host); a build of
# torch without the accessors takes the long way.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream() -> Optional[int]:
    """Handle of this thread's current stream on its current device; None for the default stream."""
    if _raw_stream is None or _device is None or not torch.cuda.is_initialized():
        return torch.cuda.current_stream().cuda_stream or None
    return _raw_stream(_device()) or None


class _SlowWay:
    """In the place of the call module: takes no call."""
    def __getattr__(self, _):
        return lambda *_: NotImplemented


def _load_fast():
    """The module of csrc/fastcall.c, whose functions take the ordinary calls to the library (2.3 us less of the
    host's time each); where it cannot, they return NotImplemented and the caller goes on through ctypes, as all
    calls do where this interpreter has no such module built."""
    if not os.path.exists(FAST_PATH) or _raw_stream is None or _device is None:
        return _SlowWay()
    loader = importlib.machinery.ExtensionFileLoader("mquant_fastcall", FAST_PATH)
    mod = importlib.util.module_from_spec(importlib.util.spec_from_file_location("mquant_fastcall", FAST_PATH, loader=loader))
    loader.exec_module(mod)
    mod.setup(torch.cuda.is_initialized, _device, _raw_stream, *(
        ctypes.cast(getattr(lib, "mquant_" + f), ctypes.c_void_p).value
        for f in ("w4a8_linear_prefill", "w4a8_linear_prefill_static", "w4a8_linear_decode", "w4a8_linear_decode_grouped",
                  "w4a8_gemv_grouped", "hadamard_quant_act", "w4g128_gemm")))
    mod.setup_serving(torch.float16, torch.float32, torch.int32, *(
        ctypes.cast(getattr(lib, "mquant_" + f), ctypes.c_void_p).value
        for f in ("qk_norm_rope", "kv_append", "paged_attention", "lora_apply")))
    return mod


_fast = _load_fast()

_linear_packers = [struct.Struct("@" + "PPPqi4x" * n) for n in range(9)]
assert _linear_packers[1].size == ctypes.sizeof(Linear)


def _linears(linears) -> bytes:
    """An array of mquant_linear_t (the layout of Linear), packed in one go: filling ctypes
    structures field by field costs 1.3 us per linear on the way to a launch."""
    vals = []
    for wp, ws, N, out in linears:
        ld = _rows(out, "y")
        _dense(ws, "w_scale")
        vals += (_dp(wp) or 0, _dp(ws) or 0, _dp(out) or 0, ld, N)
    n = len(linears)
    try:
        return (_linear_packers[n] if n < len(_linear_packers) else struct.Struct("@" + "PPPqi4x" * n)).pack(*vals)
    except struct.error:
        for i, (_, _, N, _) in enumerate(linears):
            if not -2 ** 31 <= operator.index(N) < 2 ** 31:       # index: TypeError for what is no integer
                raise MQuantError(ERR_BAD_SHAPE, f"linear {i}: N = {N}") from None
        raise


# ------------------------------------------------------------------- host

def aifs_build_perm(T: int, vis_spans: Sequence[Tuple[int, int]]):
    """-> (perm int32[T], inv_perm int32[T], n_vis) as numpy arrays (host)."""
    n = len(vis_spans)
    arr = (Span * max(n, 1))()
    for i, (s, l) in enumerate(vis_spans):
        arr[i].start, arr[i].len = int(s), int(l)
    perm = np.empty(max(T, 0), dtype=np.int32)
    inv = np.empty(max(T, 0), dtype=np.int32)
    n_vis = ctypes.c_int32(0)
    st = lib.mquant_aifs_build_perm(T, ctypes.cast(arr, ctypes.c_void_p) if n else None, n,
                                    perm.ctypes.data, inv.ctypes.data,
                                    ctypes.cast(ctypes.byref(n_vis), ctypes.c_void_p))
    _check(st, "mquant_aifs_build_perm")
    return perm, inv, int(n_vis.value)


# ----------------------------------------------------------------- device

def aifs_permute(x, perm_dev, out=None):
    T, K = x.shape
    if out is None:
        out = torch.empty((T, K), dtype=x.dtype, device=x.device)
    _rows(x, "aifs_permute x"), _rows(out, "aifs_permute out"), _dense(perm_dev, "perm")
    _check(lib.mquant_aifs_permute(_dp(x), x.stride(0), _dp(out), out.stride(0), _dp(perm_dev),
                                   T, K, _stream()), "mquant_aifs_permute")
    return out


def aifs_remap_mask(mask, perm_dev, out=None):
    T = mask.shape[0]
    if out is None:
        out = torch.empty((T, T), dtype=torch.uint8, device=mask.device)
    _dense(mask, "mask"), _dense(out, "mask_u"), _dense(perm_dev, "perm")
    _check(lib.mquant_aifs_remap_mask(_dp(mask), _dp(out), _dp(perm_dev), T, _stream()),
           "mquant_aifs_remap_mask")
    return out


def hadamard_quant_act(x, n_vis: int, s_vis: float, s_txt: float, had_block: int,
                       perm_dev=None, out=None, T: Optional[int] = None, act_bits: Optional[int] = None):
    if act_bits is None and T is None and out is not None:
        st = _fast.quant(x, n_vis, s_vis, s_txt, had_block, perm_dev, out)
        if st is not NotImplemented:
            _check(st, "mquant_hadamard_quant_act")
            return out
    rows, K = x.shape
    T = rows if T is None else T
    if out is None:
        out = torch.empty((T, K), dtype=torch.int8, device=x.device)
    _rows(x, "hadamard_quant_act x"), _dense(out, "xq"), _dense(perm_dev, "perm")
    if act_bits is None:
        _check(lib.mquant_hadamard_quant_act(_dp(x), x.stride(0), _dp(perm_dev), _dp(out), T, K, n_vis,
                                             s_vis, s_txt, had_block, _stream()),
               "mquant_hadamard_quant_act")
    else:
        _check(lib.mquant_hadamard_quant_act_bits(_dp(x), x.stride(0), _dp(perm_dev), _dp(out), T, K,
                                                  n_vis, s_vis, s_txt, had_block, act_bits, _stream()),
               "mquant_hadamard_quant_act_bits")
    return out


def hadamard_absmax(x, had_block: int, absmax_dev):
    T, K = x.shape
    _rows(x, "hadamard_absmax x")
    _check(lib.mquant_hadamard_absmax(_dp(x), x.stride(0), T, K, had_block, _dp(absmax_dev),
                                      _stream()), "mquant_hadamard_absmax")
    return absmax_dev


def w4_prepacked_bytes(N: int, K: int) -> int:
    n = int(lib.mquant_w4_prepacked_bytes(N, K))
    if n < 0:
        raise MQuantError(n, "mquant_w4_prepacked_bytes")
    return n


def w4_prepack(w_canonical, out=None):
    N, K2 = w_canonical.shape
    K = 2 * K2
    if out is None:
        out = torch.empty(w4_prepacked_bytes(N, K), dtype=torch.uint8, device=w_canonical.device)
    _dense(w_canonical, "w_canonical"), _dense(out, "w_prepacked")
    _check(lib.mquant_w4_prepack(_dp(w_canonical), _dp(out), N, K, _stream()), "mquant_w4_prepack")
    return out


def w4a8_workspace_bytes(T: int, N: int, K: int) -> int:
    n = int(lib.mquant_w4a8_workspace_bytes(T, N, K))
    if n < 0:
        raise MQuantError(n, "mquant_w4a8_workspace_bytes")
    return n


def w4a8_gemm(xq, w_prepacked, w_scale, N: int, n_vis: int, s_vis: float, s_txt: float,
              out=None, acc_out=None, workspace=None):
    T, K = xq.shape
    if out is None:
        out = torch.empty((T, N), dtype=torch.float16, device=xq.device)
    if workspace is None:
        need = w4a8_workspace_bytes(T, N, K)
        if need:
            workspace = torch.empty(need, dtype=torch.uint8, device=xq.device)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _dense(xq, "xq"), _rows(out, "y"), _dense(acc_out, "acc_out"), _dense(w_scale, "w_scale")
    _check(lib.mquant_w4a8_gemm(_dp(xq), _dp(w_prepacked), _dp(w_scale), _dp(out), out.stride(0),
                                _dp(acc_out), T, N, K, n_vis, s_vis, s_txt, _dp(workspace),
                                ws_bytes, _stream()), "mquant_w4a8_gemm")
    return out


def hadamard_dynquant_act(x, had_block: int, perm_dev=None, out=None, row_scale=None):
    T, K = x.shape
    if out is None:
        out = torch.empty((T, K), dtype=torch.int8, device=x.device)
    if row_scale is None:
        row_scale = torch.empty((T,), dtype=torch.float32, device=x.device)
    _rows(x, "x"), _dense(out, "xq"), _dense(row_scale, "row_scale"), _dense(perm_dev, "perm")
    _check(lib.mquant_hadamard_dynquant_act(_dp(x), x.stride(0), _dp(perm_dev), _dp(out),
                                            _dp(row_scale), T, K, had_block, _stream()),
           "mquant_hadamard_dynquant_act")
    return out, row_scale


def w4a8_gemm_rowscale(xq, w_prepacked, w_scale, row_scale, N: int, out=None, acc_out=None,
                       workspace=None):
    T, K = xq.shape
    if out is None:
        out = torch.empty((T, N), dtype=torch.float16, device=xq.device)
    if workspace is None:
        need = w4a8_workspace_bytes(T, N, K)
        if need:
            workspace = torch.empty(need, dtype=torch.uint8, device=xq.device)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _dense(xq, "xq"), _rows(out, "y"), _dense(acc_out, "acc_out"), _dense(row_scale, "row_scale")
    _check(lib.mquant_w4a8_gemm_rowscale(_dp(xq), _dp(w_prepacked), _dp(w_scale), _dp(row_scale),
                                         _dp(out), out.stride(0), _dp(acc_out), T, N, K,
                                         _dp(workspace), ws_bytes, _stream()),
           "mquant_w4a8_gemm_rowscale")
    return out


def w4a8_gemm_rms(xq, w_prepacked, w_scale, N: int, n_vis: int, s_vis: float, s_txt: float,
                  split_idx, split_w, split_scale, out=None, acc_out=None, workspace=None):
    """split_idx (int32) and split_scale (fp32) are HOST arrays (per-layer constants),
    split_w is a device tensor int8 [n_split, N]."""
    T, K = xq.shape
    if split_idx is None:
        n_split, idx_p, sc_p = 0, None, None
    else:
        idx = np.ascontiguousarray(split_idx, dtype=np.int32)
        sc = np.ascontiguousarray(split_scale, dtype=np.float32)
        n_split = int(idx.shape[0])
        idx_p, sc_p = idx.ctypes.data_as(ctypes.c_void_p), sc.ctypes.data_as(ctypes.c_void_p)
    if out is None:
        out = torch.empty((T, N), dtype=torch.float16, device=xq.device)
    if workspace is None:
        need = w4a8_workspace_bytes(T, N, K)
        if need:
            workspace = torch.empty(need, dtype=torch.uint8, device=xq.device)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _dense(xq, "xq"), _rows(out, "y"), _dense(acc_out, "acc_out"), _dense(split_w, "split_w")
    _check(lib.mquant_w4a8_gemm_rms(_dp(xq), _dp(w_prepacked), _dp(w_scale), _dp(out), out.stride(0),
                                    _dp(acc_out), T, N, K, n_vis, s_vis, s_txt, idx_p,
                                    _dp(split_w), sc_p, n_split, _dp(workspace),
                                    ws_bytes, _stream()), "mquant_w4a8_gemm_rms")
    return out


def w4a8_linear_prefill_workspace_bytes(T: int, N: int, K: int) -> int:
    n = int(lib.mquant_w4a8_linear_prefill_workspace_bytes(T, N, K))
    if n < 0:
        raise MQuantError(n, "mquant_w4a8_linear_prefill_workspace_bytes")
    return n


def w4a8_linear_prefill(x, perm_dev, w_prepacked, w_scale, N: int, n_vis: int, s_vis: float,
                        s_txt: float, had_block: int, workspace, out=None):
    T, K = x.shape
    if out is None:
        out = torch.empty((T, N), dtype=torch.float16, device=x.device)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = _fast.prefill(x, perm_dev, w_prepacked, w_scale, N, n_vis, s_vis, s_txt, had_block, out, workspace, ws_bytes)
    if st is not NotImplemented:
        _check(st, "mquant_w4a8_linear_prefill")
        return out
    _rows(x, "x"), _rows(out, "y"), _dense(perm_dev, "perm"), _dense(w_scale, "w_scale")
    _check(lib.mquant_w4a8_linear_prefill(_dp(x), x.stride(0), _dp(perm_dev), _dp(w_prepacked),
                                          _dp(w_scale), _dp(out), out.stride(0), T, N, K, n_vis,
                                          s_vis, s_txt, had_block, _dp(workspace), ws_bytes,
                                          _stream()), "mquant_w4a8_linear_prefill")
    return out


def w4a8_gemv_grouped(xq, linears, n_vis: int, s_vis: float, s_txt: float):
    """linears: sequence of (w_prepacked, w_scale, N, out) sharing the input xq [T, K];
    one launch computes every out [T, N]."""
    st = _fast.gemv_grouped(xq, linears, n_vis, s_vis, s_txt)
    if st is not NotImplemented:
        _check(st, "mquant_w4a8_gemv_grouped")
        return [l[3] for l in linears]
    T, K = xq.shape
    _dense(xq, "xq")
    _check(lib.mquant_w4a8_gemv_grouped(_dp(xq), T, K, n_vis, s_vis, s_txt, _linears(linears), len(linears),
                                        _stream()), "mquant_w4a8_gemv_grouped")
    return [l[3] for l in linears]


STATIC_SCRATCH_BYTES = 128 << 20


def w4a8_linear_prefill_static(x, perm_dev, w_prepacked, w_scale, N: int, n_vis: int, s_vis: float,
                               s_txt: float, had_block: int, out):
    """The fused prefill entry on the library's own scratch array; `out` is required (the
    point of the entry is that nothing gets allocated)."""
    st = _fast.prefill_static(x, perm_dev, w_prepacked, w_scale, N, n_vis, s_vis, s_txt, had_block, out)
    if st is not NotImplemented:
        _check(st, "mquant_w4a8_linear_prefill_static")
        return out
    T, K = x.shape
    _rows(x, "x"), _rows(out, "y"), _dense(perm_dev, "perm"), _dense(w_scale, "w_scale")
    _check(lib.mquant_w4a8_linear_prefill_static(_dp(x), x.stride(0), _dp(perm_dev), _dp(w_prepacked),
                                                 _dp(w_scale), _dp(out), out.stride(0), T, N, K, n_vis,
                                                 s_vis, s_txt, had_block, _stream()),
           "mquant_w4a8_linear_prefill_static")
    return out


def rope_apply(x, pos_dev, n_heads: int, head_dim: int = 128, base: float = 10000.0):
    """In place on x [T, >= n_heads*head_dim] fp16."""
    T = x.shape[0]
    _check(lib.mquant_rope_apply(_dp(x), x.stride(0), _dp(pos_dev), T, n_heads, head_dim,
                                 float(base), _stream()), "mquant_rope_apply")
    return x


def aifs_attention_workspace_bytes(T: int, n_kv_heads: int, head_dim: int = 128) -> int:
    n = int(lib.mquant_aifs_attention_workspace_bytes(T, n_kv_heads, head_dim))
    if n < 0:
        raise MQuantError(n, "mquant_aifs_attention_workspace_bytes")
    return n


def aifs_attention(q, k, v, pos_dev, n_q_heads: int, n_kv_heads: int, head_dim: int = 128,
                   out=None, workspace=None):
    """q [T, >= Hq*D], k, v [T, >= Hkv*D] fp16 views (row strides are passed on)."""
    T = q.shape[0]
    if out is None:
        out = torch.empty((T, n_q_heads * head_dim), dtype=torch.float16, device=q.device)
    if workspace is None:
        workspace = torch.empty(max(aifs_attention_workspace_bytes(T, n_kv_heads, head_dim), 256),
                                dtype=torch.uint8, device=q.device)
    ws_bytes = workspace.numel() * workspace.element_size()
    _check(lib.mquant_aifs_attention(_dp(q), q.stride(0), _dp(k), k.stride(0), _dp(v), v.stride(0),
                                     _dp(out), out.stride(0), _dp(pos_dev), T, n_q_heads, n_kv_heads,
                                     head_dim, _dp(workspace), ws_bytes, _stream()),
           "mquant_aifs_attention")
    return out


def w4a8_linear_decode(x, w_prepacked, w_scale, N: int, n_vis: int, s_vis: float, s_txt: float,
                       had_block: int, out=None):
    """x fp16 [T <= 4, K] -> y fp16 [T, N]: rotate, quantize, GEMV and dequant in one launch."""
    T, K = x.shape
    if out is None:
        out = torch.empty((T, N), dtype=torch.float16, device=x.device)
    st = _fast.decode(x, w_prepacked, w_scale, N, n_vis, s_vis, s_txt, had_block, out)
    if st is not NotImplemented:
        _check(st, "mquant_w4a8_linear_decode")
        return out
    _check(lib.mquant_w4a8_linear_decode(_dp(x), x.stride(0), _dp(w_prepacked), _dp(w_scale), _dp(out),
                                         out.stride(0), T, N, K, n_vis, s_vis, s_txt, had_block,
                                         _stream()), "mquant_w4a8_linear_decode")
    return out


def w4a8_linear_decode_grouped(x, linears, n_vis: int, s_vis: float, s_txt: float, had_block: int):
    """x fp16 [T <= 4, K]; linears: sequence of (w_prepacked, w_scale, N, out) sharing x.
    One launch rotates and quantizes x and computes every out [T, N]."""
    st = _fast.decode_grouped(x, linears, n_vis, s_vis, s_txt, had_block)
    if st is not NotImplemented:
        _check(st, "mquant_w4a8_linear_decode_grouped")
        return [l[3] for l in linears]
    T, K = x.shape
    ldx = _rows(x, "x")
    _check(lib.mquant_w4a8_linear_decode_grouped(_dp(x), ldx, T, K, n_vis, s_vis, s_txt, had_block,
                                                 _linears(linears), len(linears), _stream()),
           "mquant_w4a8_linear_decode_grouped")
    return [l[3] for l in linears]


def w4g128_prepacked_bytes(N: int, K: int) -> int:
    n = int(lib.mquant_w4g128_prepacked_bytes(N, K))
    if n < 0:
        raise MQuantError(n, "mquant_w4g128_prepacked_bytes")
    return n


def w4g128_prepack(w_canonical, scales, out=None):
    """w_canonical uint8 [N, K/2], scales fp16 [N, K/128] -> the weight-only kernel's layout."""
    N, K2 = w_canonical.shape
    K = 2 * K2
    if out is None:
        out = torch.empty(w4g128_prepacked_bytes(N, K), dtype=torch.uint8, device=w_canonical.device)
    if tuple(scales.shape) != (N, K // 128) or not scales.is_contiguous():
        raise MQuantError(ERR_BAD_SHAPE, "w4g128_prepack: scales must be contiguous [N, K/128]")
    _check(lib.mquant_w4g128_prepack(_dp(w_canonical), _dp(scales), _dp(out), N, K, _stream()),
           "mquant_w4g128_prepack")
    return out


def w4g128_gemm(x, w_prepacked, N: int, out=None):
    """x fp16 [T, K] (row stride in elements) -> y fp16 [T, N] = x W~^T, group-wise dequantised weight."""
    T, K = x.shape
    if out is None:
        out = torch.empty((T, N), dtype=torch.float16, device=x.device)
    st = _fast.weight_only(x, w_prepacked, N, out)
    if st is not NotImplemented:
        _check(st, "mquant_w4g128_gemm")
        return out
    _check(lib.mquant_w4g128_gemm(_dp(x), x.stride(0) if T > 0 else K, _dp(w_prepacked), _dp(out),
                                  out.stride(0) if T > 0 else N, T, N, K, _stream()), "mquant_w4g128_gemm")
    return out


# ----------------------------------------------------------- serving step

def _operand(t, dtype, what: str, shape=None, counted: bool = True):
    """A device operand of the serving entries: on the current device, of this type, and of `shape` (contiguous) or
    2-D with unit column stride, whose leading dimension is returned.  The ABI counts in 32 bits (scratch aside)."""
    if not t.is_cuda or t.get_device() != torch.cuda.current_device():
        raise MQuantError(ERR_UNSUPPORTED, f"{what}: expected a tensor on the current device")
    if t.dtype is not dtype:
        raise MQuantError(ERR_UNSUPPORTED, f"{what}: expected {dtype}, got {t.dtype}")
    if counted and max(t.shape, default=0) > 0x7fffffff:
        raise MQuantError(ERR_UNSUPPORTED, f"{what}: a size of {tuple(t.shape)} is beyond 32 bits")
    if shape is None:
        ld = 0 if t.dim() == 2 and t.shape[0] == 0 else _rows(t, what)
        return ld if t.shape[0] > 1 else t.shape[1] + -t.shape[1] % 8       # the stride of a single row, or of none, says nothing
    if tuple(t.shape) != shape:
        raise MQuantError(ERR_BAD_SHAPE, f"{what}: expected shape {shape}, got {tuple(t.shape)}")
    _dense(t, what)
    return 0


def _heads(t, n: int, head_dim: int, rows: int, what: str) -> int:
    ld = _operand(t, torch.float16, what)
    if t.shape[0] != rows or t.shape[1] < n * head_dim:
        raise MQuantError(ERR_BAD_SHAPE, f"{what}: expected [{rows}, >= {n * head_dim}], got {tuple(t.shape)}")
    return ld


class PagedCache:
    """A paged key/value cache (mquant_paged_cache_t) over the caller's tensors: k_pages, v_pages fp16 [n_pages,
    n_kv_heads, page_size, head_dim] and page_table int32 [n_seq, table_pages]."""

    def __init__(self, k_pages, v_pages, page_table):
        if k_pages.dim() != 4 or page_table.dim() != 2:
            raise MQuantError(ERR_BAD_SHAPE, "PagedCache: expected k_pages [pages, heads, page size, head dim], page_table [sequences, pages]")
        _operand(k_pages, torch.float16, "k_pages", tuple(k_pages.shape))
        _operand(v_pages, torch.float16, "v_pages", tuple(k_pages.shape))
        _operand(page_table, torch.int32, "page_table", tuple(page_table.shape))
        self.k_pages, self.v_pages, self.page_table = k_pages, v_pages, page_table
        (self.n_pages, self.n_kv_heads, self.page_size, self.head_dim), (self.n_seq, self.table_pages) = k_pages.shape, page_table.shape
        self.slots = self.table_pages * self.page_size
        self.device_index = k_pages.device.index
        self.struct = PagedCacheStruct(_dp(k_pages), _dp(v_pages), _dp(page_table), self.n_seq, self.n_pages, self.page_size,
                                       self.table_pages, self.n_kv_heads, self.head_dim)
        self.address = ctypes.addressof(self.struct)
        self.fast = (self.address, self.n_seq, self.n_kv_heads, self.head_dim, self.device_index)


def _step(cache, row_start_dev, pos_dev, T: int) -> None:
    if cache.device_index != torch.cuda.current_device():
        raise MQuantError(ERR_UNSUPPORTED, "cache: expected tensors on the current device")
    _operand(row_start_dev, torch.int32, "row_start", (cache.n_seq + 1,))
    _operand(pos_dev, torch.int32, "pos", (T,))


def _workspace(ws) -> None:
    if ws is not None:
        _operand(ws, ws.dtype, "workspace", tuple(ws.shape), counted=False)


def _weight(w, head_dim: int, what: str) -> None:
    if w is not None:
        _operand(w, torch.float16, what, (head_dim,))


def qk_norm_rope(q, k, q_weight, k_weight, pos_dev, n_q_heads: int, n_kv_heads: int, head_dim: int = 128, eps: float = 1e-6,
                 base: float = 10000.0, q_out=None, k_out=None):
    """q [T, >= Hq*D], k [T, >= Hkv*D] fp16 views -> (q_out, k_out); pass q_out=q, k_out=k to work in place."""
    T = q.shape[0]
    if q_out is None:
        q_out = torch.empty((T, n_q_heads * head_dim), dtype=torch.float16, device=q.device)
    if k_out is None:
        k_out = torch.empty((T, n_kv_heads * head_dim), dtype=torch.float16, device=q.device)
    st = _fast.norm(q, k, q_weight, k_weight, pos_dev, n_q_heads, n_kv_heads, head_dim, eps, base, q_out, k_out)
    if st is not NotImplemented:
        _check(st, "mquant_qk_norm_rope")
        return q_out, k_out
    lds = [_heads(t, n, head_dim, T, what) for t, n, what in ((q, n_q_heads, "q"), (q_out, n_q_heads, "q_out"),
                                                               (k, n_kv_heads, "k"), (k_out, n_kv_heads, "k_out"))]
    _weight(q_weight, head_dim, "q_weight"), _weight(k_weight, head_dim, "k_weight")
    _operand(pos_dev, torch.int32, "pos", (T,))
    _check(lib.mquant_qk_norm_rope(_dp(q), lds[0], _dp(q_out), lds[1], _dp(k), lds[2], _dp(k_out), lds[3], _dp(q_weight),
                                   _dp(k_weight), eps, _dp(pos_dev), T, n_q_heads, n_kv_heads, head_dim, base, _stream()),
           "mquant_qk_norm_rope")
    return q_out, k_out


def kv_append(q, k, v, cache: PagedCache, row_start_dev, pos_dev, n_q_heads: int, q_weight=None, k_weight=None,
              eps: float = 1e-6, base: float = 10000.0, rope_pos_dev=None, q_out=None):
    """Norm and rotation of q and k [T, heads * D] and the write of k and v to the cache's slots -> q_out."""
    T, D = q.shape[0], cache.head_dim
    if q_out is None:
        q_out = torch.empty((T, n_q_heads * D), dtype=torch.float16, device=q.device)
    st = _fast.append(q, k, v, cache.fast, row_start_dev, pos_dev, n_q_heads, q_weight, k_weight, eps, base, rope_pos_dev, q_out)
    if st is not NotImplemented:
        _check(st, "mquant_kv_append")
        return q_out
    lds = [_heads(t, n, D, T, what) for t, n, what in ((q, n_q_heads, "q"), (q_out, n_q_heads, "q_out"),
                                                        (k, cache.n_kv_heads, "k"), (v, cache.n_kv_heads, "v"))]
    _weight(q_weight, D, "q_weight"), _weight(k_weight, D, "k_weight")
    _step(cache, row_start_dev, pos_dev, T)
    if rope_pos_dev is not None:
        _operand(rope_pos_dev, torch.int32, "rope_pos", (T,))
    _check(lib.mquant_kv_append(_dp(q), lds[0], _dp(q_out), lds[1], _dp(k), lds[2], _dp(v), lds[3], _dp(q_weight), _dp(k_weight),
                                eps, _dp(row_start_dev), _dp(pos_dev), _dp(rope_pos_dev), T, n_q_heads, base, cache.address,
                                _stream()), "mquant_kv_append")
    return q_out


def paged_attention_workspace_bytes(T: int, cache: PagedCache, n_q_heads: int, max_rows: int = 0, max_kv: int = 0) -> int:
    n = int(lib.mquant_paged_attention_workspace_bytes(T, cache.n_seq, n_q_heads, cache.n_kv_heads, cache.head_dim, max_rows,
                                                       min(max_kv, cache.slots) if max_kv else cache.slots))
    if n < 0:
        raise MQuantError(n, "mquant_paged_attention_workspace_bytes")
    return n


def paged_attention(q, cache: PagedCache, row_start_dev, pos_dev, n_q_heads: int, max_rows: int = 0, max_kv: int = 0,
                    out=None, workspace=None):
    """q [T, >= Hq*D] fp16 of the step's rows -> o [T, Hq*D]; max_rows, max_kv: host bounds (0: not known)."""
    T, D = q.shape[0], cache.head_dim
    if max_kv > cache.slots:
        max_kv = cache.slots
    if out is None:
        out = torch.empty((T, n_q_heads * D), dtype=torch.float16, device=q.device)
    if workspace is None:
        need = paged_attention_workspace_bytes(T, cache, n_q_heads, max_rows, max_kv)
        if need:
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    st = _fast.attention(q, cache.fast, row_start_dev, pos_dev, n_q_heads, max_rows, max_kv, out, workspace, ws_bytes)
    if st is not NotImplemented:
        _check(st, "mquant_paged_attention")
        return out
    ldq, ldo = _heads(q, n_q_heads, D, T, "q"), _heads(out, n_q_heads, D, T, "out")
    _step(cache, row_start_dev, pos_dev, T), _workspace(workspace)
    _check(lib.mquant_paged_attention(_dp(q), ldq, cache.address, _dp(row_start_dev), _dp(pos_dev), _dp(out), ldo, T, n_q_heads,
                                      max_rows, max_kv, _dp(workspace), ws_bytes, _stream()), "mquant_paged_attention")
    return out


def lora_workspace_bytes(T: int, K: int, rank: int) -> int:
    n = int(lib.mquant_lora_workspace_bytes(T, K, rank))
    if n < 0:
        raise MQuantError(n, "mquant_lora_workspace_bytes")
    return n


def lora_apply(x, adapter_dev, a, b, scale, base, perm_dev=None, out=None, workspace=None):
    """y = base + scale[id] * (x A_id^T) B_id^T per row, id = adapter[row] (outside the adapters: y = base); x [T, K], base
    [T, N], a [adapters, rank, K], b [adapters, N, rank]; pass out=base to add in place."""
    T, K = x.shape
    N, (n_adapters, rank) = base.shape[1], a.shape[:2]
    if out is None:
        out = torch.empty((T, N), dtype=torch.float16, device=x.device)
    if workspace is None:
        workspace = torch.empty(max(lora_workspace_bytes(T, K, rank), 256), dtype=torch.uint8, device=x.device)
    ws_bytes = workspace.numel() * workspace.element_size()
    st = _fast.lora(x, adapter_dev, a, b, scale, base, perm_dev, out, workspace, ws_bytes)
    if st is not NotImplemented:
        _check(st, "mquant_lora_apply")
        return out
    ldx, ldb, ldy = (_operand(t, torch.float16, what) for t, what in ((x, "x"), (base, "base"), (out, "out")))
    if base.shape[0] != T or tuple(out.shape) != (T, N):
        raise MQuantError(ERR_BAD_SHAPE, f"lora_apply: base and out must be [{T}, {N}]")
    _operand(adapter_dev, torch.int32, "adapter", (T,))
    _operand(a, torch.float16, "a", (n_adapters, rank, K)), _operand(b, torch.float16, "b", (n_adapters, N, rank))
    _operand(scale, torch.float32, "scale", (n_adapters,)), _workspace(workspace)
    if perm_dev is not None:
        _operand(perm_dev, torch.int32, "perm", (T,))
    _check(lib.mquant_lora_apply(_dp(x), ldx, _dp(perm_dev), _dp(adapter_dev), _dp(a), _dp(b), _dp(scale), _dp(base), ldb,
                                 _dp(out), ldy, T, N, K, rank, n_adapters, _dp(workspace), ws_bytes, _stream()),
           "mquant_lora_apply")
    return out
