"""ctypes binding of libsymb.so: argument marshalling only.

Every function here has the name of the C entry point it calls (include/symb.h, include/symb_block.h) and
does nothing but turn torch tensors into device pointers and host lists into C arrays.
All arithmetic runs in the HIP kernels; there is no CPU or PyTorch fallback: if the
library is missing, `lib()` raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from dataclasses import dataclass
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsymb.so")

SYMB_OK, SYMB_ERR_INVALID_ARG, SYMB_ERR_BAD_SEGMENTS, SYMB_ERR_UNSUPPORTED, \
    SYMB_ERR_WORKSPACE_TOO_SMALL, SYMB_ERR_DEVICE = range(6)
SYMB_ADAPTER_NONE, SYMB_ADAPTER_LORA, SYMB_ADAPTER_IA3, SYMB_ADAPTER_IA3_IN = range(4)
SYMB_OP_FWD, SYMB_OP_BWD_INPUT, SYMB_OP_ADAPTER_GRAD, SYMB_OP_FWD_INPLACE, SYMB_OP_BWD_INPUT_INPLACE = range(5)
SYMB_OPT_DESCRIPTOR_REUSE, SYMB_OPT_K_SPLIT, SYMB_OPT_SMALL_BATCH_KERNELS, SYMB_OPT_SKINNY_DEEP = range(4)
SYMB_STATIC_SCRATCH_BYTES = 32 << 20
SYMB_BWD_FULL, SYMB_BWD_BASE_ONLY, SYMB_BWD_REUSE_DH = 0, 1, 2
SYMB_GRAD_OVERWRITE, SYMB_GRAD_ACCUMULATE, SYMB_GRAD_REUSE_DH, SYMB_GRAD_REUSE_HS = 0, 1, 2, 4
SYMB_MAX_RANK = 128
SYMB_WEIGHT_LINEAR, SYMB_WEIGHT_CONV1D = 0, 1
SYMB_NORM_LAYER, SYMB_NORM_RMS = 0, 1
SYMB_NORM_MAX_WIDTH = 16384
SYMB_ROTATE_HALVES, SYMB_ROTATE_ADJACENT = 0, 1

EXPORTS = ("symb_create", "symb_destroy", "symb_validate_batch", "symb_debug_row_segment_map",
           "symb_plan_row_tiles", "symb_workspace_bytes", "symb_base_linear_fwd",
           "symb_base_linear_bwd_input", "symb_base_linear_bwd_input_ex", "symb_adapter_grad", "symb_adapter_grad_ex",
           "symb_noise_add", "symb_base_linear_fwd_denoise", "symb_base_linear_fwd_seg", "symb_base_linear_bwd_input_seg",
           "symb_adapter_grad_seg",
           "symb_status_string", "symb_last_error",
           "symb_batcher_create", "symb_batcher_destroy", "symb_batcher_submit", "symb_batcher_pending",
           "symb_batcher_next_due", "symb_batcher_take",
           "symb_debug_gemm_timing_enable", "symb_debug_gemm_timing_read", "symb_debug_descriptor_stats",
           "symb_debug_set_option", "symb_debug_xcd_rule", "symb_base_linear_fwd_static",
           "symb_norm_workspace_bytes", "symb_norm_fwd", "symb_norm_bwd", "symb_kv_append", "symb_kv_workspace_bytes", "symb_kv_attention")


class symb_adapter(C.Structure):
    _fields_ = [("kind", C.c_int32), ("rank", C.c_int32), ("scale", C.c_float),
                ("A", C.c_void_p), ("B", C.c_void_p), ("dA", C.c_void_p), ("dB", C.c_void_p)]


class symb_noise(C.Structure):
    _fields_ = [("ptr", C.c_void_p), ("rows", C.c_int32), ("reserved", C.c_int32)]


class symb_batch(C.Structure):
    _fields_ = [("d_in", C.c_int32), ("d_out", C.c_int32), ("num_segments", C.c_int32),
                ("seg_offsets", C.POINTER(C.c_int32)), ("adapters", C.POINTER(symb_adapter)),
                ("weight_layout", C.c_int32)]


class symb_norm(C.Structure):
    _fields_ = [("weight", C.c_void_p), ("bias", C.c_void_p), ("dweight", C.c_void_p), ("dbias", C.c_void_p)]


class symb_norm_batch(C.Structure):
    _fields_ = [("width", C.c_int32), ("num_segments", C.c_int32), ("seg_offsets", C.POINTER(C.c_int32)),
                ("norms", C.POINTER(symb_norm)), ("kind", C.c_int32), ("eps", C.c_float), ("weight_base", C.c_float)]


class symb_kv_cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("num_pages", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("page_tokens", C.c_int32)]


class symb_kv_batch(C.Structure):
    _fields_ = [("num_segments", C.c_int32), ("seg_offsets", C.POINTER(C.c_int32)), ("past", C.POINTER(C.c_int32)),
                ("page_table", C.c_void_p), ("table_stride", C.c_int32)]


class symb_rotation(C.Structure):
    _fields_ = [("table", C.c_void_p), ("positions", C.c_int32), ("dim", C.c_int32), ("pairs", C.c_int32)]


class SymbError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__(f"{text} (status {status})")
        self.status = status


_lib = None


def lib() -> C.CDLL:
    """Loads libsymb.so; raises if it has not been built (there is no fallback path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2507_03220_amd.build` "
                               "(or __graft_entry__.build()) first; there is no fallback path")
        l = C.CDLL(LIB_PATH)
        vp, i32, u32, sz = C.c_void_p, C.c_int32, C.c_uint32, C.c_size_t
        bp = C.POINTER(symb_batch)
        l.symb_create.argtypes = [C.POINTER(vp), C.c_int]
        l.symb_destroy.argtypes = [vp]
        l.symb_validate_batch.argtypes = [bp]
        l.symb_debug_row_segment_map.argtypes = [bp, C.POINTER(i32)]
        l.symb_plan_row_tiles.argtypes = [bp, i32, C.POINTER(i32), C.POINTER(i32), C.POINTER(i32)]
        l.symb_workspace_bytes.argtypes = [bp, i32, C.POINTER(sz)]
        l.symb_base_linear_fwd.argtypes = [vp, bp, vp, vp, vp, vp, vp, vp, sz, vp]
        l.symb_base_linear_bwd_input.argtypes = [vp, bp, vp, vp, vp, u32, vp, sz, vp]
        l.symb_adapter_grad.argtypes = [vp, bp, vp, vp, vp, u32, vp, sz, vp]
        l.symb_base_linear_bwd_input_ex.argtypes = [vp, bp, vp, vp, vp, vp, u32, vp, sz, vp]
        l.symb_adapter_grad_ex.argtypes = [vp, bp, vp, vp, vp, vp, u32, vp, sz, vp]
        l.symb_base_linear_fwd_seg.argtypes = [vp, bp, C.POINTER(vp), vp, vp, C.POINTER(vp), vp, sz, vp]
        l.symb_base_linear_bwd_input_seg.argtypes = [vp, bp, C.POINTER(vp), vp, C.POINTER(vp), u32, vp, sz, vp]
        l.symb_adapter_grad_seg.argtypes = [vp, bp, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp), u32, vp, sz, vp]
        l.symb_noise_add.argtypes = [vp, bp, vp, C.POINTER(symb_noise), vp, vp]
        l.symb_base_linear_fwd_denoise.argtypes = [vp, bp, vp, vp, vp, C.POINTER(symb_noise), vp, vp, sz, vp]
        l.symb_debug_gemm_timing_enable.argtypes = [vp, i32]
        l.symb_debug_gemm_timing_read.argtypes = [vp, i32, C.POINTER(C.c_double), C.POINTER(C.c_int64),
                                                  C.POINTER(C.c_double)]
        l.symb_debug_descriptor_stats.argtypes = [vp, C.POINTER(C.c_int64), C.POINTER(C.c_int64)]
        l.symb_debug_set_option.argtypes = [vp, i32, i32]
        l.symb_debug_xcd_rule.argtypes = [vp, C.POINTER(i32), C.POINTER(i32)]
        l.symb_base_linear_fwd_static.argtypes = [vp, bp, vp, vp, vp, vp, vp, vp]
        np_, kp, cp, rp = (C.POINTER(t) for t in (symb_norm_batch, symb_kv_batch, symb_kv_cache, symb_rotation))
        i64 = C.c_int64
        l.symb_norm_workspace_bytes.argtypes = [np_, C.POINTER(sz)]
        l.symb_norm_fwd.argtypes = [vp, np_, vp, vp, vp]
        l.symb_norm_bwd.argtypes = [vp, np_, vp, vp, vp, u32, vp, sz, vp]
        l.symb_kv_append.argtypes = [vp, kp, cp, rp, vp, i64, i32, vp, i64, vp, i64, vp, i64, vp]
        l.symb_kv_workspace_bytes.argtypes = [kp, cp, i32, i32, C.POINTER(sz)]
        l.symb_kv_attention.argtypes = [vp, kp, cp, vp, i64, i32, vp, i64, C.c_float, i32, C.c_float, vp, sz, vp]
        l.symb_status_string.argtypes = [C.c_int]
        l.symb_status_string.restype = C.c_char_p
        l.symb_last_error.argtypes = [vp]
        l.symb_last_error.restype = C.c_char_p
        for name in EXPORTS:
            if name not in ("symb_status_string", "symb_last_error"):
                getattr(l, name).restype = C.c_int
        _lib = l
    return _lib


def _ptr(t) -> Optional[int]:
    """Device (or host) address of a tensor, None for None; ints pass through."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _check(status: int, handle=None) -> None:
    if status != SYMB_OK:
        l = lib()
        msg = l.symb_last_error(handle).decode() or l.symb_status_string(status).decode()
        raise SymbError(status, f"{l.symb_status_string(status).decode()}: {msg}")


@dataclass
class Adapter:
    """One segment's adapter; tensors are torch device tensors (or raw addresses)."""
    kind: int = SYMB_ADAPTER_NONE
    rank: int = 0
    scale: float = 0.0
    A: object = None
    B: object = None
    dA: object = None
    dB: object = None


class Batch:
    """Owns the C arrays of one symb_batch (host offsets + per-segment descriptors)."""

    def __init__(self, d_in: int, d_out: int, seg_offsets: Sequence[int], adapters: Sequence[Adapter],
                 weight_layout: int = 0):
        S = len(adapters)
        if len(seg_offsets) != S + 1:
            raise ValueError("seg_offsets must have num_segments + 1 entries")
        self._off = (C.c_int32 * (S + 1))(*[int(x) for x in seg_offsets])
        self._ad = (symb_adapter * max(S, 1))()
        self._keep = list(adapters)
        for i, a in enumerate(adapters):
            d = self._ad[i]
            d.kind, d.rank, d.scale = int(a.kind), int(a.rank), float(a.scale)
            d.A, d.B, d.dA, d.dB = _ptr(a.A), _ptr(a.B), _ptr(a.dA), _ptr(a.dB)
        self.c = symb_batch(int(d_in), int(d_out), S, self._off, self._ad, int(weight_layout))
        self.d_in, self.d_out, self.S = int(d_in), int(d_out), S
        self.T = int(seg_offsets[-1]) if S >= 0 and len(seg_offsets) else 0

    def ref(self):
        return C.byref(self.c)


def _int32s(values):
    v = [int(x) for x in values]
    return (C.c_int32 * max(len(v), 1))(*v)


@functools.lru_cache(maxsize=None)
def _dtype(name: str):
    import torch
    return getattr(torch, name)


def _dense(t, what: str, dtype: str, dims: int):
    """The tensor as the C ABI takes it, or ValueError: `dims` dense dimensions of that type."""
    if t.dtype is not _dtype(dtype) or t.dim() != dims or not t.is_contiguous():
        raise ValueError(f"{what}: {dims} dense dimensions of {dtype} expected, got {tuple(t.shape)} of {t.dtype}, strides {t.stride()}")
    return t


def _head_rows(t, what: str, shape) -> int:
    """Row stride of a [T][heads][dim] bf16 tensor whose rows may lie apart."""
    apart, head, element = t.stride() if t.dim() == 3 else (0, 0, 0)
    if t.dtype is not _dtype("bfloat16") or t.shape != shape or element != 1 or (head != shape[2] and shape[1] > 1):
        raise ValueError(f"{what}: {list(shape)} of bfloat16 with whole rows expected, got {tuple(t.shape)} of {t.dtype}, strides {t.stride()}")
    return apart if shape[0] > 1 else shape[1] * shape[2]      # (of a single row it says nothing)


@dataclass
class Norm:
    """One segment's norm: bf16 weight and bias, fp32 gradients (device tensors or raw addresses; None as in symb_norm)."""
    weight: object = None
    bias: object = None
    dweight: object = None
    dbias: object = None


class NormBatch:
    """Owns the C arrays of one symb_norm_batch."""

    def __init__(self, width: int, seg_offsets: Sequence[int], norms: Sequence[Norm], kind: int = SYMB_NORM_LAYER, eps: float = 1e-5,
                 weight_base: float = 0.0):
        S = len(norms)
        if len(seg_offsets) != S + 1:
            raise ValueError("seg_offsets must have num_segments + 1 entries")
        self.width, self.S, self.T = int(width), S, int(seg_offsets[-1])
        for i, n in enumerate(norms):
            for what, t, dtype in (("weight", n.weight, "bfloat16"), ("bias", n.bias, "bfloat16"), ("dweight", n.dweight, "float32"), ("dbias", n.dbias, "float32")):
                if t is not None and not isinstance(t, int) and _dense(t, f"{what} of segment {i}", dtype, 1).numel() != self.width:
                    raise ValueError(f"{what} of segment {i} has {t.numel()} elements, the width is {self.width}")
        self._off, self._keep = _int32s(seg_offsets), list(norms)
        self._norms = (symb_norm * max(S, 1))(*[(_ptr(n.weight), _ptr(n.bias), _ptr(n.dweight), _ptr(n.dbias)) for n in norms])
        self.c = symb_norm_batch(self.width, S, self._off, self._norms, int(kind), float(eps), float(weight_base))
        self._ref = C.byref(self.c)

    def ref(self):
        return self._ref


class KvCache:
    """A pool of cache pages: k [pages][kv_heads][page_tokens][head_dim] and v [pages][kv_heads][head_dim][page_tokens] of float8_e4m3fn (or
    uint8), k_scale and v_scale [pages][kv_heads] of float8_e8m0fnu (or uint8), all dense device tensors.  `empty` makes one."""

    def __init__(self, k, v, k_scale, v_scale):
        if k.dim() != 4 or v.dim() != 4 or tuple(v.shape) != (k.shape[0], k.shape[1], k.shape[3], k.shape[2]):
            raise ValueError(f"k {tuple(k.shape)} and v {tuple(v.shape)} are no cache pages")
        for what, t, dims in (("k", k, 4), ("v", v, 4), ("k_scale", k_scale, 2), ("v_scale", v_scale, 2)):
            if t.element_size() != 1 or not t.is_contiguous() or t.dim() != dims or tuple(t.shape[:2]) != tuple(k.shape[:2]):
                raise ValueError(f"{what}: dense 8-bit tensor of {tuple(k.shape[:2])} blocks expected, got {tuple(t.shape)} of {t.dtype}")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.num_pages, self.kv_heads, self.page_tokens, self.head_dim = k.shape
        self.c = symb_kv_cache(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), self.num_pages, self.kv_heads, self.head_dim, self.page_tokens)
        self._ref = C.byref(self.c)

    @classmethod
    def empty(cls, num_pages: int, kv_heads: int, head_dim: int, page_tokens: int = 64, device="cuda"):
        import torch
        make = lambda *shape, dtype: torch.zeros(shape, device=device, dtype=torch.uint8).view(dtype)  # noqa: E731
        return cls(make(num_pages, kv_heads, page_tokens, head_dim, dtype=torch.float8_e4m3fn), make(num_pages, kv_heads, head_dim, page_tokens, dtype=torch.float8_e4m3fn),
                   make(num_pages, kv_heads, dtype=torch.float8_e8m0fnu), make(num_pages, kv_heads, dtype=torch.float8_e8m0fnu))

    def ref(self):
        return self._ref


class KvBatch:
    """Owns the C arrays of one symb_kv_batch; page_table: int32 device tensor [num_segments][pages] (None for host-only calls: `table_stride` then)."""

    def __init__(self, seg_offsets: Sequence[int], past: Sequence[int], page_table, table_stride: int = 0):
        self.S, self.T = len(past), int(seg_offsets[-1])
        if len(seg_offsets) != self.S + 1:
            raise ValueError("seg_offsets must have num_segments + 1 entries")
        if page_table is not None and _dense(page_table, "page_table", "int32", 2).shape[0] != self.S:
            raise ValueError(f"page_table has {page_table.shape[0]} rows for {self.S} segments")
        self._off, self._past, self.page_table = _int32s(seg_offsets), _int32s(past), page_table
        self.c = symb_kv_batch(self.S, self._off, self._past, _ptr(page_table), page_table.shape[1] if page_table is not None else int(table_stride))
        self._ref = C.byref(self.c)

    def ref(self):
        return self._ref


class Rotation:
    """Cosines and sines by position: fp32 device tensor [positions][dim], cosines first."""

    def __init__(self, table, pairs: int = SYMB_ROTATE_HALVES):
        self.table = _dense(table, "table", "float32", 2)
        self.c = symb_rotation(table.data_ptr(), table.shape[0], table.shape[1], int(pairs))
        self._ref = C.byref(self.c)

    def ref(self):
        return self._ref


# ---- entry points, same names as the C ABI ----------------------------------------------------
def symb_create(device: int = 0) -> int:
    h = C.c_void_p()
    _check(lib().symb_create(C.byref(h), int(device)))
    return h.value


def symb_destroy(handle) -> None:
    _check(lib().symb_destroy(handle))


def symb_validate_batch(batch: Batch) -> int:
    return int(lib().symb_validate_batch(batch.ref()))


def symb_debug_row_segment_map(batch: Batch):
    import numpy as np
    out = np.empty(max(batch.T, 0), dtype=np.int32)
    _check(lib().symb_debug_row_segment_map(batch.ref(), out.ctypes.data_as(C.POINTER(C.c_int32))))
    return out


def symb_plan_row_tiles(batch: Batch, tile_m: int):
    import numpy as np
    n = max((batch.T + tile_m - 1) // tile_m, 0) if tile_m > 0 else 0
    lo = np.empty(max(n, 1), dtype=np.int32)
    hi = np.empty(max(n, 1), dtype=np.int32)
    cnt = C.c_int32(0)
    _check(lib().symb_plan_row_tiles(batch.ref(), int(tile_m), lo.ctypes.data_as(C.POINTER(C.c_int32)),
                                     hi.ctypes.data_as(C.POINTER(C.c_int32)), C.byref(cnt)))
    return lo[:cnt.value], hi[:cnt.value]


def symb_workspace_bytes(batch: Batch, op: int) -> int:
    out = C.c_size_t(0)
    _check(lib().symb_workspace_bytes(batch.ref(), int(op), C.byref(out)))
    return int(out.value)


def _ws_args(ws):
    if ws is None:
        return None, 0
    return ws.data_ptr(), ws.numel() * ws.element_size()


def symb_base_linear_fwd(handle, batch: Batch, X, W, bias, Y, Ybase=None, ws=None, stream: int = 0) -> None:
    wp, wb = _ws_args(ws)
    _check(lib().symb_base_linear_fwd(handle, batch.ref(), _ptr(X), _ptr(W), _ptr(bias), _ptr(Y), _ptr(Ybase),
                                      wp, wb, stream or None), handle)


def symb_base_linear_fwd_static(handle, batch: Batch, X, W, bias, Y, Ybase=None, stream: int = 0) -> None:
    _check(lib().symb_base_linear_fwd_static(handle, batch.ref(), _ptr(X), _ptr(W), _ptr(bias), _ptr(Y), _ptr(Ybase),
                                             stream or None), handle)


def _noise_array(batch: Batch, noise: Sequence):
    """noise: per segment None or a tensor [rows][width] (rows 1 = broadcast) or a (ptr, rows) pair."""
    if len(noise) != batch.S:
        raise ValueError("one noise entry per segment")
    arr = (symb_noise * max(batch.S, 1))()
    for i, n in enumerate(noise):
        if n is None:
            continue
        if isinstance(n, tuple):
            arr[i].ptr, arr[i].rows = _ptr(n[0]), int(n[1])
        else:
            arr[i].ptr, arr[i].rows = _ptr(n), int(n.shape[0]) if n.dim() > 1 else 1
    return arr


def _ptr_array(batch: Batch, tensors: Sequence):
    if len(tensors) != batch.S:
        raise ValueError("one buffer per segment")
    return (C.c_void_p * max(batch.S, 1))(*[_ptr(t) for t in tensors])


def symb_base_linear_fwd_seg(handle, batch: Batch, X_seg: Sequence, W, bias, Y_seg: Sequence, ws=None, stream: int = 0) -> None:
    wp, wb = _ws_args(ws)
    _check(lib().symb_base_linear_fwd_seg(handle, batch.ref(), _ptr_array(batch, X_seg), _ptr(W), _ptr(bias),
                                          _ptr_array(batch, Y_seg), wp, wb, stream or None), handle)


def symb_base_linear_bwd_input_seg(handle, batch: Batch, dY_seg: Sequence, W, dX_seg: Sequence, flags: int = SYMB_BWD_FULL,
                                   ws=None, stream: int = 0) -> None:
    wp, wb = _ws_args(ws)
    _check(lib().symb_base_linear_bwd_input_seg(handle, batch.ref(), _ptr_array(batch, dY_seg), _ptr(W),
                                                _ptr_array(batch, dX_seg), int(flags), wp, wb, stream or None), handle)


def symb_adapter_grad_seg(handle, batch: Batch, X_seg: Sequence, dY_seg: Sequence, Ybase_seg=None,
                          flags: int = SYMB_GRAD_OVERWRITE, ws=None, stream: int = 0) -> None:
    wp, wb = _ws_args(ws)
    _check(lib().symb_adapter_grad_seg(handle, batch.ref(), _ptr_array(batch, X_seg), _ptr_array(batch, dY_seg),
                                       None if Ybase_seg is None else _ptr_array(batch, Ybase_seg), int(flags),
                                       wp, wb, stream or None), handle)


def symb_noise_add(handle, batch: Batch, X, noise: Sequence, Xn, stream: int = 0) -> None:
    arr = _noise_array(batch, noise)
    _check(lib().symb_noise_add(handle, batch.ref(), _ptr(X), arr, _ptr(Xn), stream or None), handle)


def symb_base_linear_fwd_denoise(handle, batch: Batch, Xn, W, bias, noise_effect: Sequence, Y, ws=None,
                                 stream: int = 0) -> None:
    wp, wb = _ws_args(ws)
    arr = _noise_array(batch, noise_effect)
    _check(lib().symb_base_linear_fwd_denoise(handle, batch.ref(), _ptr(Xn), _ptr(W), _ptr(bias), arr, _ptr(Y),
                                              wp, wb, stream or None), handle)


def symb_base_linear_bwd_input(handle, batch: Batch, dY, W, dX, flags: int = SYMB_BWD_FULL, ws=None,
                               stream: int = 0) -> None:
    wp, wb = _ws_args(ws)
    _check(lib().symb_base_linear_bwd_input(handle, batch.ref(), _ptr(dY), _ptr(W), _ptr(dX), int(flags),
                                            wp, wb, stream or None), handle)


def symb_base_linear_bwd_input_ex(handle, batch: Batch, dY, W, dX, dXbase=None, flags: int = SYMB_BWD_FULL, ws=None,
                                  stream: int = 0) -> None:
    wp, wb = _ws_args(ws)
    _check(lib().symb_base_linear_bwd_input_ex(handle, batch.ref(), _ptr(dY), _ptr(W), _ptr(dX), _ptr(dXbase),
                                               int(flags), wp, wb, stream or None), handle)


def symb_adapter_grad_ex(handle, batch: Batch, X, dY, Ybase=None, dXbase=None, flags: int = SYMB_GRAD_OVERWRITE,
                         ws=None, stream: int = 0) -> None:
    wp, wb = _ws_args(ws)
    _check(lib().symb_adapter_grad_ex(handle, batch.ref(), _ptr(X), _ptr(dY), _ptr(Ybase), _ptr(dXbase), int(flags),
                                      wp, wb, stream or None), handle)


def symb_adapter_grad(handle, batch: Batch, X, dY, Ybase=None, flags: int = SYMB_GRAD_OVERWRITE, ws=None,
                      stream: int = 0) -> None:
    wp, wb = _ws_args(ws)
    _check(lib().symb_adapter_grad(handle, batch.ref(), _ptr(X), _ptr(dY), _ptr(Ybase), int(flags),
                                   wp, wb, stream or None), handle)


def symb_debug_gemm_timing_enable(handle, on: bool) -> None:
    _check(lib().symb_debug_gemm_timing_enable(handle, 1 if on else 0), handle)


def symb_debug_descriptor_stats(handle):
    """Returns (sent, in_place): calls that sent their descriptors / found them on the device."""
    a, b = C.c_int64(0), C.c_int64(0)
    _check(lib().symb_debug_descriptor_stats(handle, C.byref(a), C.byref(b)), handle)
    return a.value, b.value


def symb_debug_gemm_timing_read(handle, variant: int):
    """Returns (ms_total, launches, flops_total) of the GEMM launches of `variant` since enable."""
    ms, n, fl = C.c_double(0), C.c_int64(0), C.c_double(0)
    _check(lib().symb_debug_gemm_timing_read(handle, int(variant), C.byref(ms), C.byref(n), C.byref(fl)), handle)
    return ms.value, n.value, fl.value


def symb_debug_set_option(handle, option: int, value: int) -> None:
    _check(lib().symb_debug_set_option(handle, int(option), int(value)), handle)


def symb_debug_xcd_rule(handle):
    """Returns (holds, [XCD id seen for workgroup ids 0..7])."""
    ok = C.c_int32(0)
    ids = (C.c_int32 * 8)()
    _check(lib().symb_debug_xcd_rule(handle, C.byref(ok), ids), handle)
    return bool(ok.value), list(ids)


# ---- include/symb_block.h ----------------------------------------------------------------------
def symb_norm_workspace_bytes(batch: NormBatch) -> int:
    out = C.c_size_t(0)
    _check(lib().symb_norm_workspace_bytes(batch.ref(), C.byref(out)))
    return int(out.value)


def _norm_rows(batch: NormBatch, *tensors) -> None:
    bf16, shape = _dtype("bfloat16"), (batch.T, batch.width)
    for t in tensors:
        if t.dtype is not bf16 or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"dense [{batch.T}][{batch.width}] of bfloat16 expected, got {tuple(t.shape)} of {t.dtype}, strides {t.stride()}")


def symb_norm_fwd(handle, batch: NormBatch, X, Y, stream: int = 0) -> None:
    _norm_rows(batch, X, Y)
    _check((_lib or lib()).symb_norm_fwd(handle, batch._ref, X.data_ptr(), Y.data_ptr(), stream or None), handle)


def symb_norm_bwd(handle, batch: NormBatch, X, dY, dX, flags: int = SYMB_GRAD_OVERWRITE, ws=None, stream: int = 0) -> None:
    _norm_rows(batch, X, dY, dX)
    wp, wb = _ws_args(ws)
    _check((_lib or lib()).symb_norm_bwd(handle, batch._ref, X.data_ptr(), dY.data_ptr(), dX.data_ptr(), flags, wp, wb, stream or None), handle)


def symb_kv_append(handle, batch: KvBatch, cache: KvCache, rotation: Optional[Rotation], q, q_out, k, v, stream: int = 0) -> None:
    """q, q_out [T][q_heads][head_dim] (both None: keys and values only), k, v [T][kv_heads][head_dim]; rows may lie apart."""
    shape, heads, q_at, q_apart, out_at, out_apart = (batch.T, cache.kv_heads, cache.head_dim), 0, None, 0, None, 0
    if q is not None:
        heads = q.shape[1]
        q_shape = (batch.T, heads, cache.head_dim)
        q_at, q_apart, out_at, out_apart = q.data_ptr(), _head_rows(q, "q", q_shape), q_out.data_ptr(), _head_rows(q_out, "q_out", q_shape)
    _check((_lib or lib()).symb_kv_append(handle, batch._ref, cache._ref, None if rotation is None else rotation._ref, q_at, q_apart, heads, out_at, out_apart, k.data_ptr(),
                                          _head_rows(k, "k", shape), v.data_ptr(), _head_rows(v, "v", shape), stream or None), handle)


def symb_kv_workspace_bytes(batch: KvBatch, cache: KvCache, q_heads: int, window: int = 0) -> int:
    out = C.c_size_t(0)
    _check(lib().symb_kv_workspace_bytes(batch.ref(), cache.ref(), int(q_heads), int(window), C.byref(out)))
    return int(out.value)


def symb_kv_attention(handle, batch: KvBatch, cache: KvCache, q, out, scale: float, window: int = 0, cap: float = 0.0, ws=None, stream: int = 0) -> None:
    """q, out [T][q_heads][head_dim]; rows may lie apart."""
    heads = q.shape[1]
    shape = (batch.T, heads, cache.head_dim)
    wp, wb = _ws_args(ws)
    _check((_lib or lib()).symb_kv_attention(handle, batch._ref, cache._ref, q.data_ptr(), _head_rows(q, "q", shape), heads, out.data_ptr(), _head_rows(out, "out", shape),
                                             scale, window, cap, wp, wb, stream or None), handle)
