"""Thin ctypes binding of libpixelfly.so (include/pixelfly.h).

Argument marshalling only: every compute step runs in the library's HIP
kernels.  Functions carry the C names; device buffers may be given as torch
tensors (their data_ptr() is passed) or as integer device addresses, streams
as torch.cuda.Stream objects, raw hipStream_t integers or None (the current
torch stream when torch is importable, else the null stream).  A non-zero
status raises PixelflyError with the library's detail message.  There is no
fallback: if libpixelfly.so is missing the import of this module fails.
"""
from __future__ import annotations

import ctypes
import os
import re
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpixelfly.so")
HEADER = os.path.join(os.path.dirname(_HERE), "include", "pixelfly.h")

PF_OK, PF_ERR_INVALID_ARG, PF_ERR_UNSUPPORTED = 0, -1, -2
PF_ERR_WORKSPACE, PF_ERR_HIP, PF_ERR_NOMEM, PF_ERR_STATE = -3, -4, -5, -6
PF_BF16, PF_FP32 = 0, 1
PF_EPI_NONE, PF_EPI_GELU = 0, 1
PF_OP_NT, PF_OP_NN, PF_OP_TN = 0, 1, 2
PF_ACT_NONE, PF_ACT_GELU, PF_ACT_GELU_TANH, PF_ACT_SILU, PF_ACT_RELU = 0, 1, 2, 3, 4
# Kernel classes of the timing hook (pf_kernel_class).
KERNEL_CLASSES = ["spmm_fwd", "spmm_bwd_data", "sddmm", "lowrank_t", "lowrank_s", "reduce",
                  "gelu_bwd", "attn_fwd", "attn_bwd_dq", "attn_bwd_dkv", "dense", "butterfly"]
PF_KERNEL_COUNT = len(KERNEL_CLASSES)


class PixelflyError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"pixelfly status {status}: {msg}")
        self.status = status


# Load torch's HIP runtime first when torch is present: libpixelfly.so then
# binds to that same runtime (matched by SONAME) instead of bringing a second
# HIP/HSA runtime into the process, so torch tensors and streams are valid
# for the library.
try:
    import torch
except ImportError:
    torch = None

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} not built; run `python -m paper_2112_00029_amd.build` "
        "(or __graft_entry__.build())")
_lib = ctypes.CDLL(LIB_PATH)

_p = ctypes.c_void_p
_i32, _i64, _f32, _sz = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t


class pf_layout_info(ctypes.Structure):
    _fields_ = [("n_out", _i64), ("n_in", _i64), ("b", _i32), ("max_stride", _i32),
                ("eff_stride", _i32), ("s", _i32), ("nb_out", _i32), ("nb_in", _i32),
                ("nnzb", _i64), ("row_ptr", ctypes.POINTER(_i32)),
                ("col_idx", ctypes.POINTER(_i32)), ("col_ptr", ctypes.POINTER(_i32)),
                ("row_idx", ctypes.POINTER(_i32)), ("tperm", ctypes.POINTER(_i32))]


class pf_linear_plan(ctypes.Structure):
    _fields_ = [(n, _i32) for n in (
        "lowrank_t_kernel", "lowrank_t_split", "lowrank_t_tile_m", "lowrank_t_tile_n",
        "lowrank_s_kernel", "lowrank_s_split", "lowrank_s_tile_m", "lowrank_s_tile_n",
        "fwd_tile_m", "fwd_tile_n", "fwd_direct_lds", "bwd_tile_m", "bwd_tile_n",
        "bwd_direct_lds", "tn_items", "tn_split")] + [("tn_chunk", _i64),
                                                       ("workspace_bytes", ctypes.c_uint64),
                                                       ("tn_tile", _i32), ("tn_shared", _i32)]


class pf_linear_gated_plan(ctypes.Structure):
    _fields_ = [(n, _i32) for n in ("kernel", "tile_m", "tile_n", "k_step", "waves")]


_rows_p = _p  # const pf_attn_tensor *

_SIGS = {
    "pf_layout_create": (_i32, [_i64, _i64, _i32, _i32, ctypes.POINTER(_p)]),
    "pf_layout_create_from_mask": (_i32, [_i32, _i32, _i32, _p, ctypes.POINTER(_p)]),
    "pf_layout_create_attention": (_i32, [_i64, _i32, _i32, _i32, ctypes.POINTER(_p)]),
    "pf_layout_create_from_element_mask": (_i32, [_i64, _i64, _i32, _p, ctypes.POINTER(_p)]),
    "pf_layout_create_factor": (_i32, [_i64, _i32, _i32, ctypes.POINTER(_p)]),
    "pf_layout_create_butterfly": (_i32, [_i64, _i32, _i32, ctypes.POINTER(_p)]),
    "pf_butterfly_fwd": (_i32, [_p, _i64, _p, _p, _p, _p, _p]),
    "pf_butterfly_bwd_data": (_i32, [_p, _i64, _p, _p, _p, _p, _p]),
    "pf_select_mask": (_i32, [_i64, _i64, _i32, ctypes.c_double, ctypes.c_double,
                              ctypes.POINTER(_i32), ctypes.POINTER(_i32), ctypes.POINTER(_i64)]),
    "pf_layout_info_get": (_i32, [_p, ctypes.POINTER(pf_layout_info)]),
    "pf_layout_check": (_i32, [_p]),
    "pf_layout_plan_get": (_i32, [_p, ctypes.POINTER(_i32), _i32]),
    "pf_linear_plan_get": (_i32, [_p, _i32, _i64, _i32, ctypes.POINTER(pf_linear_plan)]),
    "pf_linear_gated_plan_get": (_i32, [_p, _i32, _i64, _i32, ctypes.POINTER(pf_linear_gated_plan)]),
    "pf_layout_upload": (_i32, [_p, _p]),
    "pf_layout_destroy": (None, [_p]),
    "pf_workspace_bytes": (_sz, [_p, _i64, _i32, _i32]),
    "pf_linear_fwd": (_i32, [_p, _i32, _i64, _i32, _p, _p, _p, _p, _p, _p, _i32, _p, _p, _sz, _p]),
    "pf_linear_bwd_data": (_i32, [_p, _i32, _i64, _i32, _p, _p, _p, _p, _p, _p, _i32, _p, _p, _sz,
                                  _p]),
    "pf_linear_bwd_weight": (_i32, [_p, _i32, _i64, _i32, _p, _p, _p, _p, _p, _p, _p, _p, _sz, _p]),
    "pf_linear_fwd_mixed": (_i32, [_p, _i32, _i64, _i32, _f32, _p, _p, _p, _p, _p, _p, _i32, _p, _p,
                                   _sz, _p]),
    "pf_linear_bwd_data_mixed": (_i32, [_p, _i32, _i64, _i32, _f32, _p, _p, _p, _p, _p, _p, _i32,
                                        _p, _p, _sz, _p]),
    "pf_linear_bwd_weight_mixed": (_i32, [_p, _i32, _i64, _i32, _f32, _p, _p, _p, _p, _p, _p, _p,
                                          _p, _p, _p, _sz, _p]),
    "pf_linear_fwd_act": (_i32, [_p, _i32, _i64, _i32, _p, _p, _p, _p, _p, _i32, _p, _p, _p, _p, _p,
                                 _sz, _p]),
    "pf_linear_fwd_act_mixed": (_i32, [_p, _i32, _i64, _i32, _f32, _p, _p, _p, _p, _p, _i32, _p, _p,
                                       _p, _p, _p, _sz, _p]),
    "pf_linear_act_bwd": (_i32, [_i32, _i64, _i64, _i32, _p, _p, _p, _p, _p, _sz, _p]),
    "pf_linear_act_workspace_bytes": (_sz, [_i32, _i64, _i64]),
    "pf_gelu_bwd": (_i32, [_i32, _i64, _p, _p, _p, _p]),
    "pf_layout_create_gated": (_i32, [_i64, _i64, _i32, _i32, ctypes.POINTER(_p)]),
    "pf_layout_create_gated_from_mask": (_i32, [_i32, _i32, _i32, _p, ctypes.POINTER(_p)]),
    "pf_linear_gated_fwd": (_i32, [_p, _i32, _i64, _i32, _p, _p, _p, _p, _p, _i32, _p, _p, _p, _p, _sz,
                                   _p]),
    "pf_linear_gated_fwd_mixed": (_i32, [_p, _i32, _i64, _i32, _f32, _p, _p, _p, _p, _p, _i32, _p, _p,
                                         _p, _p, _sz, _p]),
    "pf_linear_gated_bwd": (_i32, [_i32, _i64, _i64, _i32, _i32, _p, _p, _p, _p, _p, _sz, _p]),
    "pf_linear_gated_workspace_bytes": (_sz, [_i32, _i64, _i64]),
    "pf_layernorm_fwd": (_i32, [_i32, _i64, _i64, _f32, _p, _i64, _p, _p, _p, _i64, _p, _p, _p]),
    "pf_layernorm_bwd": (_i32, [_i32, _i64, _i64, _p, _i64, _p, _i64, _p, _p, _p, _p, _i64, _p, _i64,
                                _p, _p, _p, _sz, _p]),
    "pf_layernorm_workspace_bytes": (_sz, [_i32, _i64, _i64]),
    "pf_grads_create": (_i32, [_i32, _p, ctypes.POINTER(_p)]),
    "pf_grads_upload": (_i32, [_p, _p]),
    "pf_grads_destroy": (None, [_p]),
    "pf_grads_workspace_bytes": (_sz, [_p]),
    "pf_grads_clip": (_i32, [_p, _f32, _p, _p, _sz, _p]),
    "pf_grads_norm": (_i32, [_p, _p, _p, _p, _sz, _p]),
    "pf_grads_scale": (_i32, [_p, _f32, _p, _p]),
    "pf_attn_fwd": (_i32, [_p, _i32, _i32, _i32, _i32, _f32, _p, _p, _p, _p, _p, _p]),
    "pf_attn_bwd": (_i32, [_p, _i32, _i32, _i32, _i32, _f32, _p, _p, _p, _p, _p, _p, _p, _p,
                           _p, _p, _sz, _p]),
    "pf_attn_workspace_bytes": (_sz, [_i32, _i32, _i32]),
    "pf_attn_bwd_noalloc": (_i32, [_p, _i32, _i32, _i32, _i32, _f32, _p, _p, _p, _p, _p, _p, _p,
                                   _p, _p, _p]),
    "pf_relpos_create": (_i32, [_i64, _i32, _p, ctypes.POINTER(_p)]),
    "pf_relpos_create_log": (_i32, [_i64, _i32, _i64, _i32, ctypes.POINTER(_p)]),
    "pf_relpos_buckets_get": (_i32, [_p, ctypes.POINTER(ctypes.POINTER(_i32)), ctypes.POINTER(_i64),
                                     ctypes.POINTER(_i32)]),
    "pf_relpos_upload": (_i32, [_p, _p]),
    "pf_relpos_destroy": (None, [_p]),
    "pf_relpos_bias_floats": (_sz, [_p]),
    "pf_relpos_bias": (_i32, [_p, _i32, _p, _p, _p]),
    "pf_attn_relpos_fwd": (_i32, [_p, _p, _i32, _i32, _i32, _i32, _i32, _i32, _f32, _rows_p, _rows_p,
                                  _rows_p, _p, _rows_p, _p, _p, _p, _p, _sz, _p]),
    "pf_attn_relpos_bwd": (_i32, [_p, _p, _i32, _i32, _i32, _i32, _i32, _f32, _rows_p, _rows_p,
                                  _rows_p, _p, _rows_p, _p, _rows_p, _rows_p, _rows_p, _rows_p, _p, _p,
                                  _p, _sz, _p]),
    "pf_attn_relpos_workspace_bytes": (_sz, [_p, _p, _i32, _i32, _i32]),
    "pf_dense_gemm": (_i32, [_i32, _i32, _i64, _i64, _i64, _p, _p, _p, _p, _sz, _p]),
    "pf_dense_workspace_bytes": (_sz, [_i32, _i32, _i64, _i64, _i64]),
    "pf_timing_begin": (_i32, [_i32]),
    "pf_timing_end": (_i32, [ctypes.POINTER(_i32), ctypes.POINTER(ctypes.c_double)]),
    "pf_status_string": (ctypes.c_char_p, [_i32]),
    "pf_last_error": (ctypes.c_char_p, []),
}
for _name, (_res, _args) in _SIGS.items():
    _f = getattr(_lib, _name)
    _f.restype = _res
    _f.argtypes = _args


def header_functions() -> list[str]:
    """Names of the functions include/pixelfly.h declares."""
    text = open(HEADER).read()
    return sorted(set(re.findall(r"^[a-z_ ]*?\*?\s*(pf_[a-z0-9_]+)\s*\(", text, re.M)))


def _ptr(x):
    if x is None or type(x) is int:
        return x
    try:
        return x.data_ptr()
    except AttributeError:
        if isinstance(x, int):
            return x
    raise TypeError(f"expected a tensor, int address or None, got {type(x)}")


# The current stream's handle without building a torch.cuda.Stream object (a
# call of the smallest products waits for the host: 3.7 -> 0.4 us of 9.1 / 5.7 us
# for an attention forward of one block).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) if torch else None
# The same of an initialised runtime's current device (torch.cuda.current_device
# initialises it first).
_raw_device = getattr(torch._C, "_cuda_getDevice", None) if torch else None


def _current_device() -> int:
    return _raw_device() if _raw_device is not None else torch.cuda.current_device()


def _stream(s):
    if s is None:
        # An initialised runtime implies an available one.
        if torch is None or not torch.cuda.is_initialized():
            return None
        if _raw_stream is not None:
            return _raw_stream(_current_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(s, int):
        return s
    return s.cuda_stream


def _check(st: int):
    if st != PF_OK:
        raise PixelflyError(st, _lib.pf_last_error().decode())


_DTYPES = {"bf16": PF_BF16, "fp32": PF_FP32}


def _dt(dtype) -> int:
    if isinstance(dtype, int):
        return dtype  # validated by the library
    if isinstance(dtype, str) and dtype in _DTYPES:
        return _DTYPES[dtype]
    name = str(dtype)
    if "bfloat16" in name or name == "bf16":
        return PF_BF16
    if "float32" in name or name == "fp32":
        return PF_FP32
    raise ValueError(f"unsupported dtype {dtype}")


class Layout:
    """Owner of a pf_layout* (destroyed with the object)."""

    def __init__(self, handle: int):
        self.handle = handle

    @property
    def _as_parameter_(self):
        return self.handle

    def __del__(self):
        h, self.handle = getattr(self, "handle", None), None
        if h and _lib is not None:
            _lib.pf_layout_destroy(h)


def pf_layout_create(n_out: int, n_in: int, b: int, max_stride: int) -> Layout:
    h = _p()
    _check(_lib.pf_layout_create(n_out, n_in, b, max_stride, ctypes.byref(h)))
    return Layout(h.value)


def pf_layout_create_from_mask(nb_out: int, nb_in: int, b: int, block_mask) -> Layout:
    """block_mask: (nb_out, nb_in) array-like, nonzero = kept block."""
    m = np.ascontiguousarray(np.asarray(block_mask).astype(bool).astype(np.uint8))
    if m.shape != (nb_out, nb_in):
        raise ValueError(f"block_mask shape {m.shape} != ({nb_out}, {nb_in})")
    h = _p()
    _check(_lib.pf_layout_create_from_mask(nb_out, nb_in, b, m.ctypes.data_as(_p), ctypes.byref(h)))
    return Layout(h.value)


def pf_layout_create_attention(seq: int, b: int, max_stride: int, global_blocks: int = 0) -> Layout:
    h = _p()
    _check(_lib.pf_layout_create_attention(seq, b, max_stride, global_blocks, ctypes.byref(h)))
    return Layout(h.value)


def pf_layout_create_from_element_mask(n_out: int, n_in: int, b: int, elem_mask) -> Layout:
    """elem_mask: (n_out, n_in) array-like, nonzero = kept element; the layout
    is its (b, b)-block cover."""
    m = np.ascontiguousarray(np.asarray(elem_mask).astype(bool).astype(np.uint8))
    if m.shape != (n_out, n_in):
        raise ValueError(f"elem_mask shape {m.shape} != ({n_out}, {n_in})")
    h = _p()
    _check(_lib.pf_layout_create_from_element_mask(n_out, n_in, b, m.ctypes.data_as(_p),
                                                   ctypes.byref(h)))
    return Layout(h.value)


def pf_layout_create_factor(n: int, b: int, k: int) -> Layout:
    h = _p()
    _check(_lib.pf_layout_create_factor(n, b, k, ctypes.byref(h)))
    return Layout(h.value)


def pf_layout_create_gated(n_out: int, n_in: int, b: int, max_stride: int) -> Layout:
    """Two n_out x n_in projections as one matrix of 2 n_out rows in blocks of b
    that alternate gate, other factor."""
    h = _p()
    _check(_lib.pf_layout_create_gated(n_out, n_in, b, max_stride, ctypes.byref(h)))
    return Layout(h.value)


def pf_layout_create_gated_from_mask(nb_out: int, nb_in: int, b: int, block_mask) -> Layout:
    m = np.ascontiguousarray(np.asarray(block_mask) != 0, dtype=np.uint8)
    if m.shape != (nb_out, nb_in):
        raise ValueError(f"mask shape {m.shape} != ({nb_out}, {nb_in})")
    h = _p()
    _check(_lib.pf_layout_create_gated_from_mask(nb_out, nb_in, b, m.ctypes.data_as(_p), ctypes.byref(h)))
    return Layout(h.value)


def pf_layout_create_butterfly(n: int, b: int, max_stride: int) -> Layout:
    h = _p()
    _check(_lib.pf_layout_create_butterfly(n, b, max_stride, ctypes.byref(h)))
    return Layout(h.value)


def pf_butterfly_fwd(layout, T, X, F, Y, acts=None, stream=None) -> None:
    _check(_lib.pf_butterfly_fwd(layout.handle, T, _ptr(X), _ptr(F), _ptr(Y), _ptr(acts),
                                 _stream(stream)))


def pf_butterfly_bwd_data(layout, T, dY, F, dX, grads=None, stream=None) -> None:
    _check(_lib.pf_butterfly_bwd_data(layout.handle, T, _ptr(dY), _ptr(F), _ptr(dX),
                                      _ptr(grads), _stream(stream)))


def pf_select_mask(n_out: int, n_in: int, b: int, budget: float, lowrank_share: float = 0.25) -> dict:
    """Rank and maximum stride for a layer from a compute budget; returns
    dict(r=..., max_stride=..., params=...)."""
    r, ms, pr = _i32(), _i32(), _i64()
    _check(_lib.pf_select_mask(n_out, n_in, b, budget, lowrank_share, ctypes.byref(r),
                               ctypes.byref(ms), ctypes.byref(pr)))
    return dict(r=r.value, max_stride=ms.value, params=pr.value)


def pf_layout_info_get(layout: Layout) -> dict:
    """Layout metadata; index arrays are copied into numpy int32 arrays."""
    info = pf_layout_info()
    _check(_lib.pf_layout_info_get(layout.handle, ctypes.byref(info)))
    arr = lambda p, n: np.ctypeslib.as_array(p, shape=(n,)).copy() if n else np.zeros(0, np.int32)
    return {
        "n_out": info.n_out, "n_in": info.n_in, "b": info.b, "max_stride": info.max_stride,
        "eff_stride": info.eff_stride, "s": info.s, "nb_out": info.nb_out, "nb_in": info.nb_in,
        "nnzb": info.nnzb,
        "row_ptr": arr(info.row_ptr, info.nb_out + 1), "col_idx": arr(info.col_idx, info.nnzb),
        "col_ptr": arr(info.col_ptr, info.nb_in + 1), "row_idx": arr(info.row_idx, info.nnzb),
        "tperm": arr(info.tperm, info.nnzb),
    }


def pf_layout_check(layout: Layout) -> None:
    _check(_lib.pf_layout_check(layout.handle))


def pf_layout_plan_get(layout: Layout) -> dict:
    st = (_i32 * 10)()
    _check(_lib.pf_layout_plan_get(layout.handle, st, 10))
    keys = ["G_fwd", "fwd_tiles", "G_bwd", "bwd_tiles", "tn_items", "tn_kept",
            "G_fwd_wide", "fwd_tiles_wide", "G_bwd_wide", "bwd_tiles_wide"]
    return dict(zip(keys, list(st)))


def pf_linear_plan_get(layout: Layout, dtype, T: int, r: int) -> dict:
    """The kernels and splits a linear step of T tokens at rank r runs."""
    p = pf_linear_plan()
    _check(_lib.pf_linear_plan_get(layout.handle, _dt(dtype), T, r, ctypes.byref(p)))
    return {n: getattr(p, n) for n, _t in pf_linear_plan._fields_}


def pf_linear_gated_plan_get(layout: Layout, dtype, T: int, r: int) -> dict:
    """The kernel pf_linear_gated_fwd runs for T tokens at rank r."""
    p = pf_linear_gated_plan()
    _check(_lib.pf_linear_gated_plan_get(layout.handle, _dt(dtype), T, r, ctypes.byref(p)))
    return {n: getattr(p, n) for n, _t in pf_linear_gated_plan._fields_}


def pf_layout_upload(layout: Layout, stream=None) -> None:
    _check(_lib.pf_layout_upload(layout.handle, _stream(stream)))


def pf_layout_destroy(layout: Layout) -> None:
    h, layout.handle = layout.handle, None
    if h:
        _lib.pf_layout_destroy(h)


def pf_workspace_bytes(layout: Layout, T: int, r: int, dtype) -> int:
    return int(_lib.pf_workspace_bytes(layout.handle, T, r, _dt(dtype)))


def pf_linear_fwd(layout, dtype, T, r, X, Wblk, U, V, Y, T_lr, epi=PF_EPI_NONE,
                  Y_pre=None, workspace=None, ws_bytes=0, stream=None) -> None:
    _check(_lib.pf_linear_fwd(layout.handle, _dt(dtype), T, r, _ptr(X), _ptr(Wblk), _ptr(U),
                              _ptr(V), _ptr(Y), _ptr(T_lr), epi, _ptr(Y_pre), _ptr(workspace),
                              ws_bytes, _stream(stream)))


def pf_linear_bwd_data(layout, dtype, T, r, dY, Wblk, U, V, S, dX, epi=PF_EPI_NONE,
                       aux=None, workspace=None, ws_bytes=0, stream=None) -> None:
    _check(_lib.pf_linear_bwd_data(layout.handle, _dt(dtype), T, r, _ptr(dY), _ptr(Wblk),
                                   _ptr(U), _ptr(V), _ptr(S), _ptr(dX), epi, _ptr(aux),
                                   _ptr(workspace), ws_bytes, _stream(stream)))


def pf_linear_bwd_weight(layout, dtype, T, r, dY, X, T_lr, S, dWblk, dU, dV, workspace,
                         ws_bytes, stream=None) -> None:
    _check(_lib.pf_linear_bwd_weight(layout.handle, _dt(dtype), T, r, _ptr(dY), _ptr(X),
                                     _ptr(T_lr), _ptr(S), _ptr(dWblk), _ptr(dU), _ptr(dV),
                                     _ptr(workspace), ws_bytes, _stream(stream)))


def pf_linear_fwd_mixed(layout, dtype, T, r, gamma, X, Wblk, U, V, Y, T_lr, epi=PF_EPI_NONE,
                        Y_pre=None, workspace=None, ws_bytes=0, stream=None) -> None:
    _check(_lib.pf_linear_fwd_mixed(layout.handle, _dt(dtype), T, r, float(gamma), _ptr(X),
                                    _ptr(Wblk), _ptr(U), _ptr(V), _ptr(Y), _ptr(T_lr), epi,
                                    _ptr(Y_pre), _ptr(workspace), ws_bytes, _stream(stream)))


def pf_linear_bwd_data_mixed(layout, dtype, T, r, gamma, dY, Wblk, U, V, S, dX, epi=PF_EPI_NONE,
                             aux=None, workspace=None, ws_bytes=0, stream=None) -> None:
    _check(_lib.pf_linear_bwd_data_mixed(layout.handle, _dt(dtype), T, r, float(gamma), _ptr(dY),
                                         _ptr(Wblk), _ptr(U), _ptr(V), _ptr(S), _ptr(dX), epi,
                                         _ptr(aux), _ptr(workspace), ws_bytes, _stream(stream)))


def pf_linear_bwd_weight_mixed(layout, dtype, T, r, gamma, dY, X, Wblk, T_lr, S, dWblk, dU, dV,
                               dgamma, workspace, ws_bytes, stream=None) -> None:
    """dgamma: device buffer of one float32."""
    _check(_lib.pf_linear_bwd_weight_mixed(layout.handle, _dt(dtype), T, r, float(gamma),
                                           _ptr(dY), _ptr(X), _ptr(Wblk), _ptr(T_lr), _ptr(S),
                                           _ptr(dWblk), _ptr(dU), _ptr(dV), _ptr(dgamma),
                                           _ptr(workspace), ws_bytes, _stream(stream)))


def pf_linear_fwd_act(layout, dtype, T, r, X, Wblk, U, V, bias, act, residual, Y, Y_pre, T_lr,
                      workspace=None, ws_bytes=0, stream=None) -> None:
    """act: PF_ACT_*; bias, residual and Y_pre may be None."""
    _check(_lib.pf_linear_fwd_act(layout.handle, _dt(dtype), T, r, _ptr(X), _ptr(Wblk), _ptr(U),
                                  _ptr(V), _ptr(bias), act, _ptr(residual), _ptr(Y), _ptr(Y_pre),
                                  _ptr(T_lr), _ptr(workspace), ws_bytes, _stream(stream)))


def pf_linear_fwd_act_mixed(layout, dtype, T, r, gamma, X, Wblk, U, V, bias, act, residual, Y, Y_pre,
                            T_lr, workspace=None, ws_bytes=0, stream=None) -> None:
    _check(_lib.pf_linear_fwd_act_mixed(layout.handle, _dt(dtype), T, r, float(gamma), _ptr(X),
                                        _ptr(Wblk), _ptr(U), _ptr(V), _ptr(bias), act,
                                        _ptr(residual), _ptr(Y), _ptr(Y_pre), _ptr(T_lr),
                                        _ptr(workspace), ws_bytes, _stream(stream)))


def pf_linear_act_bwd(dtype, T, N, act, dY, Y_pre, dY_pre, dbias, workspace=None, ws_bytes=0,
                      stream=None) -> None:
    _check(_lib.pf_linear_act_bwd(_dt(dtype), T, N, act, _ptr(dY), _ptr(Y_pre), _ptr(dY_pre),
                                  _ptr(dbias), _ptr(workspace), ws_bytes, _stream(stream)))


def pf_linear_act_workspace_bytes(dtype, T, N) -> int:
    return int(_lib.pf_linear_act_workspace_bytes(_dt(dtype), T, N))


def pf_linear_gated_fwd(layout, dtype, T, r, X, Wblk, U, V, bias, act, H, Z, T_lr, workspace=None,
                        ws_bytes=0, stream=None) -> None:
    """act: PF_ACT_*; bias and Z may be None."""
    _check(_lib.pf_linear_gated_fwd(layout.handle, _dt(dtype), T, r, _ptr(X), _ptr(Wblk), _ptr(U), _ptr(V),
                                    _ptr(bias), act, _ptr(H), _ptr(Z), _ptr(T_lr), _ptr(workspace), ws_bytes,
                                    _stream(stream)))


def pf_linear_gated_fwd_mixed(layout, dtype, T, r, gamma, X, Wblk, U, V, bias, act, H, Z, T_lr,
                              workspace=None, ws_bytes=0, stream=None) -> None:
    _check(_lib.pf_linear_gated_fwd_mixed(layout.handle, _dt(dtype), T, r, float(gamma), _ptr(X), _ptr(Wblk),
                                          _ptr(U), _ptr(V), _ptr(bias), act, _ptr(H), _ptr(Z), _ptr(T_lr),
                                          _ptr(workspace), ws_bytes, _stream(stream)))


def pf_linear_gated_bwd(dtype, T, N, b, act, dH, Z, dZ, dbias, workspace=None, ws_bytes=0,
                        stream=None) -> None:
    _check(_lib.pf_linear_gated_bwd(_dt(dtype), T, N, b, act, _ptr(dH), _ptr(Z), _ptr(dZ), _ptr(dbias),
                                    _ptr(workspace), ws_bytes, _stream(stream)))


def pf_linear_gated_workspace_bytes(dtype, T, N) -> int:
    return int(_lib.pf_linear_gated_workspace_bytes(_dt(dtype), T, N))


def pf_layernorm_fwd(dtype, T, N, eps, X, ldx, weight, bias, Y, ldy, mean=None, rstd=None,
                     stream=None) -> None:
    """Row strides ldx, ldy in elements; weight, bias, mean and rstd may be None."""
    _check(_lib.pf_layernorm_fwd(_dt(dtype), T, N, eps, _ptr(X), ldx, _ptr(weight), _ptr(bias), _ptr(Y), ldy,
                                 _ptr(mean), _ptr(rstd), _stream(stream)))


def pf_layernorm_bwd(dtype, T, N, dY, lddy, X, ldx, weight, mean, rstd, dR, lddr, dX, lddx, dweight, dbias,
                     workspace=None, ws_bytes=0, stream=None) -> None:
    """dR: a gradient to add to dX, or None."""
    _check(_lib.pf_layernorm_bwd(_dt(dtype), T, N, _ptr(dY), lddy, _ptr(X), ldx, _ptr(weight), _ptr(mean),
                                 _ptr(rstd), _ptr(dR), lddr, _ptr(dX), lddx, _ptr(dweight), _ptr(dbias),
                                 _ptr(workspace), ws_bytes, _stream(stream)))


def pf_layernorm_workspace_bytes(dtype, T, N) -> int:
    return int(_lib.pf_layernorm_workspace_bytes(_dt(dtype), T, N))


class Grads:
    """Owner of a pf_grads* (destroyed with the object) and holder of the tensors
    it names."""

    def __init__(self, handle: int, tensors):
        self.handle = handle
        self.tensors = tensors

    def __del__(self):
        h, self.handle = getattr(self, "handle", None), None
        if h and _lib is not None:
            _lib.pf_grads_destroy(h)


# pf_grad_tensor.
_pack_grad = struct.Struct("PPqii").pack


def pf_grads_create(tensors) -> Grads:
    """tensors: gradients (scaled in place), or pairs (gradient, where its scaled
    values go); contiguous float32 or bfloat16 tensors of one device."""
    rows, keep = [], []
    for i, t in enumerate(tensors):
        src, dst = t if isinstance(t, (tuple, list)) else (t, t)
        for x in (src, dst):
            if x.dtype not in (torch.float32, torch.bfloat16) or not x.is_contiguous():
                raise ValueError(f"gradient {i}: expected a contiguous float32 or bfloat16 tensor, got {x.dtype}"
                                 f"{'' if x.is_contiguous() else ' with strides'}")
            if keep and x.device != keep[0][0].device or x.device != src.device:
                raise ValueError(f"gradient {i}: on {x.device}, the first on {(keep[0][0] if keep else src).device}")
        if src.numel() != dst.numel():
            raise ValueError(f"gradient {i}: {src.numel()} elements into {dst.numel()}")
        keep.append((src, dst))
        rows.append(_pack_grad(src.data_ptr(), dst.data_ptr(), src.numel(), _dt(src.dtype), _dt(dst.dtype)))
    h = _p()
    _check(_lib.pf_grads_create(len(rows), b"".join(rows) or None, ctypes.byref(h)))
    return Grads(h.value, keep)


def pf_grads_upload(grads, stream=None) -> None:
    dev = grads.tensors[0][0].device if grads.tensors else None
    if dev is not None and (dev.type != "cuda" or dev.index != _current_device()):
        raise ValueError(f"gradients are on {dev}, not on the GPU in use")
    _check(_lib.pf_grads_upload(grads.handle, _stream(stream)))


def pf_grads_destroy(grads) -> None:
    h, grads.handle = grads.handle, None
    if h:
        _lib.pf_grads_destroy(h)


def pf_grads_workspace_bytes(grads) -> int:
    return int(_lib.pf_grads_workspace_bytes(grads.handle))


def pf_grads_clip(grads, max_norm, norm=None, workspace=None, ws_bytes=0, stream=None) -> None:
    """norm: one float32 on the device, or None."""
    _check(_lib.pf_grads_clip(grads.handle, max_norm, _ptr(norm), _ptr(workspace), ws_bytes, _stream(stream)))


def pf_grads_norm(grads, sumsq, norm, workspace=None, ws_bytes=0, stream=None) -> None:
    """sumsq: one float64 on the device; it or norm may be None."""
    _check(_lib.pf_grads_norm(grads.handle, _ptr(sumsq), _ptr(norm), _ptr(workspace), ws_bytes,
                              _stream(stream)))


def pf_grads_scale(grads, max_norm, sumsq, stream=None) -> None:
    _check(_lib.pf_grads_scale(grads.handle, max_norm, _ptr(sumsq), _stream(stream)))


def pf_gelu_bwd(dtype, n, dH, H_pre, dH_pre, stream=None) -> None:
    _check(_lib.pf_gelu_bwd(_dt(dtype), n, _ptr(dH), _ptr(H_pre), _ptr(dH_pre), _stream(stream)))


def pf_attn_fwd(layout, B, H, S, d, scale, Q, K, V, O, lse, stream=None) -> None:
    _check(_lib.pf_attn_fwd(layout.handle, B, H, S, d, scale, _ptr(Q), _ptr(K), _ptr(V),
                            _ptr(O), _ptr(lse), _stream(stream)))


def pf_attn_bwd(layout, B, H, S, d, scale, Q, K, V, O, lse, dO, dQ, dK, dV, workspace,
                ws_bytes, stream=None) -> None:
    _check(_lib.pf_attn_bwd(layout.handle, B, H, S, d, scale, _ptr(Q), _ptr(K), _ptr(V),
                            _ptr(O), _ptr(lse), _ptr(dO), _ptr(dQ), _ptr(dK), _ptr(dV),
                            _ptr(workspace), ws_bytes, _stream(stream)))


def pf_attn_bwd_noalloc(layout, B, H, S, d, scale, Q, K, V, O, lse, dO, dQ, dK, dV,
                        stream=None) -> None:
    _check(_lib.pf_attn_bwd_noalloc(layout.handle, B, H, S, d, scale, _ptr(Q), _ptr(K), _ptr(V),
                                    _ptr(O), _ptr(lse), _ptr(dO), _ptr(dQ), _ptr(dK), _ptr(dV),
                                    _stream(stream)))


def pf_attn_workspace_bytes(B, H, S) -> int:
    return int(_lib.pf_attn_workspace_bytes(B, H, S))


class Relpos:
    """Owner of a pf_relpos* (destroyed with the object)."""

    def __init__(self, handle: int, n_buckets: int):
        self.handle, self.n_buckets = handle, n_buckets
        self.bias_floats = int(_lib.pf_relpos_bias_floats(handle))  # per head

    def __del__(self):
        h, self.handle = getattr(self, "handle", None), None
        if h and _lib is not None:
            _lib.pf_relpos_destroy(h)


def pf_relpos_create(seq: int, n_buckets: int, bucket) -> Relpos:
    """bucket: 2 seq - 1 integers, the bucket of key - query = -(seq - 1) ..
    seq - 1 (-1: not attended)."""
    b = np.asarray(bucket)
    m = np.ascontiguousarray(b, dtype=np.int32) if b.dtype.kind in "biu" else None
    if m is None or not np.array_equal(m, b):
        raise ValueError(f"bucket: expected integers of 32 bits, got {b.dtype}")
    if m.shape != (max(2 * seq - 1, 0),):
        raise ValueError(f"bucket shape {m.shape} != ({2 * seq - 1},)")
    h = _p()
    _check(_lib.pf_relpos_create(seq, n_buckets, m.ctypes.data_as(_p), ctypes.byref(h)))
    return Relpos(h.value, n_buckets)


def pf_relpos_create_log(seq: int, n_buckets: int, max_distance: int, bidirectional: bool) -> Relpos:
    h = _p()
    _check(_lib.pf_relpos_create_log(seq, n_buckets, max_distance, int(bool(bidirectional)),
                                     ctypes.byref(h)))
    return Relpos(h.value, n_buckets)


def pf_relpos_buckets_get(relpos: Relpos) -> tuple:
    """(bucket map as pf_relpos_create takes it, n_buckets); a copy."""
    b, seq, n = ctypes.POINTER(_i32)(), _i64(), _i32()
    _check(_lib.pf_relpos_buckets_get(relpos.handle, ctypes.byref(b), ctypes.byref(seq), ctypes.byref(n)))
    return np.ctypeslib.as_array(b, shape=(2 * seq.value - 1,)).copy(), n.value


def pf_relpos_upload(relpos: Relpos, stream=None) -> None:
    _check(_lib.pf_relpos_upload(relpos.handle, _stream(stream)))


def pf_relpos_destroy(relpos: Relpos) -> None:
    h, relpos.handle = relpos.handle, None
    if h:
        _lib.pf_relpos_destroy(h)


def pf_relpos_bias_floats(relpos: Relpos) -> int:
    return int(_lib.pf_relpos_bias_floats(relpos.handle))


def pf_relpos_bias(relpos, H, table, bias, stream=None) -> None:
    """table: H x n_buckets float32, bias: H x pf_relpos_bias_floats float32."""
    dev, f32 = _device(), torch.float32
    _check(_lib.pf_relpos_bias(relpos.handle, H, _flat(table, H * relpos.n_buckets, f32, "table", dev),
                               _flat(bias, H * relpos.bias_floats, f32, "bias", dev), _stream_on(stream, dev)))


# A pf_attn_tensor as bytes: a third of the time a ctypes structure takes.
_pack_rows = struct.Struct("Pqqq").pack


def _rows(t, name, dev):
    """pf_attn_tensor of a (sequences, heads, tokens, 64) bf16 view on device
    dev: any strides but the last, which must be 1."""
    s = t.stride()
    if t.dtype is not torch.bfloat16 or t.get_device() != dev or len(s) != 4:
        raise ValueError(f"{name}: expected a 4-d bfloat16 tensor on the GPU in use, got {len(s)}-d "
                         f"{t.dtype} on {t.device}")
    seq, head, tok, col = s
    if col != 1 and t.shape[3] != 1:
        raise ValueError(f"{name}: the head dim must be contiguous")
    if (seq | head | tok) & 7 or tok < 64:
        # Strides of one sequence, head or token are never used: any will do.
        B, H, n, _ = t.shape
        seq, head, tok = seq if B > 1 else 0, head if H > 1 else 0, tok if n > 1 else 64
    return _pack_rows(t.data_ptr(), seq, head, tok)


def _flat(t, n, dtype, name, dev):
    """Address of at least n contiguous elements on device dev; None and
    integers pass."""
    if t is None or isinstance(t, int):
        return t
    if t.dtype is not dtype or t.get_device() != dev or not t.is_contiguous() or t.numel() < n:
        raise ValueError(f"{name}: expected {n} contiguous {dtype} elements on the GPU in use")
    return t.data_ptr()


def _shapes(want, *pairs):
    for t, name in pairs:
        if t.shape != want:
            raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(want)}")


def _device():
    """The current device; -2, which no tensor is on, before the GPU is in use."""
    return _current_device() if torch.cuda.is_initialized() else -2


def _stream_on(s, dev):
    """_stream, with the current device at hand (-2: none)."""
    return _raw_stream(dev) if s is None and dev >= 0 and _raw_stream is not None else _stream(s)


def pf_attn_relpos_fwd(layout, relpos, scale, Q, K, V, bias, O, lse, q_start=None, kv_len=None,
                       workspace=None, ws_bytes=0, stream=None) -> None:
    """Q, O: (B, H, Sq, 64), K, V: (B, H_kv, Skv, 64) bf16 tensors of any
    strides with a contiguous last dim; bias: of pf_relpos_bias; lse: (B, H, Sq)
    float32, contiguous; q_start, kv_len: B int32 on the GPU, or None."""
    dev, f32, i32 = _device(), torch.float32, torch.int32
    q, k, v, o = _rows(Q, "Q", dev), _rows(K, "K", dev), _rows(V, "V", dev), _rows(O, "O", dev)
    sq, sk = Q.shape, K.shape
    (B, H, Sq, d), (Bk, Hk, Skv, dk) = sq, sk
    if Bk != B or dk != d:
        raise ValueError(f"K: shape {tuple(sk)} does not go with Q's {tuple(sq)}")
    _shapes(sk, (V, "V"))
    _shapes(sq, (O, "O"))
    _check(_lib.pf_attn_relpos_fwd(layout.handle, relpos.handle, B, H, Hk, Sq, Skv, d, scale, q, k, v,
                                   _flat(bias, H * relpos.bias_floats, f32, "bias", dev), o,
                                   _flat(lse, B * H * Sq, f32, "lse", dev),
                                   _flat(q_start, B, i32, "q_start", dev),
                                   _flat(kv_len, B, i32, "kv_len", dev), _ptr(workspace), ws_bytes,
                                   _stream_on(stream, dev)))


def pf_attn_relpos_bwd(layout, relpos, scale, Q, K, V, bias, O, lse, dO, dQ, dK, dV, dtable,
                       kv_len=None, workspace=None, ws_bytes=0, stream=None) -> None:
    """As pf_attn_relpos_fwd with Sq = Skv; dtable: (H, n_buckets) float32."""
    dev, f32 = _device(), torch.float32
    q, k, v, o = _rows(Q, "Q", dev), _rows(K, "K", dev), _rows(V, "V", dev), _rows(O, "O", dev)
    g, dq = _rows(dO, "dO", dev), _rows(dQ, "dQ", dev)
    dk, dv = _rows(dK, "dK", dev), _rows(dV, "dV", dev)
    sq, sk = Q.shape, K.shape
    (B, H, S, d), (Bk, Hk, Sk, d_k) = sq, sk
    if Bk != B or Sk != S or d_k != d:
        raise ValueError(f"K: shape {tuple(sk)} does not go with Q's {tuple(sq)}")
    _shapes(sk, (V, "V"), (dK, "dK"), (dV, "dV"))
    _shapes(sq, (O, "O"), (dO, "dO"), (dQ, "dQ"))
    _check(_lib.pf_attn_relpos_bwd(layout.handle, relpos.handle, B, H, Hk, S, d, scale, q, k, v,
                                   _flat(bias, H * relpos.bias_floats, f32, "bias", dev), o,
                                   _flat(lse, B * H * S, f32, "lse", dev), g, dq, dk, dv,
                                   _flat(dtable, H * relpos.n_buckets, f32, "dtable", dev),
                                   _flat(kv_len, B, torch.int32, "kv_len", dev), _ptr(workspace),
                                   ws_bytes, _stream_on(stream, dev)))


def pf_attn_relpos_workspace_bytes(layout, relpos, B, H, Sq) -> int:
    return int(_lib.pf_attn_relpos_workspace_bytes(layout.handle, relpos.handle, B, H, Sq))


def pf_dense_gemm(dtype, op, M, N, K, A, B, C, workspace=None, ws_bytes=0, stream=None) -> None:
    _check(_lib.pf_dense_gemm(_dt(dtype), op, M, N, K, _ptr(A), _ptr(B), _ptr(C),
                              _ptr(workspace), ws_bytes, _stream(stream)))


def pf_dense_workspace_bytes(dtype, op, M, N, K) -> int:
    return int(_lib.pf_dense_workspace_bytes(_dt(dtype), op, M, N, K))


def pf_timing_begin(max_launches_per_class: int) -> None:
    _check(_lib.pf_timing_begin(max_launches_per_class))


def pf_timing_end() -> dict:
    """{class name: (timed launches, mean duration in ms)}."""
    counts = (_i32 * PF_KERNEL_COUNT)()
    avg = (ctypes.c_double * PF_KERNEL_COUNT)()
    _check(_lib.pf_timing_end(counts, avg))
    return {n: (int(counts[i]), float(avg[i])) for i, n in enumerate(KERNEL_CLASSES)}


def pf_status_string(status: int) -> str:
    return _lib.pf_status_string(status).decode()


def pf_last_error() -> str:
    return _lib.pf_last_error().decode()
