"""Thin ctypes binding of the C ABI in include/lite_attn_layer.h (same names, argument marshalling only): what stands before
and behind the attention call of ``lite_attn`` in a transformer block.

Tensors are given as tuples of an integer device address (e.g. tensor.data_ptr()) and strides in elements: (address, stride_b,
stride_h, stride_n) of [batch, heads, seqlen, head_dim], (address, stride_b, stride_n) of [batch, rows, dim]; None, or an address
of 0, leaves one out where the header allows it.  Vectors, frequencies and workspaces are plain addresses.  ``hip_stream`` is the
integer value of a hipStream_t.
"""
from __future__ import annotations

import ctypes
import struct

import numpy as np

from .lite_attn import LiteAttnError, _check, _lib  # noqa: F401  (the one library, the one error type)

# element types and norms (include/lite_attn_layer.h)
LITE_ATTN_BF16 = 0
LITE_ATTN_F16 = 1
LITE_ATTN_F32 = 2
LITE_ATTN_NORM_NONE = 0
LITE_ATTN_NORM_HEAD = 1
LITE_ATTN_NORM_ROW = 2
LITE_ATTN_NORM_RMS = 3
LITE_ATTN_NORM_LAYER = 4


class RotaryDesc(ctypes.Structure):
    """lite_attn_rotary_desc_t"""
    _fields_ = [
        ("batch", ctypes.c_int32), ("seqlen", ctypes.c_int32), ("heads_q", ctypes.c_int32), ("heads_k", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("weight_dtype", ctypes.c_int32), ("norm", ctypes.c_int32),
        ("halves", ctypes.c_int32), ("pairs", ctypes.c_int32), ("grid", ctypes.c_int32 * 3), ("eps", ctypes.c_float),
    ]


class ResidualDesc(ctypes.Structure):
    """lite_attn_residual_desc_t"""
    _fields_ = [
        ("batch", ctypes.c_int32), ("seqlen", ctypes.c_int32), ("dim", ctypes.c_int32), ("tokens_per_mod", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("stream_dtype", ctypes.c_int32), ("param_dtype", ctypes.c_int32),
        ("post_norm", ctypes.c_int32), ("pre_norm", ctypes.c_int32), ("post_eps", ctypes.c_float),
        ("pre_eps", ctypes.c_float), ("residual_scale", ctypes.c_float),
    ]


# The argument structs, packed for each call (a third of the time that filling a ctypes.Structure takes): P an address, q a
# stride, four of a lite_attn_heads_t, three of a lite_attn_rows_t.
_POSITIONS = "PPqi0P"                                                  # lite_attn_positions_t
_ROTARY_FWD = struct.Struct("@" + 4 * "Pqqq" + "PP" + _POSITIONS)      # lite_attn_rotary_fwd_t
_ROTARY_BWD = struct.Struct("@" + 6 * "Pqqq" + "PP" + _POSITIONS + "PPPN")  # lite_attn_rotary_bwd_t
_RESIDUAL_FWD = struct.Struct("@" + 7 * "Pqq" + "PPP")                 # lite_attn_residual_fwd_t
_RESIDUAL_BWD = struct.Struct("@" + 8 * "Pqq" + "PPP" + 6 * "P" + "PN")  # lite_attn_residual_bwd_t
_NO_HEADS = (0, 0, 0, 0)
_NO_ROWS = (0, 0, 0)

for _n, _desc in (("rotary_fwd", RotaryDesc), ("rotary_bwd", RotaryDesc), ("residual_norm_fwd", ResidualDesc),
                  ("residual_norm_bwd", ResidualDesc)):
    _f = getattr(_lib, "lite_attn_" + _n)
    _f.argtypes = [ctypes.POINTER(_desc), ctypes.c_char_p, ctypes.c_void_p]
    _f.restype = ctypes.c_int
for _n, _desc in (("rotary_bwd_workspace", RotaryDesc), ("residual_norm_bwd_workspace", ResidualDesc)):
    _f = getattr(_lib, "lite_attn_" + _n)
    _f.argtypes = [ctypes.POINTER(_desc)]
    _f.restype = ctypes.c_size_t
_lib.lite_attn_rotary_freqs.argtypes = [ctypes.c_int32 * 3, ctypes.c_double, ctypes.c_void_p]
_lib.lite_attn_rotary_freqs.restype = ctypes.c_int


def make_rotary_desc(batch, seqlen, heads_q, heads_k, head_dim=128, *, dtype=LITE_ATTN_BF16, weight_dtype=LITE_ATTN_F32,
                     norm=LITE_ATTN_NORM_NONE, halves=False, pairs=None, grid=(1, 1, 1), eps=1e-6) -> RotaryDesc:
    """lite_attn_rotary_desc_t.  `pairs`: pairs of a head that are turned, by default all."""
    return RotaryDesc(batch, seqlen, heads_q, heads_k, head_dim, dtype, weight_dtype, norm, 1 if halves else 0,
                      head_dim // 2 if pairs is None else pairs, (ctypes.c_int32 * 3)(*grid), eps)


def lite_attn_rotary_fwd(desc, q, k, q_out, k_out, freqs, *, q_weight=0, k_weight=0, positions=0, positions_stride_b=0,
                         token_start=0, hip_stream):
    _check(_lib.lite_attn_rotary_fwd(
        desc, _ROTARY_FWD.pack(*(q or _NO_HEADS), *(k or _NO_HEADS), *(q_out or _NO_HEADS), *(k_out or _NO_HEADS), q_weight,
                               k_weight, freqs, positions, positions_stride_b, token_start), hip_stream))


def lite_attn_rotary_bwd(desc, q, k, dq_out, dk_out, dq, dk, freqs, *, q_weight=0, k_weight=0, dq_weight=0, dk_weight=0,
                         workspace=0, workspace_bytes=0, positions=0, positions_stride_b=0, token_start=0, hip_stream):
    _check(_lib.lite_attn_rotary_bwd(
        desc, _ROTARY_BWD.pack(*(q or _NO_HEADS), *(k or _NO_HEADS), *(dq_out or _NO_HEADS), *(dk_out or _NO_HEADS),
                               *(dq or _NO_HEADS), *(dk or _NO_HEADS), q_weight, k_weight, freqs, positions,
                               positions_stride_b, token_start, dq_weight, dk_weight, workspace, workspace_bytes), hip_stream))


def lite_attn_rotary_bwd_workspace(desc: RotaryDesc) -> int:
    """Bytes of workspace that the gradients of the weights need."""
    return int(_lib.lite_attn_rotary_bwd_workspace(desc))


def lite_attn_rotary_freqs(axis_pairs, theta=10000.0) -> np.ndarray:
    """-> float64 [3, sum(axis_pairs)] radians per position, on the host."""
    out = np.zeros((3, max(1, sum(axis_pairs))), dtype=np.float64)
    _check(_lib.lite_attn_rotary_freqs((ctypes.c_int32 * 3)(*axis_pairs), theta, out.ctypes.data))
    return out[:, :sum(axis_pairs)]


def make_residual_desc(batch, seqlen, dim, *, dtype=LITE_ATTN_BF16, stream_dtype=LITE_ATTN_F32, param_dtype=LITE_ATTN_F32,
                       post_norm=LITE_ATTN_NORM_NONE, pre_norm=LITE_ATTN_NORM_LAYER, post_eps=1e-6, pre_eps=1e-6,
                       residual_scale=1.0, tokens_per_mod=None) -> ResidualDesc:
    """lite_attn_residual_desc_t.  `tokens_per_mod`: by default one row of gate, scale and shift for the whole sample."""
    return ResidualDesc(batch, seqlen, dim, max(1, seqlen) if tokens_per_mod is None else tokens_per_mod, dtype, stream_dtype,
                        param_dtype, post_norm, pre_norm, post_eps, pre_eps, residual_scale)


def lite_attn_residual_norm_fwd(desc, x, y, x_out, h, *, gate=None, scale=None, shift=None, post_weight=0, pre_weight=0,
                                pre_bias=0, hip_stream):
    _check(_lib.lite_attn_residual_norm_fwd(
        desc, _RESIDUAL_FWD.pack(*(x or _NO_ROWS), *(y or _NO_ROWS), *(x_out or _NO_ROWS), *(h or _NO_ROWS),
                                 *(gate or _NO_ROWS), *(scale or _NO_ROWS), *(shift or _NO_ROWS), post_weight, pre_weight,
                                 pre_bias), hip_stream))


def lite_attn_residual_norm_bwd(desc, dh, dx_out, x_out, y, dx, dy, *, gate=None, scale=None, post_weight=0, pre_weight=0,
                                pre_bias=0, dgate=0, dscale=0, dshift=0, dpost_weight=0, dpre_weight=0, dpre_bias=0,
                                workspace=0, workspace_bytes=0, hip_stream):
    _check(_lib.lite_attn_residual_norm_bwd(
        desc, _RESIDUAL_BWD.pack(*(dh or _NO_ROWS), *(dx_out or _NO_ROWS), *(x_out or _NO_ROWS), *(y or _NO_ROWS),
                                 *(dx or _NO_ROWS), *(dy or _NO_ROWS), *(gate or _NO_ROWS), *(scale or _NO_ROWS), post_weight,
                                 pre_weight, pre_bias, dgate, dscale, dshift, dpost_weight, dpre_weight, dpre_bias, workspace,
                                 workspace_bytes), hip_stream))


def lite_attn_residual_norm_bwd_workspace(desc: ResidualDesc) -> int:
    """Bytes of workspace that the gradients of gate, scale, shift, weights and bias need."""
    return int(_lib.lite_attn_residual_norm_bwd_workspace(desc))
