"""Thin ctypes binding of the C ABI in include/lite_attn_layer.h (same names, argument marshalling only): what stands before
and behind the attention call of ``lite_attn`` in a transformer block.

Tensors are given as tuples of an integer device address (e.g. tensor.data_ptr()) and strides in elements: (address, stride_b,
stride_h, stride_n) of [batch, heads, seqlen, head_dim], (address, stride_b, stride_n) of [batch, rows, dim]; None, or an address
of 0, leaves one out where the header allows it.  Vectors, frequencies and workspaces are plain addresses.  ``hip_stream`` is the
integer value of a hipStream_t.
"""
from __future__ import annotations

import ctypes

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


class Heads(ctypes.Structure):
    """lite_attn_heads_t"""
    _fields_ = [("data", ctypes.c_void_p), ("stride_b", ctypes.c_int64), ("stride_h", ctypes.c_int64),
                ("stride_n", ctypes.c_int64)]


class Positions(ctypes.Structure):
    """lite_attn_positions_t"""
    _fields_ = [("freqs", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("positions_stride_b", ctypes.c_int64),
                ("token_start", ctypes.c_int32)]


class RotaryFwd(ctypes.Structure):
    """lite_attn_rotary_fwd_t"""
    _fields_ = [("q", Heads), ("k", Heads), ("q_out", Heads), ("k_out", Heads), ("q_weight", ctypes.c_void_p),
                ("k_weight", ctypes.c_void_p), ("at", Positions)]


class RotaryBwd(ctypes.Structure):
    """lite_attn_rotary_bwd_t"""
    _fields_ = [("q", Heads), ("k", Heads), ("dq_out", Heads), ("dk_out", Heads), ("dq", Heads), ("dk", Heads),
                ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("at", Positions),
                ("dq_weight", ctypes.c_void_p), ("dk_weight", ctypes.c_void_p), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t)]


class ResidualDesc(ctypes.Structure):
    """lite_attn_residual_desc_t"""
    _fields_ = [
        ("batch", ctypes.c_int32), ("seqlen", ctypes.c_int32), ("dim", ctypes.c_int32), ("tokens_per_mod", ctypes.c_int32),
        ("dtype", ctypes.c_int32), ("stream_dtype", ctypes.c_int32), ("param_dtype", ctypes.c_int32),
        ("post_norm", ctypes.c_int32), ("pre_norm", ctypes.c_int32), ("post_eps", ctypes.c_float),
        ("pre_eps", ctypes.c_float), ("residual_scale", ctypes.c_float),
    ]


class Rows(ctypes.Structure):
    """lite_attn_rows_t"""
    _fields_ = [("data", ctypes.c_void_p), ("stride_b", ctypes.c_int64), ("stride_n", ctypes.c_int64)]


class ResidualFwd(ctypes.Structure):
    """lite_attn_residual_fwd_t"""
    _fields_ = [("x", Rows), ("y", Rows), ("x_out", Rows), ("h", Rows), ("gate", Rows), ("scale", Rows), ("shift", Rows),
                ("post_weight", ctypes.c_void_p), ("pre_weight", ctypes.c_void_p), ("pre_bias", ctypes.c_void_p)]


class ResidualBwd(ctypes.Structure):
    """lite_attn_residual_bwd_t"""
    _fields_ = [("dh", Rows), ("dx_out", Rows), ("x_out", Rows), ("y", Rows), ("dx", Rows), ("dy", Rows), ("gate", Rows),
                ("scale", Rows), ("post_weight", ctypes.c_void_p), ("pre_weight", ctypes.c_void_p),
                ("pre_bias", ctypes.c_void_p), ("dgate", ctypes.c_void_p), ("dscale", ctypes.c_void_p),
                ("dshift", ctypes.c_void_p), ("dpost_weight", ctypes.c_void_p), ("dpre_weight", ctypes.c_void_p),
                ("dpre_bias", ctypes.c_void_p), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


for _n, _desc, _args in (("rotary_fwd", RotaryDesc, RotaryFwd), ("rotary_bwd", RotaryDesc, RotaryBwd),
                         ("residual_norm_fwd", ResidualDesc, ResidualFwd),
                         ("residual_norm_bwd", ResidualDesc, ResidualBwd)):
    _f = getattr(_lib, "lite_attn_" + _n)
    _f.argtypes = [ctypes.POINTER(_desc), ctypes.POINTER(_args), ctypes.c_void_p]
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
        desc, RotaryFwd(q or (), k or (), q_out or (), k_out or (), q_weight, k_weight,
                        (freqs, positions, positions_stride_b, token_start)), hip_stream))


def lite_attn_rotary_bwd(desc, q, k, dq_out, dk_out, dq, dk, freqs, *, q_weight=0, k_weight=0, dq_weight=0, dk_weight=0,
                         workspace=0, workspace_bytes=0, positions=0, positions_stride_b=0, token_start=0, hip_stream):
    _check(_lib.lite_attn_rotary_bwd(
        desc, RotaryBwd(q or (), k or (), dq_out or (), dk_out or (), dq or (), dk or (), q_weight, k_weight,
                        (freqs, positions, positions_stride_b, token_start), dq_weight, dk_weight, workspace,
                        workspace_bytes), hip_stream))


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
        desc, ResidualFwd(x or (), y or (), x_out or (), h or (), gate or (), scale or (), shift or (), post_weight, pre_weight,
                          pre_bias), hip_stream))


def lite_attn_residual_norm_bwd(desc, dh, dx_out, x_out, y, dx, dy, *, gate=None, scale=None, post_weight=0, pre_weight=0,
                                pre_bias=0, dgate=0, dscale=0, dshift=0, dpost_weight=0, dpre_weight=0, dpre_bias=0,
                                workspace=0, workspace_bytes=0, hip_stream):
    _check(_lib.lite_attn_residual_norm_bwd(
        desc, ResidualBwd(dh or (), dx_out or (), x_out or (), y or (), dx or (), dy or (), gate or (), scale or (),
                          post_weight, pre_weight, pre_bias, dgate, dscale, dshift, dpost_weight, dpre_weight, dpre_bias,
                          workspace, workspace_bytes), hip_stream))


def lite_attn_residual_norm_bwd_workspace(desc: ResidualDesc) -> int:
    """Bytes of workspace that the gradients of gate, scale, shift, weights and bias need."""
    return int(_lib.lite_attn_residual_norm_bwd_workspace(desc))
