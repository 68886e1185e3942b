"""Experts in 4-bit floating point (MXFP4) on torch tensors: rows to 4 bits and back, the experts' products on rows that
moe_block.sort_tokens and moe_block.dispatch put in order, SwiGLU between them, and the gradients.

As in moe_block: every function checks its tensors, enqueues one call of libfluxmoe.so on `stream` (default: the current one) and
returns; the caller owns all buffers, the outputs among them, and the calls are no part of an autograd graph.  Matrices may have any
row stride of at least a row.  Numbers in 4 bits are two uint8 tensors: codes [rows][columns / 2], two columns to a byte, and
scales [rows][columns / 32].  What the calls compute stands in include/fluxmoe.h.
"""
from __future__ import annotations

import ctypes
import functools

import torch

from . import binding as B
from .moe_block import _TYPES, _fail, _matrix, _place, _ptr, _sptr, _too_large, _whole

BLOCK = 32                      # columns that share a scale


def _as_rows(t, name, rows_of):
    """All experts' rows as those of one matrix: more than two dimensions, without gaps"""
    if t.dim() < 2 or not t.is_contiguous():
        _fail("%s must be [rows][columns], or contiguous with more dimensions" % name)
    if t.shape[:-1] != rows_of.shape[:-1]:
        _fail("%s must have the rows of the other tensors, got %s" % (name, list(t.shape)))
    return t.view(-1, t.shape[-1])


def _mx_rows(x, x_name, codes, scales):
    if not x.dim() == codes.dim() == scales.dim() == 2:
        x, codes, scales = _as_rows(x, x_name, codes), _as_rows(codes, "codes", scales), _as_rows(scales, "scales", x)
    device = _place(x, x_name)
    rows, columns = x.shape
    if columns % BLOCK:
        _fail("%s must have a multiple of %d columns, got %d" % (x_name, BLOCK, columns))
    if columns >> 32:
        _too_large()
    return (device, x, rows, columns, _matrix(x, x_name, rows, columns, device), codes, _matrix(codes, "codes", rows, columns // 2, device, torch.uint8),
            scales, _matrix(scales, "scales", rows, columns // BLOCK, device, torch.uint8))


def quantize(x, codes, scales, *, stream=None):
    """codes uint8 [...][C / 2], scales uint8 [...][C / 32] <- x [...][C] (bfloat16 or float32)."""
    device, x, rows, C, stride, codes, c_stride, scales, s_stride = _mx_rows(x, "x", codes, scales)
    B.fluxmoe_mx_quantize(x.data_ptr(), _TYPES[x.dtype], rows, C, stride, codes.data_ptr(), c_stride, scales.data_ptr(), s_stride,
                          _sptr(stream, device))


def dequantize(codes, scales, out, *, stream=None):
    """out [...][C] (bfloat16 or float32) <- codes uint8 [...][C / 2], scales uint8 [...][C / 32]."""
    device, out, rows, C, stride, codes, c_stride, scales, s_stride = _mx_rows(out, "out", codes, scales)
    B.fluxmoe_mx_dequantize(codes.data_ptr(), c_stride, scales.data_ptr(), s_stride, rows, C, out.data_ptr(), _TYPES[out.dtype], stride,
                            _sptr(stream, device))


@functools.lru_cache(maxsize=256)
def _product_desc(*fields):
    """The argument block of a kind of call: sizes, types and strides as plain numbers, nothing of its tensors."""
    return ctypes.pointer(B.MxProductDesc(*fields))


def _experts(offsets, counts, w_codes, w_scales, device):
    """(E, N, K) of the experts' weights"""
    if w_codes.dim() != 3:
        _fail("w_codes must be [experts][outputs][columns / 2]")
    E, N, half = w_codes.shape
    if (E | N | 2 * half) >> 32:
        _too_large()
    if half % (BLOCK // 2):
        _fail("w_codes must have whole blocks of %d columns, got %d" % (BLOCK, 2 * half))
    _whole(w_codes, "w_codes", (E, N, half), torch.uint8, device)
    _whole(w_scales, "w_scales", (E, N, half // (BLOCK // 2)), torch.uint8, device)
    _whole(offsets, "offsets", (E + 1,), torch.int32, device)
    _whole(counts, "counts", (E,), torch.int32, device)
    return E, N, 2 * half


def product(rows, offsets, counts, w_codes, w_scales, out, *, row_scales=None, stream=None):
    """out [n][N] (bfloat16 or float32) <- rows times their expert's weights: rows bfloat16 [n][K], or uint8 codes [n][K / 2] with
    row_scales [n][K / 32]; offsets, counts as sort_tokens gives them; w_codes [E][N][K / 2], w_scales [E][N][K / 32].  Rows of no
    expert are left as they are in out; many of them, as a large `align` of the sort leaves, cost time, and so does K no multiple of 128."""
    device = _place(rows, "rows")
    E, N, K = _experts(offsets, counts, w_codes, w_scales, device)
    n = rows.shape[0]
    s_stride = 0
    if row_scales is None:
        r_stride, r_type = _matrix(rows, "rows", n, K, device, torch.bfloat16), B.BF16
    else:
        r_stride, r_type = _matrix(rows, "rows", n, K // 2, device, torch.uint8), B.MXFP4
        s_stride = _matrix(row_scales, "row_scales", n, K // BLOCK, device, torch.uint8)
    o_stride = _matrix(out, "out", n, N, device)
    desc = _product_desc(E, N, K, r_type, _TYPES[out.dtype], 0, n, r_stride, s_stride, o_stride)
    B.fluxmoe_mx_product(desc, rows.data_ptr(), _ptr(row_scales), offsets.data_ptr(), counts.data_ptr(), w_codes.data_ptr(),
                         w_scales.data_ptr(), out.data_ptr(), _sptr(stream, device))


def product_grad(d_out, offsets, counts, w_codes, w_scales, d_rows, *, stream=None):
    """d_rows [n][K] (bfloat16 or float32) <- d_out bfloat16 [n][N], and what product was given.  Rows of no expert are left as they
    are in d_rows."""
    device = _place(d_out, "d_out")
    E, N, K = _experts(offsets, counts, w_codes, w_scales, device)
    n = d_out.shape[0]
    o_stride = _matrix(d_out, "d_out", n, N, device, torch.bfloat16)
    r_stride = _matrix(d_rows, "d_rows", n, K, device)
    desc = _product_desc(E, N, K, _TYPES[d_rows.dtype], B.BF16, 0, n, r_stride, 0, o_stride)
    B.fluxmoe_mx_product_grad(desc, d_out.data_ptr(), offsets.data_ptr(), counts.data_ptr(), w_codes.data_ptr(), w_scales.data_ptr(),
                              d_rows.data_ptr(), _sptr(stream, device))


def _gate_up(gate_up, h, h_name):
    device = _place(gate_up, "gate_up")
    if h.dim() != 2:
        _fail("%s must be [rows][ffn]" % h_name)
    rows, F = h.shape
    if F >> 31:
        _too_large()
    return device, rows, F, _matrix(gate_up, "gate_up", rows, 2 * F, device), _matrix(h, h_name, rows, F, device)


def swiglu(gate_up, h, *, stream=None):
    """h [rows][F] <- silu(gate_up[:, :F]) * gate_up[:, F:]."""
    device, rows, F, stride, h_stride = _gate_up(gate_up, h, "h")
    B.fluxmoe_swiglu(gate_up.data_ptr(), _TYPES[gate_up.dtype], rows, F, stride, h.data_ptr(), _TYPES[h.dtype], h_stride,
                     _sptr(stream, device))


def swiglu_grad(gate_up, d_h, d_gate_up, *, stream=None):
    """d_gate_up [rows][2 F] (gate_up's type; may be gate_up itself) <- gate_up, d_h [rows][F]."""
    device, rows, F, stride, h_stride = _gate_up(gate_up, d_h, "d_h")
    d_stride = _matrix(d_gate_up, "d_gate_up", rows, 2 * F, device, gate_up.dtype)
    B.fluxmoe_swiglu_grad(gate_up.data_ptr(), _TYPES[gate_up.dtype], rows, F, stride, d_h.data_ptr(), _TYPES[d_h.dtype], h_stride,
                          d_gate_up.data_ptr(), d_stride, _sptr(stream, device))
