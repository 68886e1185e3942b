"""The operators around the routed experts on torch tensors: the router in front of fluxmoe_expert_ffn, tokens sorted by
expert and back for experts that run elsewhere, the norms on either side of a block, and their gradients.

Every function checks its tensors, enqueues one call of libfluxmoe.so on `stream` (default: the current one) and returns; the
caller owns all buffers, the outputs among them, and keeps them until the work is done.  Matrices may have any row stride of at
least a row; a row's elements lie next to each other.  What the calls compute stands in include/fluxmoe.h.

The calls write into the tensors' memory and are no part of an autograd graph, also where a tensor requires a gradient: a program
calls the gradients itself, or from a torch.autograd.Function of its own.  eps and scale are numbers; the norms take a tensor
of one, too, and read it at the call, which waits for it where it is on the GPU.
"""
from __future__ import annotations

import ctypes
import functools

import torch

from . import binding as B

_TYPES = {torch.bfloat16: B.BF16, torch.float32: B.F32}
# of a device number, without the Stream object that torch.cuda.current_stream makes (2.7 us of a call's 9)
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _fail(what):
    raise ValueError(what)


def _too_large():
    # a call's sizes, or-ed together, go past 32 bits (or below 0): ctypes would hand on their low half
    _fail("a size is not from 0 to 2^32 - 1")


def _sptr(stream, device):
    if stream is None:
        return _current_stream(device) if _current_stream else torch.cuda.current_stream(device).cuda_stream
    return stream.cuda_stream if isinstance(stream, torch.cuda.Stream) else stream


def _place(t, name):
    """The tensor's device, which has to be the current one."""
    device = t.get_device()
    if device < 0 or device != torch.cuda.current_device():
        _fail("%s must be on the current GPU" % name)
    return device


def _matrix(t, name, rows, cols, device, dtype=None):
    """Row stride of a [rows][cols] matrix (the width where there is but one row)."""
    if t.shape != (rows, cols):
        _fail("%s must be [%d][%d], got %s" % (name, rows, cols, list(t.shape)))
    if (t.dtype != dtype) if dtype is not None else (t.dtype not in _TYPES):
        _fail("%s has type %s" % (name, t.dtype))
    if t.get_device() != device:
        _fail("%s is on another device" % name)
    step, element = t.stride()
    if element != 1 and cols > 1:
        _fail("the elements of a row of %s must lie next to each other" % name)
    if rows <= 1:
        return cols
    if step < cols:                      # an expanded row: the norms' call takes a stride of 0 for the width
        _fail("the rows of %s overlap (stride %d)" % (name, step))
    return step


def _whole(t, name, shape, dtype, device):
    """A contiguous tensor of this shape and type."""
    if t.shape != shape or t.dtype != dtype or not t.is_contiguous() or t.get_device() != device:
        _fail("%s must be contiguous %s %s on the operator's device, got %s %s" % (name, list(shape), dtype, list(t.shape), t.dtype))


def _ptr(t):
    return None if t is None else t.data_ptr()


# ------------------------------------------------------------------------------------------ router
def _route_flags(score, renormalize):
    if score not in ("softmax", "sigmoid"):
        _fail("score must be 'softmax' or 'sigmoid', got %r" % (score,))
    return (B.ROUTE_SIGMOID if score == "sigmoid" else 0) | (B.ROUTE_RENORMALIZE if renormalize else 0)


def _logits(logits):
    if logits.dim() != 2:
        _fail("logits must be [tokens][experts]")
    device = _place(logits, "logits")
    T, E = logits.shape
    if (T | E) >> 32:
        _too_large()
    return device, T, E, _matrix(logits, "logits", T, E, device)


def route(logits, ids, gates, *, bias=None, scale=1.0, score="softmax", renormalize=True, stream=None):
    """ids (int32), gates (float32) [T][K] <- logits [T][E]; bias float32 [E], sigmoid scores only."""
    device, T, E, stride = _logits(logits)
    if ids.dim() != 2:
        _fail("ids must be [tokens][top_k]")
    K = ids.shape[1]
    if K >> 32:
        _too_large()
    _whole(ids, "ids", (T, K), torch.int32, device)
    _whole(gates, "gates", (T, K), torch.float32, device)
    if bias is not None:
        _whole(bias, "bias", (E,), torch.float32, device)
    B.fluxmoe_route(logits.data_ptr(), _TYPES[logits.dtype], T, E, stride, _ptr(bias), K, scale, _route_flags(score, renormalize),
                    ids.data_ptr(), gates.data_ptr(), _sptr(stream, device))


def route_grad(logits, ids, d_gates, d_logits, *, scale=1.0, score="softmax", renormalize=True, stream=None):
    """d_logits [T][E] (the logits' type) <- d_gates float32 [T][K]; ids as route gave them."""
    device, T, E, stride = _logits(logits)
    if ids.dim() != 2:
        _fail("ids must be [tokens][top_k]")
    K = ids.shape[1]
    if K >> 32:
        _too_large()
    _whole(ids, "ids", (T, K), torch.int32, device)
    _whole(d_gates, "d_gates", (T, K), torch.float32, device)
    d_stride = _matrix(d_logits, "d_logits", T, E, device, logits.dtype)
    B.fluxmoe_route_grad(logits.data_ptr(), _TYPES[logits.dtype], T, E, stride, ids.data_ptr(), K, scale,
                         _route_flags(score, renormalize), d_gates.data_ptr(), d_logits.data_ptr(), d_stride, _sptr(stream, device))


# ------------------------------------------------------------------------------------------ tokens by expert and back
def sorted_rows(tokens, top_k, n_experts, align=1) -> int:
    """Rows that the pairs of such a batch can take: what row_pair and the rows' matrices must hold."""
    if (tokens | top_k | n_experts | align) >> 32:
        _too_large()
    return B.fluxmoe_sorted_rows(tokens, top_k, n_experts, align)


def sort_workspace_bytes(tokens, top_k, n_experts) -> int:
    if (tokens | top_k | n_experts) >> 32:
        _too_large()
    return B.fluxmoe_sort_workspace_bytes(tokens, top_k, n_experts)


def sort_tokens(ids, n_experts, offsets, counts, pair_row, row_pair, workspace=None, *, align=1, stream=None):
    """offsets [E + 1], counts [E], pair_row [T][K], row_pair [rows] (all int32) <- ids int32 [T][K]; workspace: bytes."""
    if ids.dim() != 2:
        _fail("ids must be [tokens][top_k]")
    device = _place(ids, "ids")
    T, K = ids.shape
    if (T | K | n_experts | align) >> 32:
        _too_large()
    _whole(ids, "ids", (T, K), torch.int32, device)
    _whole(offsets, "offsets", (n_experts + 1,), torch.int32, device)
    _whole(counts, "counts", (n_experts,), torch.int32, device)
    _whole(pair_row, "pair_row", (T, K), torch.int32, device)
    _whole(row_pair, "row_pair", (row_pair.numel(),), torch.int32, device)
    if workspace is not None:
        _whole(workspace, "workspace", (workspace.numel(),), torch.uint8, device)
    B.fluxmoe_sort_tokens(ids.data_ptr(), T, K, n_experts, align, offsets.data_ptr(), counts.data_ptr(), pair_row.data_ptr(),
                          row_pair.data_ptr(), row_pair.numel(), _ptr(workspace), 0 if workspace is None else workspace.numel(),
                          _sptr(stream, device))


def _order(pair_row, row_pair, H, device):
    if pair_row.dim() != 2:
        _fail("pair_row must be [tokens][top_k]")
    T, K = pair_row.shape
    if (T | K | H) >> 32:
        _too_large()
    _whole(pair_row, "pair_row", (T, K), torch.int32, device)
    if row_pair is not None:
        _whole(row_pair, "row_pair", (row_pair.numel(),), torch.int32, device)
    return T, K


def dispatch(x, pair_row, row_pair, rows, *, stream=None):
    """rows [row_pair.numel()][H] <- x [T][H], both of one type; rows of no pair become 0."""
    device = _place(x, "x")
    H = x.shape[-1]
    T, K = _order(pair_row, row_pair, H, device)
    x_stride = _matrix(x, "x", T, H, device)
    rows_stride = _matrix(rows, "rows", row_pair.numel(), H, device, x.dtype)
    B.fluxmoe_dispatch(x.data_ptr(), _TYPES[x.dtype], T, H, x_stride, pair_row.data_ptr(), K, row_pair.data_ptr(), row_pair.numel(),
                       rows.data_ptr(), rows_stride, _sptr(stream, device))


def combine(rows, pair_row, gates, out, *, accumulate=False, stream=None):
    """out [T][H] <- sum over k of gates [T][K] (None: ones, the gradient of dispatch) times rows [n][H]."""
    device = _place(rows, "rows")
    n, H = rows.shape[0], rows.shape[-1]
    T, K = _order(pair_row, None, H, device)
    rows_stride = _matrix(rows, "rows", n, H, device)
    out_stride = _matrix(out, "out", T, H, device)
    if gates is not None:
        _whole(gates, "gates", (T, K), torch.float32, device)
    B.fluxmoe_combine(rows.data_ptr(), _TYPES[rows.dtype], n, H, rows_stride, pair_row.data_ptr(), _ptr(gates), T, K, out.data_ptr(),
                      _TYPES[out.dtype], out_stride, B.FFN_ACCUMULATE if accumulate else 0, _sptr(stream, device))


def combine_grad(d_out, rows, pair_row, row_pair, gates, d_rows, d_gates, *, stream=None):
    """d_rows [n][H] (the rows' type), d_gates float32 [T][K] <- d_out [T][H], and what combine was given."""
    device = _place(d_out, "d_out")
    n, H = row_pair.numel(), d_out.shape[-1]
    T, K = _order(pair_row, row_pair, H, device)
    d_out_stride = _matrix(d_out, "d_out", T, H, device)
    rows_stride = _matrix(rows, "rows", n, H, device)
    d_rows_stride = _matrix(d_rows, "d_rows", n, H, device, rows.dtype)
    _whole(gates, "gates", (T, K), torch.float32, device)
    _whole(d_gates, "d_gates", (T, K), torch.float32, device)
    B.fluxmoe_combine_grad(d_out.data_ptr(), _TYPES[d_out.dtype], d_out_stride, rows.data_ptr(), _TYPES[rows.dtype], n, H, rows_stride,
                           pair_row.data_ptr(), row_pair.data_ptr(), gates.data_ptr(), T, K, d_rows.data_ptr(), d_rows_stride,
                           d_gates.data_ptr(), _sptr(stream, device))


# ------------------------------------------------------------------------------------------ norms around a block
@functools.lru_cache(maxsize=256)
def _norm_desc(*fields):
    """The argument block of a kind of call: sizes, types and constants as plain numbers, nothing of its tensors."""
    return ctypes.pointer(B.NormDesc(*fields))


def _norm_inputs(residual, w_pre, y, gate, w_post, gate_sigmoid, zero_centred):
    """(T, H, device, flags) of the tensors that the forward and the gradient call share"""
    device = _place(residual, "residual")
    if residual.dim() != 2:
        _fail("residual must be [tokens][hidden]")
    T, H = residual.shape
    if (T | H) >> 32:
        _too_large()
    if w_pre.dtype not in _TYPES:
        _fail("w_pre has type %s" % w_pre.dtype)
    _whole(w_pre, "w_pre", (H,), w_pre.dtype, device)
    flags = B.NORM_ZERO_CENTRED if zero_centred else 0
    if y is None and (gate is not None or w_post is not None):
        _fail("a gate or w_post without y")
    if w_post is not None:
        _whole(w_post, "w_post", (H,), w_pre.dtype, device)
    if gate is not None:
        token = gate.dim() == 2
        _whole(gate, "gate", (T, 1) if token else (H,), torch.float32, device)
        flags |= (B.NORM_GATE_TOKEN if token else B.NORM_GATE_CHANNEL) | (B.NORM_GATE_SIGMOID if gate_sigmoid else 0)
    elif gate_sigmoid:
        _fail("gate_sigmoid without a gate")
    return T, H, device, flags


def block_norm(residual, w_pre, normed, *, y=None, gate=None, w_post=None, residual_out=None, eps=1e-6, scale=1.0, gate_sigmoid=False,
               zero_centred=False, stream=None):
    """residual_out, normed (bfloat16) [T][H] <- residual, y [T][H]; gate float32 [T][1] or [H]; without y the norm alone."""
    T, H, device, flags = _norm_inputs(residual, w_pre, y, gate, w_post, gate_sigmoid, zero_centred)
    if (residual_out is None) != (y is None):
        _fail("residual_out is given where y is")
    r_stride = _matrix(residual, "residual", T, H, device)
    n_stride = _matrix(normed, "normed", T, H, device, torch.bfloat16)
    y_stride = o_stride = y_type = 0
    if y is not None:
        y_stride, y_type = _matrix(y, "y", T, H, device), _TYPES[y.dtype]
        o_stride = _matrix(residual_out, "residual_out", T, H, device, residual.dtype)
    desc = _norm_desc(H, y_type, _TYPES[residual.dtype], _TYPES[w_pre.dtype], flags, float(eps), float(scale), 0, y_stride, r_stride,
                      o_stride, n_stride)
    B.fluxmoe_block_norm(desc, T, _ptr(y), residual.data_ptr(), _ptr(gate), _ptr(w_post), w_pre.data_ptr(), _ptr(residual_out),
                         normed.data_ptr(), _sptr(stream, device))


def block_norm_grad_workspace_bytes(tokens, hidden) -> int:
    if (tokens | hidden) >> 32:
        _too_large()
    return B.fluxmoe_block_norm_grad_workspace_bytes(tokens, hidden)


def block_norm_grad(residual_out, w_pre, d_normed, d_residual, d_w_pre, workspace, *, d_residual_out=None, y=None, gate=None, w_post=None,
                    d_y=None, d_gate=None, d_w_post=None, eps=1e-6, scale=1.0, gate_sigmoid=False, zero_centred=False, stream=None):
    """d_residual, d_y [T][H] and float32 d_gate, d_w_pre, d_w_post <- d_normed (bfloat16), d_residual_out (None: 0), and what
    block_norm was given and left; workspace: uint8, block_norm_grad_workspace_bytes of them."""
    T, H, device, flags = _norm_inputs(residual_out, w_pre, y, gate, w_post, gate_sigmoid, zero_centred)
    for name, given, grad in (("y", y, d_y), ("gate", gate, d_gate), ("w_post", w_post, d_w_post)):
        if (given is None) != (grad is None):
            _fail("d_%s is given where %s is" % (name, name))
    rt = residual_out.dtype
    o_stride = _matrix(residual_out, "residual_out", T, H, device)
    dn_stride = _matrix(d_normed, "d_normed", T, H, device, torch.bfloat16)
    dr_stride = _matrix(d_residual, "d_residual", T, H, device, rt)
    do_stride = _matrix(d_residual_out, "d_residual_out", T, H, device, rt) if d_residual_out is not None else 0
    y_stride = dy_stride = y_type = 0
    if y is not None:
        y_stride, y_type = _matrix(y, "y", T, H, device), _TYPES[y.dtype]
        dy_stride = _matrix(d_y, "d_y", T, H, device, y.dtype)
    _whole(d_w_pre, "d_w_pre", (H,), torch.float32, device)
    if d_w_post is not None:
        _whole(d_w_post, "d_w_post", (H,), torch.float32, device)
    if d_gate is not None:
        _whole(d_gate, "d_gate", tuple(gate.shape), torch.float32, device)
    _whole(workspace, "workspace", (workspace.numel(),), torch.uint8, device)
    desc = _norm_desc(H, y_type, _TYPES[rt], _TYPES[w_pre.dtype], flags, float(eps), float(scale), 0, y_stride, 0, o_stride,
                      0, dy_stride, dr_stride, do_stride, dn_stride)
    B.fluxmoe_block_norm_grad(desc, T, _ptr(y), residual_out.data_ptr(), _ptr(gate), _ptr(w_post), w_pre.data_ptr(), _ptr(d_residual_out),
                              d_normed.data_ptr(), d_residual.data_ptr(), _ptr(d_y), _ptr(d_gate), _ptr(d_w_post), d_w_pre.data_ptr(),
                              workspace.data_ptr(), workspace.numel(), _sptr(stream, device))
