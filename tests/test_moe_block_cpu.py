"""Host side of the operators around the routed experts: sizes, and what the calls refuse.  Nothing is launched: every call here is
turned down before that, or has nothing to do."""
import ctypes

import pytest
import torch

from paper_2604_02715_amd import binding as B
from paper_2604_02715_amd import moe_block as M

P = 1 << 20                     # stands for a device address; no accepted call reaches it


def refused(status, fn, *args, **kw):
    with pytest.raises(B.FluxmoeError) as e:
        fn(*args, **kw)
    assert e.value.status == status, str(e.value)
    return str(e.value)


def route(logits=P, type_=B.F32, T=4, E=8, stride=8, bias=None, K=2, scale=1.0, flags=0, ids=P, w=P):
    B.fluxmoe_route(logits, type_, T, E, stride, bias, K, scale, flags, ids, w)


def route_grad(logits=P, type_=B.F32, T=4, E=8, stride=8, ids=P, K=2, scale=1.0, flags=0, dw=P, d=P, d_stride=8):
    B.fluxmoe_route_grad(logits, type_, T, E, stride, ids, K, scale, flags, dw, d, d_stride)


BAD_ROUTES = [dict(type_=2), dict(T=(1 << 20) + 1), dict(E=0), dict(E=4097, stride=4097), dict(K=0), dict(K=9), dict(E=100, stride=100, K=65),
              dict(flags=4), dict(logits=None), dict(ids=None), dict(stride=7), dict(logits=P + 2), dict(ids=P + 1)]


@pytest.mark.parametrize("kw", BAD_ROUTES + [dict(bias=P), dict(w=None), dict(w=P + 2), dict(flags=B.ROUTE_SIGMOID, bias=P + 2)])
def test_route_refuses(kw):
    refused(-1, route, **kw)


@pytest.mark.parametrize("kw", BAD_ROUTES + [dict(dw=None), dict(d=None), dict(d_stride=7), dict(d=P + 2)])
def test_route_grad_refuses(kw):
    refused(-1, route_grad, **kw)


def test_no_tokens_is_no_work():
    route(T=0, logits=None, ids=None, w=None)
    route_grad(T=0, logits=None, ids=None, dw=None, d=None)
    B.fluxmoe_combine(None, 0, 0, 64, 64, None, None, 0, 2, None, 0, 64)
    B.fluxmoe_dispatch(None, 0, 0, 64, 64, None, 2, None, 0, None, 64)
    B.fluxmoe_combine_grad(None, 0, 64, None, 0, 0, 64, 64, None, None, None, 0, 2, None, 64, None)


def test_sizes():
    assert B.fluxmoe_sorted_rows(100, 8, 160) == 800
    assert B.fluxmoe_sorted_rows(100, 8, 160, 16) == 800 + 160 * 15          # every expert's group can be one row short of a multiple
    assert B.fluxmoe_sorted_rows(1, 10, 512, 16) == 10 + 10 * 15             # ten pairs have ten groups at most
    assert B.fluxmoe_sorted_rows(0, 10, 512, 16) == 0
    assert B.fluxmoe_sort_workspace_bytes(1, 10, 512) == 0
    assert B.fluxmoe_sort_workspace_bytes(1 << 20, 64, 4096) == (1 << 16) * 4096 * 4
    assert B.fluxmoe_block_norm_grad_workspace_bytes(0, 4096) == 0
    one, many = (B.fluxmoe_block_norm_grad_workspace_bytes(T, 4096) for T in (1, 100000))
    assert one == 2 * 4096 * 4 and many >= one


def sort(ids=P, T=4, K=2, E=8, align=1, offsets=P, counts=P, pair_row=P, row_pair=P, cap=8, ws=None, ws_bytes=0):
    B.fluxmoe_sort_tokens(ids, T, K, E, align, offsets, counts, pair_row, row_pair, cap, ws, ws_bytes)


@pytest.mark.parametrize("status,kw", [(-1, dict(T=(1 << 20) + 1)), (-1, dict(E=0)), (-1, dict(E=4097)), (-1, dict(K=0)), (-1, dict(K=65)), (-1, dict(align=0)),
                                       (-1, dict(align=1025)), (-1, dict(ids=None)), (-1, dict(offsets=None)), (-1, dict(counts=None)),
                                       (-1, dict(pair_row=None)), (-1, dict(row_pair=None)), (-1, dict(ids=P + 2)), (-1, dict(cap=1 << 31)),
                                       (-2, dict(cap=7)), (-2, dict(align=2, cap=15)), (-2, dict(T=5000, cap=10000)),
                                       (-2, dict(T=5000, cap=10000, ws=P, ws_bytes=9))])
def test_sort_refuses(status, kw):
    text = refused(status, sort, **kw)
    assert status == -1 or "need" in text


def dispatch(x=P, type_=0, T=4, H=64, xs=64, pair_row=P, K=2, row_pair=P, cap=8, rows=P, rs=64):
    B.fluxmoe_dispatch(x, type_, T, H, xs, pair_row, K, row_pair, cap, rows, rs)


@pytest.mark.parametrize("kw", [dict(type_=3), dict(T=(1 << 20) + 1), dict(H=0), dict(H=(1 << 20) + 1), dict(K=0), dict(K=65), dict(cap=1 << 31), dict(x=None),
                                dict(pair_row=None), dict(row_pair=None), dict(rows=None), dict(xs=63), dict(rs=63), dict(x=P + 1), dict(rows=P + 1),
                                dict(type_=1, x=P + 2)])
def test_dispatch_refuses(kw):
    refused(-1, dispatch, **kw)


def combine(rows=P, rt=0, cap=8, H=64, rs=64, pair_row=P, w=P, T=4, K=2, out=P, ot=1, os=64, flags=0):
    B.fluxmoe_combine(rows, rt, cap, H, rs, pair_row, w, T, K, out, ot, os, flags)


@pytest.mark.parametrize("kw", [dict(rt=2), dict(ot=2), dict(flags=2), dict(rows=None), dict(pair_row=None), dict(out=None), dict(rs=63), dict(os=0),
                                dict(rows=P + 1), dict(out=P + 2), dict(w=P + 2), dict(H=0), dict(K=65), dict(T=1 << 21)])
def test_combine_refuses(kw):
    refused(-1, combine, **kw)


def combine_grad(d=P, ot=1, ds=64, rows=P, rt=0, cap=8, H=64, rs=64, pair_row=P, row_pair=P, w=P, T=4, K=2, dr=P, drs=64, dw=P):
    B.fluxmoe_combine_grad(d, ot, ds, rows, rt, cap, H, rs, pair_row, row_pair, w, T, K, dr, drs, dw)


@pytest.mark.parametrize("kw", [dict(rt=2), dict(ot=2), dict(d=None), dict(rows=None), dict(pair_row=None), dict(row_pair=None), dict(w=None), dict(dr=None),
                                dict(dw=None), dict(ds=63), dict(rs=63), dict(drs=63), dict(d=P + 2), dict(rows=P + 1), dict(dr=P + 1), dict(dw=P + 2)])
def test_combine_grad_refuses(kw):
    refused(-1, combine_grad, **kw)


def desc(**kw):
    fields = dict(hidden=64, y_type=B.F32, residual_type=B.BF16, weight_type=B.BF16, flags=0, eps=1e-6, scale=1.0)
    return ctypes.pointer(B.NormDesc(**dict(fields, **kw)))


def norm(d, T=4, y=P, residual=P, gate=None, w_post=None, w_pre=P, out=P, n=P):
    B.fluxmoe_block_norm(d, T, y, residual, gate, w_post, w_pre, out, n)


def norm_grad(d, T=4, y=P, r=P, gate=None, w_post=None, w_pre=P, do=P, dn=P, dr=P, dy=P, dg=None, dwo=None, dwi=P, ws=P, ws_bytes=1 << 30):
    B.fluxmoe_block_norm_grad(d, T, y, r, gate, w_post, w_pre, do, dn, dr, dy, dg, dwo, dwi, ws, ws_bytes)


BAD_DESCS = [dict(hidden=0), dict(hidden=(1 << 20) + 1), dict(y_type=2), dict(residual_type=9), dict(weight_type=2), dict(flags=16), dict(flags=3),
             dict(flags=1), dict(flags=2), dict(flags=4), dict(eps=-1e-6), dict(eps=float("nan")), dict(y_stride=63), dict(residual_stride=1),
             dict(residual_out_stride=1 << 41), dict(normed_stride=5), dict(d_y_stride=1), dict(d_normed_stride=63)]


@pytest.mark.parametrize("fn", [norm, norm_grad])
@pytest.mark.parametrize("kw", BAD_DESCS)
def test_norm_refuses_descriptions(fn, kw):
    refused(-1, fn, desc(**kw))


@pytest.mark.parametrize("kw", [dict(T=1 << 21), dict(residual=None), dict(w_pre=None), dict(n=None), dict(out=None), dict(y=None), dict(gate=P),
                                dict(y=None, out=None, w_post=P), dict(y=P + 2), dict(residual=P + 1), dict(n=P + 1), dict(out=P + 1), dict(w_pre=P + 1)])
def test_norm_refuses(kw):
    refused(-1, norm, desc(), **kw)
    refused(-1, norm, None)
    refused(-1, norm, desc(residual_out_stride=128))         # in the residual's place with another stride


@pytest.mark.parametrize("status,kw", [(-1, dict(r=None)), (-1, dict(w_pre=None)), (-1, dict(dn=None)), (-1, dict(dr=None)), (-1, dict(dwi=None)), (-1, dict(dy=None)),
                                       (-1, dict(y=None)), (-1, dict(dg=P)), (-1, dict(dwo=P)), (-1, dict(w_post=P)), (-1, dict(dwi=P + 2)),
                                       (-1, dict(ws=P + 8)), (-2, dict(ws=None)), (-2, dict(ws_bytes=100))])
def test_norm_grad_refuses(status, kw):
    refused(status, norm_grad, desc(), **kw)


def test_norm_grad_refuses_another_stride_in_an_inputs_place():
    assert "stride" in refused(-1, norm_grad, desc(d_residual_stride=128))
    assert "stride" in refused(-1, norm_grad, desc(d_y_stride=128), dr=2 * P, do=4 * P)


def test_tensors_are_checked_before_the_library_is_called():
    x = torch.zeros(4, 8)
    for call in (lambda: M.route(x, torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)),
                 lambda: M.sort_tokens(torch.zeros(4, 2, dtype=torch.int32), 8, x, x, x, x),
                 lambda: M.dispatch(x, x, x, x), lambda: M.combine(x, x, None, x),
                 lambda: M.block_norm(x, x[0], x)):
        with pytest.raises(ValueError, match="must be on the current GPU"):
            call()


def test_norm_refuses_a_reserved_field():
    refused(-1, norm, B.NormDesc(64, B.F32, B.F32, B.F32, 0, 1e-6, 1.0, 1))


@pytest.mark.parametrize("rows,fine", [(1, True), (2, False), (4, False)])
def test_rows_that_overlap(rows, fine):
    """The norms' call takes a stride of 0 for the width: a row expanded over the tokens has it, too, and no such rows behind it."""
    expanded = torch.zeros(1, 8).expand(rows, 8)
    if fine:
        assert M._matrix(expanded, "y", rows, 8, -1) == 8
    else:
        for t in (expanded, torch.zeros(64).as_strided((rows, 8), (4, 1))):
            with pytest.raises(ValueError, match="overlap"):
                M._matrix(t, "y", rows, 8, -1)
