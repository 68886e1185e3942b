"""Host side of the experts in 4-bit floating point and of routing within groups: what the calls refuse.  Nothing is launched: every call
here is turned down before that, or has nothing to do."""
import ctypes

import pytest
import torch

from paper_2604_02715_amd import binding as B
from paper_2604_02715_amd import moe_block as M
from paper_2604_02715_amd import mx_experts as X

P = 1 << 20                     # stands for a device address; no accepted call reaches it
BIG = (1 << 32) + 32


def refused(fn, *args, **kw):
    with pytest.raises(B.FluxmoeError) as e:
        fn(*args, **kw)
    assert e.value.status == -1, str(e.value)
    return str(e.value)


def route(logits=P, type_=B.F32, T=4, E=32, stride=32, bias=None, K=4, groups=4, top_groups=2, scale=1.0, flags=0, ids=P, w=P):
    B.fluxmoe_route_grouped(logits, type_, T, E, stride, bias, K, groups, top_groups, scale, flags, ids, w)


@pytest.mark.parametrize("kw", [dict(groups=0), dict(groups=5), dict(groups=33), dict(E=4096, stride=4096, groups=128), dict(top_groups=0), dict(top_groups=5),
                                dict(K=17), dict(flags=B.ROUTE_GROUP_TOP2), dict(flags=8), dict(bias=P), dict(type_=2), dict(T=(1 << 20) + 1), dict(K=0),
                                dict(logits=None), dict(ids=None), dict(w=None), dict(stride=31), dict(w=P + 2)])
def test_route_refuses(kw):
    refused(route, **kw)


def test_the_flag_of_groups_is_not_the_plain_routers():
    refused(B.fluxmoe_route, P, B.F32, 4, 32, 32, None, 4, 1.0, B.ROUTE_SIGMOID | B.ROUTE_GROUP_TOP2, P, P)


def quantize(x=P, type_=B.BF16, rows=4, columns=64, xs=64, codes=P, cs=32, scales=P, ss=2):
    B.fluxmoe_mx_quantize(x, type_, rows, columns, xs, codes, cs, scales, ss)


def dequantize(x=P, type_=B.BF16, rows=4, columns=64, xs=64, codes=P, cs=32, scales=P, ss=2):
    B.fluxmoe_mx_dequantize(codes, cs, scales, ss, rows, columns, x, type_, xs)


@pytest.mark.parametrize("fn", [quantize, dequantize])
@pytest.mark.parametrize("kw", [dict(type_=2), dict(columns=0), dict(columns=48), dict(columns=(1 << 20) + 32, xs=1 << 21, cs=1 << 20, ss=1 << 16),
                                dict(rows=(1 << 32) + 1), dict(xs=63), dict(cs=31), dict(ss=1), dict(xs=1 << 40), dict(x=None), dict(codes=None),
                                dict(scales=None), dict(x=P + 1), dict(type_=B.F32, x=P + 2)])
def test_rows_refuse(fn, kw):
    refused(fn, **kw)


def product(E=3, N=16, K=64, rows_type=B.BF16, out_type=B.F32, reserved=0, cap=8, rs=0, ss=0, os=0, rows=P, row_scales=None, offsets=P, counts=P,
            codes=P, scales=P, out=P, desc=True):
    d = ctypes.pointer(B.MxProductDesc(E, N, K, rows_type, out_type, reserved, cap, rs, ss, os)) if desc else None
    B.fluxmoe_mx_product(d, rows, row_scales, offsets, counts, codes, scales, out)


def grad(E=3, N=16, K=64, rows_type=B.F32, out_type=B.BF16, reserved=0, cap=8, rs=0, ss=0, os=0, rows=P, offsets=P, counts=P, codes=P, scales=P,
         out=P, desc=True):
    d = ctypes.pointer(B.MxProductDesc(E, N, K, rows_type, out_type, reserved, cap, rs, ss, os)) if desc else None
    B.fluxmoe_mx_product_grad(d, out, offsets, counts, codes, scales, rows)


BAD = [dict(E=0), dict(E=4097), dict(N=0), dict(N=(1 << 20) + 1), dict(K=0), dict(K=80), dict(K=(1 << 20) + 32), dict(reserved=1), dict(cap=1 << 31), dict(rs=63),
       dict(os=15), dict(os=1 << 40), dict(rows=None), dict(out=None), dict(offsets=None), dict(counts=None), dict(codes=None), dict(scales=None),
       dict(rows=P + 1), dict(out=P + 1), dict(offsets=P + 2), dict(counts=P + 2), dict(codes=P + 8), dict(desc=False)]


@pytest.mark.parametrize("kw", BAD + [dict(rows_type=B.F32), dict(out_type=B.MXFP4), dict(row_scales=P), dict(rows_type=B.MXFP4),
                                      dict(rows_type=B.MXFP4, row_scales=P, rs=31), dict(rows_type=B.MXFP4, row_scales=P, ss=1), dict(rows_type=3)])
def test_product_refuses(kw):
    refused(product, **kw)


@pytest.mark.parametrize("kw", BAD + [dict(rows_type=B.MXFP4), dict(out_type=B.F32), dict(rows_type=3)])
def test_product_grad_refuses(kw):
    refused(grad, **kw)


def swiglu(x=P, type_=B.BF16, rows=4, F=64, xs=128, h=P, h_type=B.BF16, hs=64):
    B.fluxmoe_swiglu(x, type_, rows, F, xs, h, h_type, hs)


def swiglu_grad(x=P, type_=B.BF16, rows=4, F=64, xs=128, h=P, h_type=B.BF16, hs=64, d=P, ds=128):
    B.fluxmoe_swiglu_grad(x, type_, rows, F, xs, h, h_type, hs, d, ds)


@pytest.mark.parametrize("kw", [dict(type_=2), dict(h_type=2), dict(rows=1 << 31), dict(F=0), dict(F=(1 << 20) + 1, xs=1 << 22, hs=1 << 21), dict(xs=127),
                                dict(hs=63), dict(x=None), dict(h=None), dict(x=P + 1), dict(h_type=B.F32, h=P + 2)])
def test_swiglu_refuses(kw):
    refused(swiglu, **kw)
    refused(swiglu_grad, **kw)


@pytest.mark.parametrize("kw", [dict(d=None), dict(ds=127), dict(d=P + 1)])
def test_swiglu_grad_refuses(kw):
    refused(swiglu_grad, **kw)


def test_no_rows_are_no_work():
    route(T=0, logits=None, ids=None, w=None)
    quantize(rows=0, x=None, codes=None, scales=None)
    dequantize(rows=0, x=None, codes=None, scales=None)
    product(cap=0, rows=None, out=None)
    grad(cap=0, rows=None, out=None)
    swiglu(rows=0, x=None, h=None)
    swiglu_grad(rows=0, x=None, h=None, d=None)


# ---------------------------------------------------------------- on tensors
@pytest.fixture
def on_the_gpu(monkeypatch):
    """what is looked at behind the tensors' place"""
    monkeypatch.setattr(X, "_place", lambda t, name: -1)
    monkeypatch.setattr(M, "_place", lambda t, name: -1)


def u8(*shape):
    return torch.zeros(*shape, dtype=torch.uint8)


def test_tensors_of_the_cpu_are_refused():
    x = torch.zeros(2, 64)
    with pytest.raises((ValueError, RuntimeError)):
        X.quantize(x, u8(2, 32), u8(2, 2))


@pytest.mark.parametrize("x,codes,scales", [((2, 48), (2, 24), (2, 1)), ((2, 64), (3, 32), (2, 2)), ((2, 64), (2, 32), (1, 2)), ((2, 64), (2, 31), (2, 2)),
                                            ((2, 64), (2, 32), (2, 3)), ((64,), (32,), (2,))])
def test_quantize_shapes(on_the_gpu, x, codes, scales):
    for call in (lambda: X.quantize(torch.zeros(x), u8(codes), u8(scales)), lambda: X.dequantize(u8(codes), u8(scales), torch.zeros(x))):
        with pytest.raises(ValueError):
            call()


def test_quantize_types_and_gaps(on_the_gpu):
    for x, codes, scales in ((torch.zeros(2, 64, dtype=torch.float16), u8(2, 32), u8(2, 2)), (torch.zeros(2, 64), u8(2, 32).int(), u8(2, 2)),
                             (torch.zeros(2, 64), u8(2, 32), u8(2, 2).float()), (torch.zeros(2, 128)[:, ::2], u8(2, 32), u8(2, 2)),
                             (torch.zeros(2, 3, 128)[..., :64], u8(2, 3, 32), u8(2, 3, 2)), (torch.zeros(1, 64).expand(2, 64), u8(2, 32), u8(2, 2))):
        with pytest.raises(ValueError):
            X.quantize(x, codes, scales)


def operands(E=2, N=16, K=64, n=4):
    i32 = torch.int32
    return dict(rows=torch.zeros(n, K, dtype=torch.bfloat16), offsets=torch.zeros(E + 1, dtype=i32), counts=torch.zeros(E, dtype=i32), w_codes=u8(E, N, K // 2),
                w_scales=u8(E, N, K // 32), out=torch.zeros(n, N))


@pytest.mark.parametrize("kw", [dict(rows=torch.zeros(4, 64)), dict(rows=torch.zeros(4, 32, dtype=torch.bfloat16)), dict(offsets=torch.zeros(2, dtype=torch.int32)),
                                dict(counts=torch.zeros(3, dtype=torch.int32)), dict(counts=torch.zeros(2)), dict(w_codes=u8(2, 16, 24)), dict(w_codes=u8(16, 32)),
                                dict(w_codes=u8(2, 16, 64)[..., ::2]), dict(w_scales=u8(2, 16, 1)), dict(out=torch.zeros(3, 16)), dict(out=torch.zeros(4, 17)),
                                dict(out=torch.zeros(4, 16, dtype=torch.float16)), dict(row_scales=u8(4, 2)), dict(rows=u8(4, 32), row_scales=u8(4, 3)),
                                dict(rows=u8(4, 32), row_scales=u8(3, 2))])
def test_product_tensors(on_the_gpu, kw):
    with pytest.raises(ValueError):
        X.product(**{**operands(), **kw})


@pytest.mark.parametrize("kw", [dict(d_out=torch.zeros(4, 16)), dict(d_out=torch.zeros(4, 15, dtype=torch.bfloat16)), dict(d_rows=torch.zeros(4, 32)),
                                dict(d_rows=torch.zeros(5, 64)), dict(d_rows=torch.zeros(4, 64, dtype=torch.float16)), dict(w_scales=u8(2, 16, 3))])
def test_product_grad_tensors(on_the_gpu, kw):
    o = operands()
    o = dict(d_out=o["out"].bfloat16(), offsets=o["offsets"], counts=o["counts"], w_codes=o["w_codes"], w_scales=o["w_scales"], d_rows=torch.zeros(4, 64))
    with pytest.raises(ValueError):
        X.product_grad(**{**o, **kw})


@pytest.mark.parametrize("x,h", [((4, 64), (4, 33)), ((4, 64), (3, 32)), ((4, 64), (32,))])
def test_swiglu_tensors(on_the_gpu, x, h):
    with pytest.raises(ValueError):
        X.swiglu(torch.zeros(x), torch.zeros(h))
    with pytest.raises(ValueError):
        X.swiglu_grad(torch.zeros(x), torch.zeros(h), torch.zeros(x))
    with pytest.raises(ValueError):
        X.swiglu_grad(torch.zeros(4, 64), torch.zeros(4, 32), torch.zeros(4, 64, dtype=torch.bfloat16))


def test_sizes_past_32_bits(on_the_gpu):
    big = lambda *s: u8(*[1 for _ in s]).expand(*s)
    with pytest.raises(ValueError, match="2\\^32"):
        X.quantize(big(2, BIG), big(2, BIG // 2), big(2, BIG // 32))
    o = operands()
    for codes in (big(BIG, 16, 32), big(2, BIG, 32), big(2, 16, BIG // 2)):
        with pytest.raises(ValueError, match="2\\^32"):
            X.product(**{**o, "w_codes": codes})
    with pytest.raises(ValueError, match="2\\^32"):
        X.swiglu(big(2, BIG), big(2, BIG // 2))
    logits, ids, gates = torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2)
    for kw in (dict(groups=BIG), dict(groups=2, top_groups=BIG), dict(groups=-1)):
        with pytest.raises(ValueError, match="2\\^32"):
            M.route(logits, ids, gates, **kw)
    with pytest.raises(ValueError, match="group_score"):
        M.route(logits, ids, gates, group_score="sum")
