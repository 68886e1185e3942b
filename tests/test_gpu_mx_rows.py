"""Rows to 4-bit floating point and back against the definition in 64 bits, bit by bit: ties, saturation, every scale, subnormal numbers,
blocks with infinities and NaN, widths from one block on, strides, other dimensions."""
import math

import pytest
import torch

from paper_2604_02715_amd import mx_experts as X
from tests import mx_plain as plain

pytestmark = pytest.mark.gpu


def quantized(x, codes=None, scales=None):
    u8 = dict(dtype=torch.uint8, device="cuda")
    if codes is None:
        codes = torch.full((*x.shape[:-1], x.shape[-1] // 2), 0xEE, **u8)
        scales = torch.full((*x.shape[:-1], x.shape[-1] // 32), 0xEE, **u8)
    X.quantize(x, codes, scales)
    torch.cuda.synchronize()
    return codes, scales


def check(x_cpu, x_gpu):
    codes, scales = quantized(x_gpu)
    want_codes, want_scales = plain.quantize(x_cpu)
    assert torch.equal(scales.cpu(), want_scales)
    assert torch.equal(codes.cpu(), want_codes)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("R,C", [(1, 32), (3, 32), (1, 64), (5, 96), (7, 160), (2, 2048), (3, 2080), (1, 5120), (65, 1536), (300, 256)])
def test_random_rows(R, C, dtype):
    g = torch.Generator().manual_seed(R * C)
    x = (torch.randn(R, C, generator=g) * torch.exp2(torch.randint(-9, 9, (R, C // 32), generator=g).float()).repeat_interleave(32, 1)).to(dtype)
    x[0, :32] = 0.0
    check(x, x.cuda())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_every_border_at_every_scale(dtype):
    """All numbers n / 16 up to 8, the numbers next to them and their negatives, at each power of two of the type, a block's largest being
    4, 6, or 7.75 times the scale; powers below the smallest scale and subnormal numbers among them."""
    grid = torch.arange(0, 128, dtype=torch.float64) / 16
    grid = torch.cat([grid, -grid])
    rows = []
    for e in range(-133 if dtype == torch.bfloat16 else -149, 126):
        for top in (4.0, 6.0, 7.75):
            v = (grid[grid.abs() <= top] * 2.0 ** e).to(dtype)
            if dtype == torch.float32:
                inf = torch.tensor(math.inf)
                v = torch.cat([v, torch.nextafter(v, inf), torch.nextafter(v, -inf)])
            v = v[torch.isfinite(v) & (v.double().abs() <= top * 2.0 ** e)]
            n = -(-v.numel() // 31) * 31
            v = torch.cat([v, v.new_zeros(n - v.numel())]).view(-1, 31)
            rows.append(torch.cat([v, torch.full((v.shape[0], 1), top * 2.0 ** e, dtype=torch.float64).to(dtype)], dim=1))
    x = torch.cat(rows)
    x = x[torch.isfinite(x).all(dim=1)]
    check(x, x.cuda())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_infinities_and_nan_take_their_block_alone(dtype):
    x = torch.randn(4, 128, generator=torch.Generator().manual_seed(2)).to(dtype)
    x[0, 3], x[1, 40], x[2, 70], x[3, 127] = math.inf, -math.inf, math.nan, -math.nan
    codes, scales = quantized(x.cuda())
    assert scales.cpu().eq(255).nonzero().tolist() == [[0, 0], [1, 1], [2, 2], [3, 3]]
    check(x, x.cuda())
    out = torch.empty(4, 128, dtype=dtype, device="cuda")
    X.dequantize(codes, scales, out)
    assert torch.isnan(out).sum(dim=1).tolist() == [32] * 4


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_every_code_at_every_scale_comes_back(dtype):
    codes = torch.arange(256, dtype=torch.uint8).view(1, 16, 16).expand(256, 16, 16).reshape(256 * 16, 16).contiguous()
    scales = torch.arange(256, dtype=torch.uint8)[:, None].expand(256, 16).reshape(-1, 1).contiguous()
    out = torch.empty(256 * 16, 32, dtype=dtype, device="cuda")
    X.dequantize(codes.cuda(), scales.cuda(), out)
    want = plain.values(codes, scales).to(dtype)
    got = out.cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0))
    assert torch.equal(torch.signbit(got[:4080]), torch.signbit(want[:4080]))        # of zeros, too


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("R,C", [(1, 32), (5, 96), (33, 160), (2, 5120), (3, 14336)])
def test_codes_come_back_as_numbers(R, C, dtype):
    codes, scales = plain.random_weights(1, R, C, R + C)
    codes, scales = codes[0], scales[0]
    out = torch.full((R, C), math.nan, dtype=dtype, device="cuda")
    X.dequantize(codes, scales, out)
    assert torch.equal(out.cpu().double(), plain.values(codes, scales))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("x_gap,x_shift,c_gap,c_shift,s_gap,s_shift", [(8, 0, 4, 0, 3, 0), (1, 0, 1, 0, 1, 1), (0, 1, 0, 0, 0, 0), (0, 0, 0, 3, 0, 0),
                                                                       (64, 8, 16, 4, 0, 2)])
def test_strides_leave_what_lies_between(dtype, x_gap, x_shift, c_gap, c_shift, s_gap, s_shift):
    R, C = 9, 224

    def place(width, gap, shift, t, fill):
        whole = torch.full((R * (width + gap) + shift + 16,), fill, dtype=t, device="cuda")
        return whole, whole[shift:shift + R * (width + gap)].view(R, width + gap)[:, :width]

    _, x = place(C, x_gap, x_shift, dtype, 7.0)
    x.copy_(torch.randn(R, C, generator=torch.Generator().manual_seed(4)))
    codes_all, codes = place(C // 2, c_gap, c_shift, torch.uint8, 0xEE)
    scales_all, scales = place(C // 32, s_gap, s_shift, torch.uint8, 0xEE)
    quantized(x, codes, scales)
    want_codes, want_scales = plain.quantize(x)
    assert torch.equal(codes.cpu(), want_codes) and torch.equal(scales.cpu(), want_scales)
    out_all, out = place(C, x_gap, x_shift, dtype, 7.0)
    X.dequantize(codes, scales, out)
    assert torch.equal(out.cpu().double(), plain.values(want_codes, want_scales))
    codes.fill_(0xEE), scales.fill_(0xEE), out.fill_(7.0)
    assert bool((codes_all == 0xEE).all()) and bool((scales_all == 0xEE).all()) and bool((out_all == 7.0).all())


def test_all_experts_at_once_and_no_rows():
    x = torch.randn(3, 7, 64, device="cuda")
    codes, scales = quantized(x)
    assert codes.shape == (3, 7, 32) and torch.equal(codes.cpu(), plain.quantize(x)[0])
    back = torch.empty_like(x)
    X.dequantize(codes, scales, back)
    assert torch.equal(back.cpu().double(), plain.values(codes, scales))
    quantized(torch.empty(0, 64, device="cuda"))


def test_long_rows_past_32_bits():
    """2^31 + 2^21 numbers: places past 32 bits in bytes of every matrix but the codes'"""
    R, C = 2049, 1 << 20
    x = torch.zeros(R, C, dtype=torch.bfloat16, device="cuda")
    x[0, :32], x[-1, -32:] = torch.arange(32), torch.arange(32) * 0.25
    codes, scales = quantized(x)
    assert torch.equal(codes[-1, -16:].cpu(), plain.quantize(x[-1:, -32:])[0][0])
    assert torch.equal(codes[0, :16].cpu(), plain.quantize(x[:1, :32])[0][0])
    assert int(codes.count_nonzero()) == int(codes[0, :16].count_nonzero()) + int(codes[-1, -16:].count_nonzero())
    X.dequantize(codes, scales, x)
    assert torch.equal(x[-1, -32:].cpu().double(), plain.values(codes[-1:, -16:], scales[-1:, -1:])[0])
