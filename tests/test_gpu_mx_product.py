"""Products with experts' weights in 4 bits, and their gradient, against 64 bits: one row to many, experts without rows, groups with gaps,
widths that are not whole tiles, strides, NaN in rows that are not theirs, counts that do not fit the matrix, places past 32 bits.

Tolerance: the terms are exact in FP32, a sum of K of them is off by at most K u of the sum of their magnitudes (u = 2^-23, as the
matrix instructions may cut instead of round), and an output by half a step of its type, eps / 2 of itself."""
import math

import pytest
import torch

from paper_2604_02715_amd import mx_experts as X
from tests import mx_plain as plain

pytestmark = pytest.mark.gpu
U = 2.0 ** -23
BF16, F32 = torch.bfloat16, torch.float32


def near(got, want, size, terms):
    """rows of no expert (NaN in `want`) still hold what was there"""
    eps = torch.finfo(got.dtype).eps / 2
    got = got.cpu().double()
    rows = torch.isnan(want).all(dim=1)
    assert bool((got[rows] == 7.0).all())
    got, want, size = got[~rows], want[~rows], size[~rows]
    far = (got - want).abs() - (eps * want.abs() + terms * U * size * (1 + eps) + 1e-37)
    assert got.numel() == 0 or float(far.max()) <= 0, float(far.max())


def rows_in(n, K, mx, seed, scale=1.0):
    """(rows, row_scales or None, their values in 64 bits)"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = scale * torch.randn(n, K, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(K, generator=g, device="cuda"))
    if not mx:
        x = x.to(BF16)
        return x, None, x.cpu().double()
    codes = torch.empty(n, K // 2, dtype=torch.uint8, device="cuda")
    scales = torch.empty(n, K // 32, dtype=torch.uint8, device="cuda")
    X.quantize(x, codes, scales)
    return codes, scales, plain.values(codes, scales)


def check(counts, N, K, mx, out_type, align=1, ahead=0, behind=0, seed=0):
    offsets, n_rows, n = plain.groups(counts, align, ahead)
    n += behind
    wc, ws = plain.random_weights(len(counts), N, K, seed + N)
    x, xs, x64 = rows_in(n, K, mx, seed + K)
    out = torch.full((n, N), 7.0, dtype=out_type, device="cuda")
    X.product(x, offsets, n_rows, wc, ws, out, row_scales=xs)
    near(out, *plain.products(x64, offsets, n_rows, plain.values(wc, ws)), K)
    again = torch.full_like(out, 7.0)
    X.product(x, offsets, n_rows, wc, ws, again, row_scales=xs)
    assert torch.equal(again, out)


def check_grad(counts, N, K, out_type, align=1, ahead=0, behind=0, seed=0):
    offsets, n_rows, n = plain.groups(counts, align, ahead)
    n += behind
    wc, ws = plain.random_weights(len(counts), N, K, seed + N)
    d, _, d64 = rows_in(n, N, False, seed + K)
    back = torch.full((n, K), 7.0, dtype=out_type, device="cuda")
    X.product_grad(d, offsets, n_rows, wc, ws, back)
    near(back, *plain.products(d64, offsets, n_rows, plain.values(wc, ws), transposed=True), N)
    again = torch.full_like(back, 7.0)
    X.product_grad(d, offsets, n_rows, wc, ws, again)
    assert torch.equal(again, back)


GROUPS = [[1], [0, 0, 1, 0], [2, 0, 1], [16], [17, 15], [33, 1, 0, 64], [5] * 70, [130, 3], [257, 255, 0, 1], [0, 400], [3] * 300 + [40]]
WIDTHS = [(1, 32), (16, 32), (7, 96), (64, 128), (130, 160), (65, 512), (257, 288), (300, 1056)]


@pytest.mark.parametrize("out_type", [BF16, F32])
@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("counts", GROUPS, ids=lambda c: "%dx%d" % (len(c), max(c)))
def test_groups(counts, mx, out_type):
    check(counts, 72, 224, mx, out_type, behind=3)


@pytest.mark.parametrize("out_type", [BF16, F32])
@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("N,K", WIDTHS)
def test_widths(N, K, mx, out_type):
    check([3, 0, 20], N, K, mx, out_type)
    check([300, 1, 70], N, K, mx, out_type)


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("counts,align,ahead,behind", [([5, 0, 17, 1], 16, 0, 0), ([5, 90, 1], 8, 3, 9), ([1, 1, 1], 64, 1, 1)])
def test_rows_of_no_expert_are_left(counts, align, ahead, behind, mx):
    check(counts, 40, 128, mx, F32, align, ahead, behind)
    check_grad(counts, 40, 128, F32, align, ahead, behind)


@pytest.mark.parametrize("counts,N,K,mx", [([1, 0, 1], 1024, 2048, False), ([1, 0, 1], 1024, 2048, True), ([520], 768, 1024, False), ([520], 768, 1024, True),
                                           ([200, 312], 512, 2048, True), ([700], 260, 4128, False), ([64, 64], 96, 8192, True)])
def test_larger(counts, N, K, mx):
    check(counts, N, K, mx, BF16)


@pytest.mark.parametrize("out_type", [BF16, F32])
@pytest.mark.parametrize("counts", GROUPS, ids=lambda c: "%dx%d" % (len(c), max(c)))
def test_gradient_groups(counts, out_type):
    check_grad(counts, 72, 224, out_type, behind=3)


@pytest.mark.parametrize("out_type", [BF16, F32])
@pytest.mark.parametrize("N,K", WIDTHS)
def test_gradient_widths(N, K, out_type):
    check_grad([3, 0, 20], N, K, out_type)
    check_grad([300, 1, 70], N, K, out_type)


@pytest.mark.parametrize("counts,N,K", [([1, 0, 1], 2048, 512), ([520], 1024, 768), ([200, 312], 2048, 512), ([700], 4099, 288)])
def test_gradient_larger(counts, N, K):
    check_grad(counts, N, K, BF16)


def test_gradient_against_differences():
    """<d_out, product> is linear in the rows: its difference along a step is the gradient's product with the step"""
    offsets, counts, n = plain.groups([3, 0, 9])
    wc, ws = plain.random_weights(3, 48, 96, 1)
    d, _, d64 = rows_in(n, 48, False, 2)
    back = torch.empty(n, 96, device="cuda")
    X.product_grad(d, offsets, counts, wc, ws, back)
    for row, col in [(0, 0), (2, 95), (3, 1), (11, 40)]:
        x = torch.zeros(n, 96, dtype=BF16, device="cuda")
        x[row, col] = 1.0
        out = torch.zeros(n, 48, device="cuda")
        X.product(x, offsets, counts, wc, ws, out)
        want = float((out.cpu().double() * d64).sum())
        assert abs(float(back[row, col]) - want) <= 48 * U * float((out.cpu().double() * d64).abs().sum()) * 2


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("counts", [[4, 9], [150, 70]])
@pytest.mark.parametrize("gap,shift", [(16, 0), (1, 0), (0, 1), (7, 5)])
def test_strides(counts, gap, shift, mx):
    offsets, n_rows, n = plain.groups(counts)
    N, K = 88, 160
    wc, ws = plain.random_weights(2, N, K, 3)
    x, xs, _ = rows_in(n, K, mx, 4)

    def place(t, fill=7):
        whole = torch.full((n * (t.shape[1] + gap) + shift,), fill, dtype=t.dtype, device="cuda")
        view = whole[shift:].view(n, t.shape[1] + gap)[:, :t.shape[1]]
        view.copy_(t)
        return whole, view

    want = torch.zeros(n, N, dtype=BF16, device="cuda")
    X.product(x, offsets, n_rows, wc, ws, want, row_scales=xs)
    whole, out = place(torch.zeros_like(want))
    X.product(place(x)[1], offsets, n_rows, wc, ws, out, row_scales=None if xs is None else place(xs)[1])
    # the kernels for rows elsewhere may add up in another order: both are within the bound, a BF16 step apart at most
    assert torch.allclose(out.float(), want.float(), rtol=2.0 ** -7, atol=1e-4)
    out.fill_(7)
    assert bool((whole == 7).all())
    if not mx:
        want = torch.zeros(n, K, dtype=BF16, device="cuda")
        d = rows_in(n, N, False, 5)[0]
        X.product_grad(d, offsets, n_rows, wc, ws, want)
        whole, back = place(torch.zeros_like(want))
        X.product_grad(place(d)[1], offsets, n_rows, wc, ws, back)
        assert torch.allclose(back.float(), want.float(), rtol=2.0 ** -7, atol=1e-4)
        back.fill_(7)
        assert bool((whole == 7).all())


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("counts", [[3, 20, 5], [70, 20, 150]])
def test_nan_stays_with_its_row(counts, mx):
    """NaN in rows between the groups, in one row of a group, and in one output's weights"""
    offsets, n_rows, n = plain.groups(counts, align=16, ahead=2)
    N, K = 80, 192
    wc, ws = plain.random_weights(3, N, K, 6)
    x, xs, _ = rows_in(n, K, mx, 7)
    clean, out = torch.full((n, N), 7.0, device="cuda"), torch.full((n, N), 7.0, device="cuda")
    X.product(x, offsets, n_rows, wc, ws, clean, row_scales=xs)
    hit = torch.ones(n, dtype=torch.bool)
    for o, c in zip(offsets.tolist(), counts):
        hit[o:o + c] = False
    bad = int(offsets[1]) + 1
    hit[bad] = True
    if mx:
        xs[hit.cuda(), K // 32 - 1] = 255
    else:
        x[hit.cuda(), K - 1] = math.nan
    ws[2, 5, 3] = 255
    X.product(x, offsets, n_rows, wc, ws, out, row_scales=xs)
    o2, c2 = int(offsets[2]), counts[2]
    want = torch.zeros(n, N, dtype=torch.bool)
    want[bad], want[o2:o2 + c2, 5] = True, True
    assert torch.equal(torch.isnan(out).cpu(), want)
    assert torch.equal(out[~want.cuda()], clean[~want.cuda()])
    if not mx:
        d = torch.randn(n, N, device="cuda").to(BF16)
        clean, back = torch.full((n, K), 7.0, device="cuda"), torch.full((n, K), 7.0, device="cuda")
        ws[2, 5, 3] = 120
        X.product_grad(d, offsets, n_rows, wc, ws, clean)
        d[hit.cuda(), N - 1] = math.nan
        ws[2, 5, 3] = 255
        X.product_grad(d, offsets, n_rows, wc, ws, back)
        want = torch.zeros(n, K, dtype=torch.bool)
        want[bad], want[o2:o2 + c2, 96:128] = True, True
        assert torch.equal(torch.isnan(back).cpu(), want)
        assert torch.equal(back[~want.cuda()], clean[~want.cuda()])


@pytest.mark.parametrize("mx", [False, True])
def test_counts_that_do_not_fit_the_matrix(mx):
    """what lies outside is not done, and nothing outside is touched"""
    n, N, K = 40, 24, 64
    wc, ws = plain.random_weights(5, N, K, 8)
    x, xs, x64 = rows_in(n, K, mx, 9)
    i32 = dict(dtype=torch.int32, device="cuda")
    offsets, counts = torch.tensor([0, -5, 38, 40, 1 << 30, 3], **i32), torch.tensor([3, 4, 1000, 5, 2 ** 31 - 1], **i32)
    whole = torch.full((n + 64, N), 7.0, device="cuda")
    X.product(x, offsets, counts, wc, ws, whole[32:32 + n], row_scales=xs)
    done = torch.zeros(n + 64, dtype=torch.bool)
    done[32:35], done[70:72] = True, True
    assert bool((whole[~done.cuda()] == 7.0).all()) and not bool((whole[done.cuda()] == 7.0).any())
    counts[:] = -1
    again = torch.full((n, N), 7.0, device="cuda")
    X.product(x, offsets, counts, wc, ws, again, row_scales=xs)
    assert bool((again == 7.0).all())


def test_no_rows_at_all():
    wc, ws = plain.random_weights(2, 8, 32, 1)
    zero = torch.zeros(3, dtype=torch.int32, device="cuda")
    X.product(torch.empty(0, 32, dtype=BF16, device="cuda"), zero, zero[:2], wc, ws, torch.empty(0, 8, device="cuda"))
    X.product_grad(torch.empty(0, 8, dtype=BF16, device="cuda"), zero, zero[:2], wc, ws, torch.empty(0, 32, device="cuda"))
    out = torch.full((5, 8), 7.0, device="cuda")
    X.product(torch.zeros(5, 32, dtype=BF16, device="cuda"), zero, zero[:2], wc, ws, out)
    assert bool((out == 7.0).all())


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("count", [2, 200])
def test_places_past_32_bits(count, mx):
    """the last expert's weights begin 4.5 GB into the codes, the last rows 4.3 GB into rows and outputs"""
    E, N, K = 41, 16384, 14336
    wc = torch.zeros(E, N, K // 2, dtype=torch.uint8, device="cuda")
    ws = torch.zeros(E, N, K // 32, dtype=torch.uint8, device="cuda")
    wc[-1], ws[-1] = (t[0] for t in plain.random_weights(1, N, K, 3))
    n, stride = 2 ** 17, 2 ** 14 if not mx else 2 ** 15
    x_all = torch.zeros(n * stride + K, dtype=torch.uint8 if mx else BF16, device="cuda")
    x = x_all[:n * stride].view(n, stride)[:, :K // 2 if mx else K]
    small, xs, x64 = rows_in(count, K, mx, 4)
    x[-count:] = small
    scales = None
    if mx:
        scales = torch.zeros(n, K // 32, dtype=torch.uint8, device="cuda")
        scales[-count:] = xs
    offsets = torch.full((E + 1,), n - count, dtype=torch.int32, device="cuda")
    offsets[-1] = n
    counts = torch.zeros(E, dtype=torch.int32, device="cuda")
    counts[-1] = count
    out = torch.full((n, N), 7.0, dtype=BF16, device="cuda")
    X.product(x, offsets, counts, wc, ws, out, row_scales=scales)
    few = torch.arange(0, N, 257)
    w = plain.values(wc[-1][few.cuda()], ws[-1][few.cuda()])
    got = out[-count:][:, few.cuda()].cpu().double()
    want, size = x64 @ w.t(), x64.abs() @ w.abs().t()
    assert bool(((got - want).abs() <= 2.0 ** -8 * want.abs() + K * U * size).all())
    assert bool((out[:-count] == 7.0).all())
    if not mx:
        d = torch.zeros(n, N, dtype=BF16, device="cuda")
        d[-count:] = rows_in(count, N, False, 5)[0]
        out = x.fill_(7.0)                                   # [n][K], 2^14 apart
        X.product_grad(d, offsets, counts, wc, ws, out)
        w, d64 = plain.values(wc[-1], ws[-1])[:, :96], d[-count:].cpu().double()
        got, want, size = out[-count:, :96].cpu().double(), d64 @ w, d64.abs() @ w.abs()
        assert bool(((got - want).abs() <= 2.0 ** -8 * want.abs() + N * U * size).all())
        assert bool((out[:-count] == 7.0).all())


@pytest.mark.parametrize("mx", [False, True])
def test_rows_far_apart(mx):
    """rows more than 4 GB apart, places that no 32 bits hold within a tile"""
    n, N, K, stride = 3, 40, 64, (1 << 32) + 16 if mx else (1 << 31) + 8
    offsets, counts, _ = plain.groups([1, 2])
    wc, ws = plain.random_weights(2, N, K, 1)
    x, xs, x64 = rows_in(n, K, mx, 2)
    far = torch.empty((n - 1) * stride + K, dtype=x.dtype, device="cuda").as_strided((n, x.shape[1]), (stride, 1))
    far.copy_(x)
    if mx:
        scales = torch.empty((n - 1) * ((1 << 31) + 4) + 4, dtype=torch.uint8, device="cuda").as_strided((n, K // 32), ((1 << 31) + 4, 1))
        scales.copy_(xs)
        xs = scales
    out = torch.full((n, N), 7.0, device="cuda")
    X.product(far, offsets, counts, wc, ws, out, row_scales=xs)
    near(out, *plain.products(x64, offsets, counts, plain.values(wc, ws)), K)
    if not mx:
        d, _, d64 = rows_in(n, N, False, 3)
        whole = torch.full(((n - 1) * stride + K,), 7.0, dtype=BF16, device="cuda")
        back = whole.as_strided((n, K), (stride, 1))
        X.product_grad(d, offsets, counts, wc, ws, back)
        near(back, *plain.products(d64, offsets, counts, plain.values(wc, ws), transposed=True), N)
        far = whole.as_strided((n, N), (stride, 1))
        far.copy_(d)
        back = torch.full((n, K), 7.0, device="cuda")
        X.product_grad(far, offsets, counts, wc, ws, back)
        near(back, *plain.products(d64, offsets, counts, plain.values(wc, ws), transposed=True), N)


@pytest.mark.parametrize("mx", [False, True])
def test_most_experts(mx):
    counts = [0] * 4096
    for e, c in ((0, 1), (15, 2), (16, 17), (1000, 1), (1001, 3), (4095, 5)):
        counts[e] = c
    check(counts, 24, 64, mx, F32)
    check_grad(counts, 24, 64, F32)


def test_other_stream():
    offsets, counts, n = plain.groups([5, 60])
    wc, ws = plain.random_weights(2, 64, 128, 1)
    x = rows_in(n, 128, False, 2)[0]
    want, out = torch.zeros(n, 64, device="cuda"), torch.zeros(n, 64, device="cuda")
    X.product(x, offsets, counts, wc, ws, want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    X.product(x, offsets, counts, wc, ws, out, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(out, want)
