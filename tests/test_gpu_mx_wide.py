"""Products with experts' weights in 4 bits, and their gradient, where calls are large enough for the wide tiles: tiles of 128 and 256 rows,
the ends of superblocks and of tiles, rows at any address, experts without rows, NaN in rows and weights, against 64 bits on a sample of
the outputs.  Tolerances as in the tests of small calls."""
import math

import pytest
import torch

from paper_2604_02715_amd import mx_experts as X
from tests import mx_plain as plain

pytestmark = pytest.mark.gpu
U = 2.0 ** -23
BF16, F32 = torch.bfloat16, torch.float32
# Rows of the experts.  With so many outputs (columns for the gradient) as below the first take tiles of 128 rows and the second of 256.
FEW, MANY = [100, 0, 129, 1], [300, 513, 0, 70]


def shifted(t, gap, shift):
    """the same matrix with rows further apart, and in another place"""
    whole = torch.full((t.shape[0] * (t.shape[1] + gap) + shift,), math.nan, dtype=t.dtype, device="cuda")
    view = whole[shift:].view(t.shape[0], t.shape[1] + gap)[:, :t.shape[1]]
    view.copy_(t)
    return view


def sample(n):
    return torch.unique(torch.cat([torch.arange(0, n, 61), torch.arange(max(0, n - 5), n)]))


def check(got, want, size, terms, cols, eps):
    got = got[:, cols.cuda()].cpu().double()
    rows = torch.isnan(want).all(dim=1)
    assert bool((got[rows] == 7.0).all())
    far = ((got - want).abs() - (eps * want.abs() + terms * U * size * (1 + eps)))[~rows]
    assert float(far.max()) <= 0, float(far.max())


def product(counts, N, K, out_type, gap=0, shift=0):
    offsets, n_rows, n = plain.groups(counts, align=4, ahead=2)
    wc, ws = plain.random_weights(len(counts), N, K, N + K)
    x = torch.randn(n, K, generator=torch.Generator(device="cuda").manual_seed(K), device="cuda").to(BF16)
    rows = shifted(x, gap, shift) if gap or shift else x
    out = torch.full((n, N), 7.0, dtype=out_type, device="cuda")
    X.product(rows, offsets, n_rows, wc, ws, out)
    cols = sample(N)
    w = plain.values(wc[:, cols.cuda()], ws[:, cols.cuda()])
    check(out, *plain.products(x.cpu().double(), offsets, n_rows, w), K, cols, torch.finfo(out_type).eps / 2)
    again = torch.full_like(out, 7.0)
    X.product(rows, offsets, n_rows, wc, ws, again)
    assert torch.equal(out, again)


def gradient(counts, N, K, out_type, gap=0, shift=0):
    offsets, n_rows, n = plain.groups(counts, align=4, ahead=2)
    wc, ws = plain.random_weights(len(counts), N, K, N + K)
    d = torch.randn(n, N, generator=torch.Generator(device="cuda").manual_seed(N), device="cuda").to(BF16)
    rows = shifted(d, gap, shift) if gap or shift else d
    back = torch.full((n, K), 7.0, dtype=out_type, device="cuda")
    X.product_grad(rows, offsets, n_rows, wc, ws, back)
    cols = sample(K)
    w = plain.values(wc, ws)[..., cols]
    check(back, *plain.products(d.cpu().double(), offsets, n_rows, w, transposed=True), N, cols, torch.finfo(out_type).eps / 2)
    again = torch.full_like(back, 7.0)
    X.product_grad(rows, offsets, n_rows, wc, ws, again)
    assert torch.equal(back, again)


@pytest.mark.parametrize("out_type", [BF16, F32])
@pytest.mark.parametrize("counts,N", [(FEW, 16391), (MANY, 33001), ([600] * 3, 21856), ([257, 2, 255], 21760)])
@pytest.mark.parametrize("K", [32, 128, 160, 256, 288, 544, 1056])
def test_product(counts, N, K, out_type):
    product(counts, N, K, out_type)


@pytest.mark.parametrize("counts,N", [(FEW, 16390), (MANY, 33000)])
@pytest.mark.parametrize("K", [32, 160, 512, 1056])
@pytest.mark.parametrize("gap,shift", [(16, 0), (1, 0), (0, 1), (7, 5)])
def test_product_rows_anywhere(counts, N, K, gap, shift):
    product(counts, N, K, BF16, gap, shift)


@pytest.mark.parametrize("out_type", [BF16, F32])
@pytest.mark.parametrize("counts,K", [(FEW, 16416), (MANY, 16384), ([600] * 3, 5632), ([257, 2, 255], 5632)])
@pytest.mark.parametrize("N", [8, 72, 256, 264, 520, 1048])
def test_gradient(counts, K, N, out_type):
    gradient(counts, N, K, out_type)


@pytest.mark.parametrize("counts,K", [(FEW, 16416), (MANY, 16384), ([600] * 3, 5632)])
@pytest.mark.parametrize("N,gap,shift", [(8, 1, 0), (9, 0, 0), (71, 0, 0), (250, 6, 0), (257, 7, 0), (264, 0, 3), (517, 0, 1), (1027, 5, 2)])
def test_gradient_rows_anywhere(counts, K, N, gap, shift):
    gradient(counts, N, K, BF16, gap, shift)


@pytest.mark.parametrize("counts,K", [([600] * 3, 4096), ([700, 0, 513, 130], 3968), ([300, 0, 513, 600], 16384)])
@pytest.mark.parametrize("N,gap,shift", [(8, 1, 0), (9, 0, 0), (250, 6, 0), (257, 7, 0), (264, 0, 3), (264, 0, 0), (1027, 5, 2)])
def test_gradient_rows_anywhere_of_many_rows(counts, K, N, gap, shift):
    gradient(counts, N, K, BF16, gap, shift)


@pytest.mark.parametrize("out_type", [BF16, F32])
@pytest.mark.parametrize("counts,K", [([257, 2, 255], 6912), ([70] * 5, 8200 // 32 * 32)])
@pytest.mark.parametrize("N", [8, 264, 1048])
def test_gradient_few_tiles(counts, K, N, out_type):
    gradient(counts, N, K, out_type)


@pytest.mark.parametrize("counts,N", [(FEW, 16390), (MANY, 33000)])
@pytest.mark.parametrize("gap", [0, 1])
def test_nan_stays_with_its_row(counts, N, gap):
    offsets, n_rows, n = plain.groups(counts, align=4, ahead=2)
    K = 288
    wc, ws = plain.random_weights(4, N, K, 6)
    ws[0] = ws[0].clamp(max=124)
    x = torch.randn(n, K, device="cuda").to(BF16)
    clean, out = torch.full((n, N), 7.0, device="cuda"), torch.full((n, N), 7.0, device="cuda")
    rows = shifted(x, gap, 0)
    X.product(rows, offsets, n_rows, wc, ws, clean)
    x[3, K - 1], x[0] = math.inf, math.nan               # a row of the first expert; one of none
    ws[3, 5, 3] = 255
    X.product(shifted(x, gap, 0), offsets, n_rows, wc, ws, out)
    o3, c3 = int(offsets[3]), counts[3]
    want = torch.zeros(n, N, dtype=torch.bool, device="cuda")
    want[3], want[o3:o3 + c3, 5] = True, True
    assert torch.equal(out[~want], clean[~want])
    assert bool(torch.isnan(out[o3:o3 + c3, 5]).all()) and not bool(torch.isfinite(out[3]).any())
    # the row's infinity meets weights of both signs and zeros: as in the plain form
    w = plain.values(wc[0], ws[0])[:, K - 1]
    assert torch.equal(torch.isposinf(out[3]).cpu(), w > 0) and torch.equal(torch.isnan(out[3]).cpu(), w == 0)


@pytest.mark.parametrize("counts", [FEW, MANY])
@pytest.mark.parametrize("N,gap", [(264, 0), (261, 0)])
def test_gradient_nan_stays_with_its_row(counts, N, gap):
    gradient_nan(counts, N, 16416)


@pytest.mark.parametrize("K", [3968, 16416])
def test_gradient_nan_stays_with_its_row_of_many_rows(K):
    gradient_nan([700, 513, 0, 130], 261, K)


def gradient_nan(counts, N, K):
    offsets, n_rows, n = plain.groups(counts, align=4, ahead=2)
    wc, ws = plain.random_weights(4, N, K, 6)
    d = torch.randn(n, N, device="cuda").to(BF16)
    clean, back = torch.full((n, K), 7.0, device="cuda"), torch.full((n, K), 7.0, device="cuda")
    X.product_grad(d, offsets, n_rows, wc, ws, clean)
    d[3, N - 1], d[0] = math.nan, math.nan
    ws[3, N - 1, 3] = 255
    X.product_grad(d, offsets, n_rows, wc, ws, back)
    o3, c3 = int(offsets[3]), counts[3]
    want = torch.zeros(n, K, dtype=torch.bool, device="cuda")
    want[3], want[o3:o3 + c3, 96:128] = True, True
    assert torch.equal(torch.isnan(back), want)
    assert torch.equal(back[~want], clean[~want])


def test_counts_that_do_not_fit_the_matrix():
    n, N, K = 700, 40000, 64
    wc, ws = plain.random_weights(4, N, K, 8)
    x = torch.randn(n, K, device="cuda").to(BF16)
    i32 = dict(dtype=torch.int32, device="cuda")
    offsets, counts = torch.tensor([0, -5, 690, 1 << 30, 3], **i32), torch.tensor([3, 400, 100000, 2 ** 31 - 1], **i32)
    whole = torch.full((n + 600, N), 7.0, device="cuda")
    X.product(x, offsets, counts, wc, ws, whole[300:300 + n])
    done = torch.zeros(n + 600, dtype=torch.bool, device="cuda")
    done[300:303], done[990:1000] = True, True
    assert bool((whole[~done] == 7.0).all()) and not bool((whole[done] == 7.0).all(dim=1).any())


def test_rows_in_4_bits_of_many_rows():
    """tiles of 256 rows at their ends, scales at any address"""
    for counts, N, K, gap in (([300, 0, 513, 70], 1000, 544, 0), ([300, 0, 513, 70], 1000, 544, 3), ([257, 255], 520, 1024, 1), ([600], 257, 32, 0)):
        offsets, n_rows, n = plain.groups(counts, align=4, ahead=2)
        wc, ws = plain.random_weights(len(counts), N, K, N + K)
        x, xs = (t[0] for t in plain.random_weights(1, n, K, K))
        out = torch.full((n, N), 7.0, device="cuda")
        scales = torch.zeros(n, K // 32 + gap, dtype=torch.uint8, device="cuda")[:, :K // 32]
        scales.copy_(xs)
        X.product(x, offsets, n_rows, wc, ws, out, row_scales=scales)
        cols = torch.arange(N)
        check(out, *plain.products(plain.values(x, xs), offsets, n_rows, plain.values(wc, ws)), K, cols, 2.0 ** -24)
