"""Weights at the ends of their range: products with rows in 4 bits take every code at every scale as it is; with BF16 rows, and in the gradient,
a weight counts as BF16, which holds all but the largest at scales 253 and 254: those are infinite.

One term to a sum, whose other numbers are 0: the results are exact, their rounding to FP32 apart (2^-24)."""
import pytest
import torch

from paper_2604_02715_amd import mx_experts as X
from tests import mx_plain as plain

pytestmark = pytest.mark.gpu
BF16_MOST = 255 * 2.0 ** 120
SCALES = [0, 1, 2, 10, 252, 253, 254]


def weights(scale, N, K):
    """output n's first column is code n % 16, the others 0"""
    codes = torch.zeros(1, N, K // 2, dtype=torch.uint8, device="cuda")
    codes[0, :, 0] = torch.arange(N, device="cuda") % 16
    return codes, torch.full((1, N, K // 32), scale, dtype=torch.uint8, device="cuda")


def other(scale):
    return 2.0 ** (100 if scale < 100 else -100)


@pytest.mark.parametrize("rows", [3, 40, 700])
@pytest.mark.parametrize("scale", SCALES)
def test_product(scale, rows):
    N, K = 16400 if rows == 700 else 48, 64
    wc, ws = weights(scale, N, K)
    offsets, counts, n = plain.groups([rows])
    x = torch.zeros(n, K, dtype=torch.bfloat16, device="cuda")
    x[:, 0] = other(scale)
    out = torch.empty(n, N, device="cuda")
    w = plain.values(wc, ws)[0, :, 0]
    codes, scales = torch.empty(n, K // 2, dtype=torch.uint8, device="cuda"), torch.empty(n, K // 32, dtype=torch.uint8, device="cuda")
    X.quantize(x, codes, scales)                             # powers of two: exact
    X.product(codes, offsets, counts, wc, ws, out, row_scales=scales)
    assert torch.equal(out.cpu().double(), (w * other(scale)).expand(n, N))
    X.product(x, offsets, counts, wc, ws, out)
    fits = w.abs() <= BF16_MOST
    assert bool(fits.all()) == (scale < 253)
    assert torch.equal(out[:, fits.cuda()].cpu().double(), (w * other(scale))[fits].expand(n, -1))
    assert bool(torch.isinf(out[:, ~fits.cuda()]).all())


@pytest.mark.parametrize("rows", [3, 40, 700])
@pytest.mark.parametrize("scale", SCALES)
def test_gradient(scale, rows):
    N, K = 48, 16416 if rows == 700 else 64
    wc, ws = weights(scale, N, K)
    offsets, counts, n = plain.groups([rows])
    w = plain.values(wc, ws)[0, :, 0]
    fits = w.abs() <= BF16_MOST
    for at in (0, 3, 13) if scale < 253 else (0, 3, 11):     # codes that fit (4 and 6 do not at 253, 2 and more not at 254)
        d = torch.zeros(n, N, dtype=torch.bfloat16, device="cuda")
        d[:, at] = other(scale)
        codes = wc.clone()
        codes[0, ~fits.cuda()] = 0                           # an infinite weight meets zeros
        back = torch.empty(n, K, device="cuda")
        X.product_grad(d, offsets, counts, codes, ws, back)
        want = torch.zeros(n, K, dtype=torch.float64)
        want[:, 0] = w[at] * other(scale)
        assert torch.equal(back.cpu().double(), want)
    back = torch.empty(n, K, device="cuda")
    d.fill_(other(scale))                                    # (of ones the partial sums, 18 * 2^125 at scale 252, would be infinite themselves)
    X.product_grad(d, offsets, counts, wc, ws, back)
    assert bool(torch.isfinite(back[:, 0]).all()) == bool(fits.all())
