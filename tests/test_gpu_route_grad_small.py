"""Gradient of sigmoid gates divided by their sum where the chosen sigmoids are below the normal numbers: the gates are ordinary
numbers there, and so are their gradients, though 1 / sum is not.

Tolerance: as in the longer tests (three times (log2(E) + 16) u of the largest term), and a score below the normal numbers is off
by half a spacing more, 2^-150 of at least 3.3e-39: 3.4 u, of which the gradient's terms hold six."""
import math

import pytest
import torch

import test_gpu_route as R
from paper_2604_02715_amd import moe_block as M

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("E,K", [(2, 2), (8, 2), (160, 8), (512, 10)])
def test_sigmoids_below_the_normal_numbers(E, K):
    T = 64
    g = torch.Generator().manual_seed(E)
    logits = -88.6 + 1.2 * torch.rand(T, E, generator=g)
    logits[::2, E // 2:] = -math.inf                         # where fewer are left than K, pairs without an expert
    ids, gates = R.run(logits.cuda(), K, score="sigmoid", renormalize=True, scale=2.5)
    d_gates = 3.0 * torch.randn(T, K, generator=g)
    got = torch.full((T, E), math.nan, device="cuda")
    M.route_grad(logits.cuda(), ids.int().cuda(), d_gates.cuda(), got, scale=2.5, score="sigmoid", renormalize=True)
    want = R.grad_64(logits, ids, d_gates, "sigmoid", True, 2.5)
    want = torch.where(logits == -math.inf, 0.0, want)
    tol = (3 * (math.log2(E) + 16) + 21) * R.U * 2.5 * d_gates.abs().amax(dim=1, keepdim=True).double()
    assert bool(torch.isfinite(gates).all())
    assert bool(((got.cpu().double() - want).abs() <= tol).all())
