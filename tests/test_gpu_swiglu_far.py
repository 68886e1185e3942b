"""SwiGLU of gates whose e^g leaves FP32's normal numbers while h, or a gradient, does not: against 64 bits, between near gates, beside NaN.

Tolerances: those of the other gates (16 u of the result; for the gate's gradient of |d u p| (1 + |g| (1 - p)), u = 2^-24, then half a step of the
output and the smallest subnormal number).  They hold: the power of 2 is good to 1 ulp (2 u), its argument to 2^-26, its correction
adds u, products are in 64 bits and rounded once."""
import math

import pytest
import torch

from paper_2604_02715_amd import mx_experts as X
from test_gpu_swiglu import TYPES, near, plain

pytestmark = pytest.mark.gpu
GATES = [-80.0, -86.9, -87.0, -87.1, -87.34, -88.0, -88.5, -88.8, -95.5, -103.9, -104.1, -120.0, -150.0, -199.0, -201.0, -300.0, -700.0, -800.0, -3e4, -3e38]
# (up, gradient of h)
OTHERS = [(1.0, 1.0), (-1e30, 1e-3), (3e38, 0.5), (-1e-3, 1e25), (1e-20, -1e38)]


def call(g, u, d, t, th):
    """(gate_up, d) one row of them"""
    return torch.cat([g, u]).to(t)[None].cuda(), d.to(th)[None].cuda()


def both(gate_up, d):
    h, back = torch.full_like(d, math.nan), torch.full_like(gate_up, math.nan)
    X.swiglu(gate_up, h)
    X.swiglu_grad(gate_up, d, back)
    return h, back


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("th", TYPES)
@pytest.mark.parametrize("near_gates", [0, 1])
@pytest.mark.parametrize("behind", [0, 1])                   # one more column: no whole pieces
def test_far_below(t, th, near_gates, behind):
    cases = [(g, u, d) for g in GATES for u, d in OTHERS]
    cases = [c for case in cases for c in [case] + [(0.75, 2.0, -3.0)] * near_gates] + [(1.0, 1.0, 1.0)] * behind
    g, u, d = (torch.tensor(x) for x in zip(*cases))
    gate_up, d = call(g, u, d, t, th)
    h, back = both(gate_up, d)
    want, want_back, size = plain(gate_up, d)
    near(h, want, want.abs())
    near(back, want_back, size)
    X.swiglu_grad(gate_up, d, gate_up)                       # into its own rows
    assert torch.equal(gate_up, back)


def test_far_gates_are_not_lost():
    """the formula's own numbers: e^88 is finite, and so is what it divides"""
    g = torch.tensor([-88.0, -88.5, -95.0, -100.0])
    u = torch.tensor([1.0, 1.0, 1e30, 1e30])
    gate_up, d = call(g, u, torch.ones(4), torch.float32, torch.float32)
    h, back = both(gate_up, d)
    e = torch.exp(g.double())
    assert torch.allclose(h[0].cpu().double(), g * e * u, rtol=2.0 ** -20, atol=0)
    assert torch.allclose(back[0, :4].cpu().double(), u * e * (1 + g.double()), rtol=2.0 ** -20, atol=0)
    assert torch.allclose(back[0, 4:6].cpu().double(), (g * e)[:2], rtol=2.0 ** -20, atol=0)


@pytest.mark.parametrize("t", TYPES)
def test_beside_nan_and_infinities(t):
    """a NaN does not hide a far gate of its piece; infinite gates are as the formula has them: infinite, or NaN"""
    g = torch.tensor([math.nan, -90.0, math.inf, -math.inf, -90.0, 1.0, math.nan, math.nan] * 2)
    u = torch.full((16,), 1e30)
    gate_up, d = call(g, u, torch.ones(16), t, t)
    h, back = both(gate_up, d)
    clean = torch.isfinite(g)
    only, only_d = call(torch.where(clean, g, 0.5), u, torch.ones(16), t, t)
    want_h, want_back = both(only, only_d)
    assert torch.equal(h[0].cpu()[clean], want_h[0].cpu()[clean])
    assert torch.equal(back.view(2, 16).cpu()[:, clean], want_back.view(2, 16).cpu()[:, clean])
    assert bool((want_h[0].cpu()[g == -90.0] < -1e-8).all())
    assert torch.equal(torch.isnan(h[0].cpu()), torch.isnan(g) | torch.isneginf(g)) and bool(torch.isposinf(h[0].cpu()[torch.isposinf(g)]).all())
