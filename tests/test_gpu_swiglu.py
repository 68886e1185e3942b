"""SwiGLU and its gradient against 64 bits, the gradient against differences, too: widths that are not whole pieces, strides, far gates, in place.

Tolerances: u = 2^-24.  e^-|g| is good to 2 ulp (4 u); the sum, the quotient and up to five products add 8 u: 16 u of the result, and for
the gate's gradient 16 u of |d u p| (1 + |g| (1 - p)), as 1 + g (1 - p) can cancel.  Then the output's own rounding, eps / 2, and the
smallest subnormal number where it underflows."""
import math

import pytest
import torch

from paper_2604_02715_amd import mx_experts as X

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = [torch.bfloat16, torch.float32]


def plain(gate_up, d):
    g, u = gate_up.cpu().double().chunk(2, dim=1)
    p, q = torch.sigmoid(g), torch.sigmoid(-g)
    h, d = g * p * u, d.cpu().double()
    size = (d * u * p).abs() * (1 + g.abs() * q)
    return h, torch.cat([d * u * p * (1 + g * q), d * g * p], dim=1), torch.cat([size, (d * g * p).abs()], dim=1)


def near(got, want, size):
    eps = torch.finfo(got.dtype).eps / 2
    tiny = 2.0 ** (-133 if got.dtype == torch.bfloat16 else -149)
    far = (got.cpu().double() - want).abs() - (eps * want.abs() + 16 * U * size * (1 + eps) + 4 * tiny)
    assert float(far.max()) <= 0, float(far.max())


def inputs(R, F, t, th, seed):
    g = torch.Generator().manual_seed(seed)
    return (3 * torch.randn(R, 2 * F, generator=g)).to(t).cuda(), torch.randn(R, F, generator=g).to(th).cuda()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("th", TYPES)
@pytest.mark.parametrize("R,F", [(1, 1), (1, 512), (3, 8), (5, 1536), (2, 4100), (7, 33), (600, 16), (1, 14336)])
def test_both_directions(R, F, t, th):
    gate_up, d = inputs(R, F, t, th, R * F)
    h, back = torch.full((R, F), math.nan, dtype=th, device="cuda"), torch.full_like(gate_up, math.nan)
    X.swiglu(gate_up, h)
    X.swiglu_grad(gate_up, d, back)
    want, want_back, size = plain(gate_up, d)
    near(h, want, want.abs())
    near(back, want_back, size)
    X.swiglu_grad(gate_up, d, gate_up)                       # into its own rows
    assert torch.equal(gate_up, back)


def test_gradient_against_differences():
    gate_up, d = inputs(4, 64, torch.float32, torch.float32, 1)
    back = torch.empty_like(gate_up)
    X.swiglu_grad(gate_up, d, back)
    x = gate_up.cpu().double()
    f = lambda x: (plain(x, d)[0] * d.cpu().double()).sum()
    for at in [(0, 0), (1, 17), (3, 63), (2, 64), (0, 127)]:
        step = torch.zeros_like(x)
        step[at] = 1e-5
        want = float(f(x + step) - f(x - step)) / 2e-5
        assert abs(float(back[at]) - want) <= 1e-6 * max(1.0, abs(want)) + 1e-8


@pytest.mark.parametrize("g,h,dg", [(0.0, 0.0, 0.5), (200.0, 200.0, 1.0), (-200.0, 0.0, 0.0), (3e38, 3e38, 1.0), (-3e38, 0.0, 0.0), (88.8, 88.8, 1.0),
                                    (-88.8, 0.0, 0.0), (1e-40, 0.0, 0.5)])
def test_far_gates(g, h, dg):
    gate_up = torch.tensor([[g] * 4 + [1.0] * 4], device="cuda")
    out, back, d = torch.empty(1, 4, device="cuda"), torch.empty(1, 8, device="cuda"), torch.ones(1, 4, device="cuda")
    X.swiglu(gate_up, out)
    X.swiglu_grad(gate_up, d, back)
    assert torch.allclose(out.cpu(), torch.full((1, 4), h), rtol=1e-6, atol=1e-35)
    assert torch.allclose(back[:, :4].cpu(), torch.full((1, 4), dg), rtol=1e-6, atol=1e-35)
    assert torch.allclose(back[:, 4:].cpu(), torch.full((1, 4), h), rtol=1e-6, atol=1e-35)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("gap,shift", [(8, 0), (1, 0), (0, 1), (5, 3)])
def test_strides(t, gap, shift):
    R, F = 6, 40
    gate_up, d = inputs(R, F, t, t, 5)

    def place(x):
        whole = torch.full((R * (x.shape[1] + gap) + shift,), 9.0, dtype=t, device="cuda")
        view = whole[shift:].view(R, x.shape[1] + gap)[:, :x.shape[1]]
        view.copy_(x)
        return whole, view

    h_all, h = place(torch.zeros(R, F))
    back_all, back = place(torch.zeros(R, 2 * F))
    want_h, want_back = torch.empty_like(d), torch.empty_like(gate_up)
    X.swiglu(gate_up, want_h)
    X.swiglu_grad(gate_up, d, want_back)
    X.swiglu(place(gate_up)[1], h)
    X.swiglu_grad(place(gate_up)[1], place(d)[1], back)
    assert torch.equal(h, want_h) and torch.equal(back, want_back)
    h.fill_(9.0), back.fill_(9.0)
    assert bool((h_all == 9.0).all()) and bool((back_all == 9.0).all())


def test_no_rows():
    e = lambda F: torch.empty(0, F, device="cuda")
    X.swiglu(e(64), e(32))
    X.swiglu_grad(e(64), e(32), e(64))
