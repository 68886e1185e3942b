"""Gradient of a gate through its sigmoid where the gate is far open or far shut: g (1 - g) with 1 - g taken from a rounded g
keeps three digits at 10 and none from 17 on.

The gradient of the sigmoid's value g comes from the plain form in 64 bits, by differentiation, and is multiplied by
sigmoid(v) sigmoid(-v) there.  Tolerance: that of a gate's gradient without a sigmoid, of the absolute terms times the same factor
(4 (depth + 8) u for the terms' sizes as in the shorter tests, the sums over the tokens), and 8 u for the factor: e^-|v| to
2 ulp, a sum, a square, a quotient, and the products with scale and sum."""
import math

import pytest
import torch

import test_gpu_block_norm as N

pytestmark = pytest.mark.gpu
VALUES = [0.0, 1.0, 4.0, 8.0, 10.0, 12.0, 15.0, 16.6, 17.5, 20.0, 30.0, 60.0, 80.0]


@pytest.mark.parametrize("T,H", [(52, 64), (31, 2048), (17, 2051), (600, 512), (5, 8200)])
@pytest.mark.parametrize("gate", ["token", "channel"])
@pytest.mark.parametrize("y,residual,weight,post", [("f32", "bf16", "bf16", True), ("bf16", "f32", "f32", False), ("f32", "f32", "f32", True),
                                                    ("bf16", "bf16", "bf16", False)])
def test_gates_far_open_and_far_shut(T, H, gate, y, residual, weight, post):
    scale = 0.7
    d = N.make(T, H, y, residual, weight, gate, post, T + H)
    values = torch.tensor([s * v for v in VALUES for s in (1.0, -1.0)])
    v = values.repeat(d["gate"].numel() // values.numel() + 1)[:d["gate"].numel()].view(d["gate"].shape)
    g = torch.Generator().manual_seed(T)
    d_n = torch.randn(T, H, generator=g).to(torch.bfloat16)
    d_r = torch.randn(T, H, generator=g).to(N.TYPES[residual])
    got = N.run_gradient(dict(d, gate=v), d_n, d_r, scale, True, False)["gate"].cpu().double()

    opened = torch.sigmoid(v.double())
    slope = opened * torch.sigmoid(-v.double())
    want = N.gradients_64(dict(d, gate=opened), d_n, d_r, scale, False, False)["gate"] * slope
    w = d["w_pre"].double().abs()
    rstd = (d["residual"].double().square().mean(1, keepdim=True) + N.EPS).rsqrt()
    h, dn = (d["residual"].double() * rstd).abs(), d_n.double().abs()
    dr = d_r.double().abs() + rstd * (dn * w + h * (dn * w * h).mean(1, keepdim=True))
    inner = d["y"].double()
    if post:
        inner = inner * (inner.square().mean(1, keepdim=True) + N.EPS).rsqrt() * d["w_post"].double()
    size = scale * (dr * inner.abs()).sum(1 if gate == "token" else 0).view(v.shape) * slope
    tol = (N.depth(H, H % 8 == 0) + 8) * N.U
    over_t = 2 * T / 256 + 64 if gate == "channel" else 0
    assert bool(((got - want).abs() <= (4 * tol + 2 * over_t * N.U + 8 * N.U) * size + 2.0 ** -126).all())
