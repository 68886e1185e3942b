"""The norms on no tokens, in every kind of call: nothing to do in the forward call; sums over no tokens, which are 0, in the
gradient.  An empty tensor's address is NULL."""
import math

import pytest
import torch

import test_gpu_block_norm as N
from paper_2604_02715_amd import moe_block as M

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H", [64, 250, 8200])
@pytest.mark.parametrize("y,residual,weight,gate,post", N.KINDS)
@pytest.mark.parametrize("sigmoid", [False, True])
def test_no_tokens(H, y, residual, weight, gate, post, sigmoid):
    sigmoid = sigmoid and gate is not None
    d = {k: N.cuda(v) for k, v in N.make(0, H, y, residual, weight, gate, post, 1).items()}
    has = y is not None
    n = torch.empty(0, H, dtype=torch.bfloat16, device="cuda")
    M.block_norm(d["residual"], d["w_pre"], n, y=d["y"], gate=d["gate"], w_post=d["w_post"],
                 residual_out=torch.empty_like(d["residual"]) if has else None, gate_sigmoid=sigmoid)
    like = lambda t: None if t is None else torch.full(t.shape, math.nan, dtype=torch.float32, device="cuda")
    d_w, d_w_post, d_gate = like(d["w_pre"]), like(d["w_post"]), like(d["gate"])
    for d_out in (None, torch.empty_like(d["residual"])):
        M.block_norm_grad(d["residual"], d["w_pre"], n, torch.empty_like(d["residual"]), d_w, torch.empty(0, dtype=torch.uint8, device="cuda"),
                          d_residual_out=d_out, y=d["y"], gate=d["gate"], w_post=d["w_post"], d_y=torch.empty_like(d["y"]) if has else None,
                          d_gate=d_gate, d_w_post=d_w_post, gate_sigmoid=sigmoid)
        for t in (d_w, d_w_post, d_gate):
            if t is not None:
                assert torch.equal(t, torch.zeros_like(t))
                t.fill_(math.nan)
