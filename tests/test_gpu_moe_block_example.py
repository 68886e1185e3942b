"""The operators around the routed experts together with the path they stand around: examples/moe_block.py served against the
oracle's FFN and norms in 64 bits, and its gradients against differentiation of the whole block in 64 bits."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from oracle import ffn as offn
from paper_2604_02715_amd import inputs

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("example_moe_block", os.path.join(ROOT, "examples", "moe_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def rms_norm(x, w):
    return x / (x.square().mean(1, keepdim=True) + 1e-6).sqrt() * w


def test_serving_matches_the_oracle(example):
    cfg = inputs.CONFIGS["c1_tiny"]
    block, (w13, w2) = example.make_block(cfg)
    try:
        x = inputs.activations(cfg)
        residual = x.cuda()
        b = block.buffers(cfg.tokens)
        normed = block.serve(residual, b)
        torch.cuda.synchronize()
        assert block.pool.device_errors() == 0 and bool((block.pool.page_table == -1).all())
        # the norm in front, from the input
        n0 = rms_norm(x.double(), block.w_norm.cpu().double())
        assert bool(((b["normed"].cpu().double() - n0).abs() <= 2.0 ** -8 * n0.abs()).all())
        # choice and gates, from what the norm gave
        logits = (b["normed"].float() @ block.router.float().t()).cpu().double()
        ids = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :cfg.top_k]
        assert torch.equal(b["ids"].cpu().long(), ids)
        gates = torch.softmax(torch.gather(logits, 1, ids), dim=1)
        assert float((b["gates"].cpu().double() - gates).abs().max()) <= 1e-5
        # the FFN and the stream behind it
        y = offn.moe_ffn(inputs.bits_u16(b["normed"].cpu()), ids.int().numpy(), gates.float().numpy(),
                         lambda e: (inputs.bits_u16(w13[e]), inputs.bits_u16(w2[e])), round_h=True)
        assert offn.rel_frobenius(b["out"].cpu().numpy(), y) <= 1e-3
        r = x.double() + b["out"].cpu().double()
        assert bool(((residual.cpu().double() - r).abs() <= 2.0 ** -8 * r.abs() + 1e-6).all())
        n1 = rms_norm(r, block.w_next.cpu().double())
        assert bool(((normed.cpu().double() - n1).abs() <= 2.0 ** -8 * n1.abs() + 1e-5).all())
    finally:
        block.pool.close()


def test_gradients_of_the_block(example):
    cfg = inputs.scaled(inputs.CONFIGS["c1_tiny"], hidden=128, ffn=192)
    block, (w13, w2) = example.make_block(cfg, seed=3)
    try:
        T = 48
        x = torch.randn(T, cfg.hidden, generator=torch.Generator().manual_seed(5))
        d_out = torch.randn(T, cfg.hidden, generator=torch.Generator().manual_seed(6))
        block.freeze()
        b = block.buffers(T)
        stream, d_residual, d_router, d_w = block.forward_backward(x.cuda(), lambda s: d_out.cuda(), b)
        assert block.pool.device_errors() == 0

        xs, router, w = (t.double().requires_grad_(True) for t in (x, block.router.cpu(), block.w_norm.cpu()))
        n = rms_norm(xs, w)
        logits = n @ router.t()
        ids = b["ids"].cpu().long()
        gates = torch.softmax(torch.gather(logits, 1, ids), dim=1)
        want = xs
        for e in range(cfg.n_experts):
            a, c = w13[e].double(), w2[e].double()
            y = (torch.nn.functional.silu(n @ a[0]) * (n @ a[1])) @ c
            want = want + (gates * (ids == e)).sum(1, keepdim=True) * y
        (want * d_out.double()).sum().backward()
        off = lambda got, exact: float((got.cpu().double() - exact).norm() / exact.norm())
        # the norm's output and its gradient pass through BF16 (2^-9 relative each, forward and back), the products through FP32
        assert off(stream, want.detach()) <= 4e-3
        assert off(d_residual, xs.grad) <= 1e-2 and off(d_router, router.grad) <= 1e-2 and off(d_w, w.grad) <= 1e-2
    finally:
        block.pool.close()


def test_training_lowers_the_loss(example):
    block, _ = example.make_block(inputs.CONFIGS["c1_tiny"])
    try:
        losses = example.train(block)
        assert np.isfinite(losses).all() and losses[-1] < 0.7 * losses[0]
    finally:
        block.pool.close()
