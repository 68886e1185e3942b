"""eps and scale of the norms given as tensors of one number: their value at the call counts, also where a program changes them in
place between two calls."""
import pytest
import torch

from paper_2604_02715_amd import moe_block as M

pytestmark = pytest.mark.gpu
T, H = 5, 64


def tensors():
    g = torch.Generator().manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=g).cuda()
    return dict(residual=rand(T, H), y=rand(T, H), w=rand(H), d_n=rand(T, H).to(torch.bfloat16))


def forward(t, **kw):
    out, n = torch.empty(T, H, device="cuda"), torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
    M.block_norm(t["residual"], t["w"], n, y=t["y"], residual_out=out, **kw)
    return out, n


def gradient(t, **kw):
    d_r, d_y, d_w = torch.empty(T, H, device="cuda"), torch.empty(T, H, device="cuda"), torch.empty(H, device="cuda")
    ws = torch.empty(M.block_norm_grad_workspace_bytes(T, H), dtype=torch.uint8, device="cuda")
    M.block_norm_grad(t["residual"], t["w"], t["d_n"], d_r, d_w, ws, y=t["y"], d_y=d_y, **kw)
    return d_r, d_y, d_w


@pytest.mark.parametrize("call", [forward, gradient])
@pytest.mark.parametrize("name", ["scale", "eps"])
@pytest.mark.parametrize("device", ["cpu", "cuda"])
def test_a_scalar_that_changes_in_place(call, name, device):
    t = tensors()
    scalar = torch.tensor(0.5, device=device)
    for value in (0.5, 2.0, 0.25):
        scalar.fill_(value)
        got, want = call(t, **{name: scalar}), call(t, **{name: value})
        assert all(torch.equal(a, b) for a, b in zip(got, want)), value
