"""The norms around a block where a workgroup walks through several rows: the next row's loads under way, the LDS of the sums in
turn, a last step in which some workgroups have no row.  At most 768 workgroups of four rows (up to 512 columns), 1024 of one
(up to 1536), 768 (2048) or 256 (more than 4096) run at once, so that every batch here takes two steps at least.  Plain forms and
tolerances are those of the shorter batches."""
import pytest
import torch

import test_gpu_block_norm as N

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,H", [(7001, 264), (2051, 1032), (1601, 2048), (777, 5120), (515, 8192)])
@pytest.mark.parametrize("y,residual,weight,gate,post", N.KINDS)
@pytest.mark.parametrize("sigmoid,zero_centred,pad", [(False, False, 0), (True, True, 16)])
def test_forward(T, H, y, residual, weight, gate, post, sigmoid, zero_centred, pad):
    N.test_forward(T, H, y, residual, weight, gate, post, sigmoid, zero_centred, pad)


@pytest.mark.parametrize("T,H", [(5003, 264), (4099, 512), (1201, 1032), (777, 5120), (515, 8192)])
@pytest.mark.parametrize("y,residual,weight,gate,post", N.KINDS)
@pytest.mark.parametrize("sigmoid,zero_centred", [(False, False), (True, True)])
def test_gradient(T, H, y, residual, weight, gate, post, sigmoid, zero_centred):
    N.test_gradient_against_the_formula(T, H, y, residual, weight, gate, post, sigmoid, zero_centred, 0)


@pytest.mark.parametrize("T,H", [(7001, 64), (1601, 2048), (515, 8192)])
def test_rows_do_not_depend_on_their_neighbours(T, H):
    """Each row alone, in another order and beside other rows has the same bits."""
    d = {k: N.cuda(v) for k, v in N.make(T, H, "bf16", "f32", "f32", "token", True, 3).items()}

    def run(rows):
        out, n = torch.empty(len(rows), H, device="cuda"), torch.empty(len(rows), H, dtype=torch.bfloat16, device="cuda")
        N.M.block_norm(d["residual"][rows].contiguous(), d["w_pre"], n, y=d["y"][rows].contiguous(), gate=d["gate"][rows].contiguous(),
                       w_post=d["w_post"], residual_out=out)
        return out, n

    straight = run(torch.arange(T))
    turned = run(torch.arange(T).flip(0))
    assert all(torch.equal(a, b.flip(0)) for a, b in zip(straight, turned))
    for t in (0, 1, T // 2, T - 1):
        assert all(torch.equal(a[t:t + 1], b) for a, b in zip(straight, run(torch.tensor([t]))))
