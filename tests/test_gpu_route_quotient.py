"""The scores that the choice by sigmoids goes by are the divisions 1 / (1 + e^-logit), to the bit, for each of the 2^23 significands
that the divisor can have.

Each divisor d = 1 + k 2^-23 below 2 is reached by a logit of its own, found in torch's exp (and its neighbours, where rounding
needs them).  A row has that logit at the first and at the last expert and, between them, an expert whose logit is plus infinity
and whose bias is q - 1, q the division's result: its score of 1 plus the bias is q exactly, as q is a multiple of 2^-24 from 1/2 to 1.
Equal scores go to the lowest expert, so the order first, middle, last comes out for equal scores and for no others."""
import math

import pytest
import torch

from paper_2604_02715_amd import moe_block as M

pytestmark = pytest.mark.gpu
N = 1 << 23


def divisor(logits):
    return 1.0 + torch.exp(-logits)


def logits_of_all_divisors():
    """logits[k] with divisor(logits[k]) = 1 + k 2^-23"""
    k = torch.arange(N, device="cuda", dtype=torch.float64)
    d = (1.0 + k / N).float()
    start = (-torch.log(k / N)).float()                      # plus infinity for k = 0
    logits, open_ = start.clone(), divisor(start) != d
    for step in range(1, 9):
        for way in (-math.inf, math.inf):
            other = start
            for _ in range(step):
                other = torch.nextafter(other, torch.full_like(other, way))
            hit = open_ & (divisor(other) == d)
            logits = torch.where(hit, other, logits)
            open_ &= ~hit
    assert not bool(open_.any()) and bool((divisor(logits) == d).all())
    return logits


@pytest.mark.parametrize("E", [4096, 500])
def test_every_divisor(E):
    logits = logits_of_all_divisors()
    q = 1.0 / divisor(logits)
    level = (q.double() * 2.0 ** 24).long()                  # q as a multiple of 2^-24
    assert torch.equal(level.double() * 2.0 ** -24, q.double())
    level, order = torch.sort(level)
    logits = logits[order]
    middle = E - 2                                           # experts between the first and the last: as many values of q at once
    lows = torch.arange(1 << 23, (1 << 24) + 1, middle, device="cuda")
    if E < 1000:                                             # another of the kernels: some of the range
        lows = lows[::16]
    ends = torch.searchsorted(level, torch.stack([lows, lows + middle])).tolist()
    seen = 0
    for low, first, end in zip(lows.tolist(), *ends):
        T = end - first
        if T == 0:
            continue
        bias = torch.zeros(E, device="cuda")
        values = (low + torch.arange(middle, device="cuda")).clamp(max=1 << 24)
        bias[1:-1] = (values.double() * 2.0 ** -24 - 1.0).float()
        x = torch.full((T, E), -math.inf, device="cuda")
        x[:, 0] = x[:, -1] = logits[first:end]
        at = (level[first:end] - low + 1)[:, None]
        x.scatter_(1, at, math.inf)
        ids, gates = torch.empty(T, 3, dtype=torch.int32, device="cuda"), torch.empty(T, 3, device="cuda")
        M.route(x, ids, gates, bias=bias, score="sigmoid", renormalize=False)
        want = torch.cat([torch.zeros_like(at), at, torch.full_like(at, E - 1)], dim=1)
        assert torch.equal(ids.long(), want), "scores from %d times 2^-24" % low
        seen += T
    assert seen == N if E > 1000 else seen > N // 32
