"""fluxmoe_route_grouped against a plain form: which groups are kept, ties of groups and experts, groups of one, masks that leave a group or
a row empty, and the gradient through the experts it chose.

Tolerance of the gates: as the router's without groups, (|l - m| + log2(E) + 16) 2^-24 of the gate.  Choices go by 32-bit scores, each
step rounded as written, and are compared exactly: by softmax on the logits themselves, by sigmoids on scores that a bias on a grid of
2^-8 keeps apart (or makes equal to the bit)."""
import math

import pytest
import torch

from paper_2604_02715_amd import moe_block as M

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def plain_choice(key, groups, top_groups, K, by):
    """ids [T][K] from float64 keys (minus infinity: never)"""
    T, E = key.shape
    best = torch.sort(key.view(T, groups, -1), dim=2, descending=True).values
    score = best[..., 0]
    if by == "top2" and E > groups:
        score = score + torch.where(best[..., 1] > -math.inf, best[..., 1], 0.0)
    score = torch.where(best[..., 0] > -math.inf, score, -math.inf)
    order = torch.sort(score, dim=1, descending=True, stable=True).indices[:, :top_groups]
    kept = torch.zeros(T, groups, dtype=torch.bool).scatter_(1, order, True)
    key = torch.where(kept.repeat_interleave(E // groups, dim=1), key, -math.inf)
    chosen = torch.sort(key, dim=1, descending=True, stable=True)
    return torch.where(chosen.values[:, :K] > -math.inf, chosen.indices[:, :K], -1)


def run(logits, K, **kw):
    T = logits.shape[0]
    ids = torch.full((T, K), -7, dtype=torch.int32, device="cuda")
    gates = torch.full((T, K), math.nan, device="cuda")
    M.route(logits, ids, gates, **kw)
    torch.cuda.synchronize()
    return ids.cpu().long(), gates.cpu().double()


def check_gates(logits, ids, gates, score, renormalize, scale=1.0):
    l = torch.where(torch.isnan(logits), -math.inf, logits.double())
    p = torch.sigmoid(l) if score == "sigmoid" else torch.softmax(l, dim=1).nan_to_num(0.0)
    p = torch.where(ids >= 0, torch.gather(p, 1, ids.clamp(min=0)), 0.0)
    if renormalize:
        p = p / p.sum(dim=1, keepdim=True).clamp(min=1e-300)
    spread = float(l[torch.isfinite(l)].max() - l[torch.isfinite(l)].min()) if bool(torch.isfinite(l).any()) else 0.0
    assert float((gates - scale * p).abs().max()) <= (spread + math.log2(l.shape[1]) + 16) * U * scale * max(1e-30, float(p.max()))


SHAPES = [(8, 2, 1, 2), (16, 4, 2, 4), (32, 32, 5, 5), (64, 8, 3, 8), (60, 5, 2, 7), (63, 9, 4, 8), (160, 8, 3, 8), (256, 8, 4, 8), (256, 64, 7, 20),
          (512, 8, 4, 10), (512, 64, 64, 64), (1024, 16, 2, 33), (2000, 50, 9, 10), (4096, 64, 3, 8), (4096, 2, 1, 64), (130, 5, 1, 26)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("E,G,KG,K", SHAPES)
def test_softmax(E, G, KG, K, renormalize, dtype):
    g = torch.Generator().manual_seed(E + G)
    logits = (2 * torch.randn(37, E, generator=g)).to(dtype)          # BF16 ones often tie
    logits[3] = 1.0
    logits[4, : E // G] = -math.inf
    logits[5] = -math.inf
    logits[6, E // 2:] = -math.inf
    logits[7, ::2] = math.nan
    ids, gates = run(logits.cuda(), K, renormalize=renormalize, groups=G, top_groups=KG)
    key = torch.where(torch.isnan(logits), -math.inf, logits).double()
    assert torch.equal(ids, plain_choice(key, G, KG, K, "max"))
    ok = [t for t in range(37) if t != 7]                             # a NaN has no softmax in 64 bits' plain form
    check_gates(logits[ok], ids[ok], gates[ok], "softmax", renormalize)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("by", ["max", "top2"])
@pytest.mark.parametrize("E,G,KG,K", SHAPES)
def test_sigmoid(E, G, KG, K, by, dtype):
    g = torch.Generator().manual_seed(E * G)
    logits = (2 * torch.randn(29, E, generator=g)).to(dtype)
    logits[2] = 0.0
    logits[4, : E // G] = -math.inf
    logits[5] = -math.inf
    logits[6, 1:] = -math.inf
    bias = torch.randint(-64, 65, (E,), generator=g) / 256.0
    for scale, renormalize in ((2.5, True), (1.0, False)):
        ids, gates = run(logits.cuda(), K, bias=bias.cuda(), score="sigmoid", renormalize=renormalize, scale=scale, groups=G, top_groups=KG,
                         group_score=by)
        # scores as the device rounds them: through the same steps in 32 bits
        x = logits.cuda().float()
        key = (1.0 / (1.0 + torch.exp(-x)) + bias.cuda()).cpu()
        key = torch.where(torch.isneginf(logits.float()), -math.inf, key)
        best = torch.sort(key.view(29, G, -1), dim=2, descending=True).values
        if by == "top2" and E > G:                                    # the sum of two is rounded, too
            two = best[..., 0] + torch.where(best[..., 1] > -math.inf, best[..., 1], torch.zeros(()))
            want = []
            for t in range(29):
                score = torch.where(best[t, :, 0] > -math.inf, two[t], -math.inf)
                kept = torch.sort(score, descending=True, stable=True).indices[:KG]
                k = torch.full((E,), -math.inf)
                for i in kept.tolist():
                    k[i * (E // G):(i + 1) * (E // G)] = key[t, i * (E // G):(i + 1) * (E // G)]
                s = torch.sort(k, descending=True, stable=True)
                want.append(torch.where(s.values[:K] > -math.inf, s.indices[:K], -1))
            want = torch.stack(want)
        else:
            want = plain_choice(key.double(), G, KG, K, "max")
        assert torch.equal(ids, want)
        check_gates(logits, ids, gates, "sigmoid", renormalize, scale)


def test_groups_that_tie_go_to_the_lower_one():
    logits = torch.zeros(1, 64)
    logits[0, [10, 26, 42]] = 1.0                                     # groups 1, 3, 5 of eight experts
    ids, _ = run(logits.cuda(), 4, groups=8, top_groups=2)
    assert ids.tolist() == [[10, 26, 8, 9]]
    ids, _ = run(logits.cuda(), 4, groups=8, top_groups=2, score="sigmoid", group_score="top2")
    assert ids.tolist() == [[10, 26, 8, 9]]


def test_top2_prefers_two_good_experts_to_one_better():
    logits = torch.full((1, 16), -2.0)
    logits[0, 3], logits[0, [8, 9]] = 3.0, 2.0
    kw = dict(groups=4, top_groups=1, score="sigmoid")
    assert run(logits.cuda(), 2, group_score="max", **kw)[0].tolist() == [[3, 0]]
    assert run(logits.cuda(), 2, group_score="top2", **kw)[0].tolist() == [[8, 9]]


def test_a_group_with_one_expert_left_counts_that_one():
    logits = torch.full((1, 8), -math.inf)
    logits[0, 1], logits[0, 6] = 2.0, 1.0
    bias = torch.full((8,), -3e38)                                    # two of them would be minus infinity
    for group_score in ("max", "top2"):
        ids, _ = run(logits.cuda(), 2, bias=bias.cuda(), score="sigmoid", groups=4, top_groups=2, group_score=group_score)
        assert ids.tolist() == [[1, 6]]
    logits[0, 0] = 2.0
    ids, _ = run(logits.cuda(), 2, bias=bias.cuda(), score="sigmoid", groups=4, top_groups=1, group_score="top2")
    assert ids.tolist() == [[6, -1]]                                  # -3e38 comes before a sum of minus infinity
    ids, _ = run(logits.cuda(), 3, bias=bias.cuda(), score="sigmoid", groups=4, top_groups=2, group_score="top2")
    assert ids.tolist() == [[0, 1, 6]]


@pytest.mark.parametrize("T,E,G,KG,K", [(1, 512, 8, 4, 10), (20000, 160, 8, 3, 8), (9000, 256, 8, 4, 8), (5000, 64, 8, 2, 4), (3000, 1024, 32, 4, 8)])
def test_many_rows(T, E, G, KG, K):
    logits = torch.randn(T, E, generator=torch.Generator().manual_seed(T)).to(torch.bfloat16)
    ids, gates = run(logits.cuda(), K, groups=G, top_groups=KG)
    assert torch.equal(ids, plain_choice(logits.double(), G, KG, K, "max"))
    check_gates(logits, ids, gates, "softmax", True)


def test_one_group_is_no_groups():
    logits = torch.randn(50, 48, device="cuda")
    assert all(torch.equal(a, b) for a, b in zip(run(logits, 6), run(logits, 6, groups=1, top_groups=1)))
    assert torch.equal(run(logits, 6, score="sigmoid", group_score="top2")[0], run(logits, 6, score="sigmoid")[0])


def test_unaligned_rows():
    whole = torch.randn(21 * 67 + 1, generator=torch.Generator().manual_seed(1)).cuda()
    logits = whole[1:].view(21, 67)[:, :64]
    ids, _ = run(logits, 5, groups=8, top_groups=2)
    assert torch.equal(ids, plain_choice(logits.cpu().double(), 8, 2, 5, "max"))


@pytest.mark.parametrize("score,renormalize", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
def test_gradient_of_the_chosen(score, renormalize):
    T, E, K = 33, 64, 6
    logits = torch.randn(T, E, generator=torch.Generator().manual_seed(9)).cuda()
    ids = torch.empty(T, K, dtype=torch.int32, device="cuda")
    gates, d = torch.empty(T, K, device="cuda"), torch.randn(T, K, device="cuda")
    kw = dict(score=score, renormalize=renormalize, scale=1.5)
    M.route(logits, ids, gates, groups=8, top_groups=3, **kw)
    back = torch.empty_like(logits)
    M.route_grad(logits, ids, d, back, **kw)
    x = logits.cpu().double().requires_grad_(True)
    p = torch.sigmoid(x) if score == "sigmoid" else torch.softmax(x, dim=1)
    p = torch.gather(p, 1, ids.cpu().long())
    if renormalize:
        p = p / p.sum(dim=1, keepdim=True)
    (1.5 * p * d.cpu().double()).sum().backward()
    assert float((back.cpu().double() - x.grad).abs().max()) <= 3 * 40 * U * 1.5 * float(d.abs().max())
