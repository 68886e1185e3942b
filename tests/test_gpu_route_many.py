"""The router on so many tokens that a row is spread over few lanes (65 to 512 experts, 16 choices at most), by the plain forms and
tolerances of the shorter batches, and against the same rows routed a few at a time, where other kernels run: the choice is the
same to the bit, also in ties, under masks and in rows with nothing to choose.

A gate's sum is added up in another order there: (log2(E) + 16) u from either side."""
import math

import pytest
import torch

import test_gpu_route as R
from paper_2604_02715_amd import moe_block as M

pytestmark = pytest.mark.gpu
T = 16391                        # more than the longest batch that goes the other way; the last workgroup has a part of its rows
PIECE = 1024
SHAPES = [(65, 1), (65, 8), (128, 9), (129, 16), (160, 8), (192, 9), (193, 16), (256, 8), (257, 10), (257, 16), (509, 16), (512, 1), (512, 10)]


def in_pieces(logits, K, bias=None, **kw):
    parts = [R.run(logits[t:t + PIECE], K, bias, **kw) for t in range(0, logits.shape[0], PIECE)]
    return torch.cat([ids for ids, _ in parts]), torch.cat([gates for _, gates in parts])


def same(logits, K, bias=None, **kw):
    ids, gates = R.run(logits, K, bias, **kw)
    want_ids, want = in_pieces(logits, K, bias, **kw)
    assert torch.equal(ids, want_ids)
    tol = 2 * (math.log2(logits.shape[1]) + 16) * R.U
    assert bool(((gates - want).abs() <= tol * want.abs() + 2.0 ** -126).all())
    return ids, gates


def bias_of(E):
    return (torch.randn(E, generator=torch.Generator().manual_seed(E)) * 30).round() * 0.001


@pytest.mark.parametrize("E,K", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_choice_and_gates(E, K, dtype):
    logits = R.make_logits(T, E, dtype, 1000 * E + K)
    dev = logits.cuda()
    R.check(logits, dev, K, "softmax", K % 2 == 0)
    R.check(logits, dev, K, "sigmoid", K % 2 == 1, scale=2.5, bias=bias_of(E))


@pytest.mark.parametrize("E,K", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_as_the_same_rows_a_few_at_a_time(E, K, dtype):
    logits = R.make_logits(T, E, dtype, 7 * E + K).cuda()
    for renormalize in (True, False):
        same(logits, K, score="softmax", renormalize=renormalize)
        same(logits, K, bias_of(E), score="sigmoid", renormalize=renormalize, scale=2.5)


@pytest.mark.parametrize("E,K", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_equal_scores_go_to_the_lowest_expert(E, K, dtype):
    logits = R.make_logits(T, E, torch.float32, 5).mul(2).round().div(2).to(dtype)      # few distinct values
    logits[::5] = 0.0
    logits[1::5, ::2] = -0.0                                                           # equal to the zeros between them
    logits[1::5, 1::2] = 0.0
    ids = R.check(logits, logits.cuda(), K, "softmax", True)
    first = torch.arange(K).expand(len(range(0, T, 5)), K)
    assert torch.equal(ids[::5], first) and torch.equal(ids[1::5], first[:len(range(1, T, 5))])
    same(logits.cuda(), K, score="sigmoid", renormalize=False)
    same(logits.cuda(), K, bias_of(E).mul(10).round().div(10), score="sigmoid", renormalize=True)


@pytest.mark.parametrize("E,K", SHAPES)
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_masks_infinities_and_nan(E, K, score):
    lowest = torch.finfo(torch.float32).min
    some = R.make_logits(13, E, torch.float32, 9)
    some[0] = -math.inf                                      # nothing to choose
    some[1] = -math.inf
    some[1, E // 2] = 0.3                                    # one expert
    some[2] = lowest                                         # masks of the type's lowest value are numbers like others
    some[3] = lowest
    some[3, E - 1] = 1.0
    some[4, ::2] = math.nan
    some[5] = math.nan
    some[6, 1::2] = -math.inf
    some[7] = 200.0
    some[8] = -200.0
    some[9, 0], some[9, 1:] = 3.0e38, -3.0e38
    some[10, 3] = math.inf
    logits = some.repeat((T + 12) // 13, 1)[:T].cuda()
    for renormalize in (True, False):
        ids, gates = same(logits, K, score=score, renormalize=renormalize)
        assert bool(torch.isfinite(gates).all()) and bool(((ids >= 0) | (gates == 0)).all())
        assert bool((ids[0::13] == -1).all()) and bool((ids[5::13] == -1).all())
        assert bool((ids[1::13, 0] == E // 2).all()) and bool((ids[1::13, 1:] == -1).all())
        if score == "softmax":
            assert bool((ids[10::13, 0] == 3).all())
            assert bool((gates[3::13, 0] == 1.0).all()) and bool((ids[3::13, 0] == E - 1).all())


@pytest.mark.parametrize("E,K", [(96, 8), (160, 16), (509, 10), (512, 10)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_and_alignment(E, K, dtype):
    wide = R.make_logits(T, E + 13, dtype, 3).cuda()
    for at in (0, 1, 8):                                     # rows that start at 16 bytes, and rows that do not
        view = wide[:, at:at + E]
        for score in ("softmax", "sigmoid"):
            got, want = R.run(view, K, score=score), R.run(view.contiguous(), K, score=score)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_on_another_stream_and_again():
    logits = R.make_logits(T, 160, torch.bfloat16, 8).cuda()
    ids, gates = R.run(logits, 8, score="sigmoid")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = [torch.empty(T, 8, dtype=torch.int32, device="cuda"), torch.empty(T, 8, device="cuda")]
    for _ in range(3):
        M.route(logits, *other, score="sigmoid", stream=side)
        side.synchronize()
        assert torch.equal(other[0].cpu().long(), ids) and torch.equal(other[1].cpu(), gates)
