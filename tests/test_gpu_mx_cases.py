"""Products with experts in 4 bits, and their gradient, against 64 bits, by every kernel that there is for them: the calls of mx_cases, which the
library's rule is asked about first, with both types of output.  On a sample of the outputs where there are many.  Rows of no expert keep what
was there, and the same call gives the same bits.

Tolerance: the terms are exact in FP32, a sum of n of them is off by at most n u of the sum of their magnitudes (u = 2^-23, as the matrix
instructions may cut instead of round), and an output by half a step of its type."""
import math

import pytest
import torch

import mx_cases as M
from paper_2604_02715_amd import mx_experts as X
from tests import mx_plain as plain

pytestmark = pytest.mark.gpu
U = 2.0 ** -23
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    return M.compile_rule(tmp_path_factory.mktemp("mx_cases"))


def apart(t, gap, shift, fill):
    """the same matrix with rows `gap` elements further apart, from element `shift` on; what lies between is `fill`"""
    if not gap and not shift:
        return t
    whole = torch.full((t.shape[0] * (t.shape[1] + gap) + shift,), fill, dtype=t.dtype, device="cuda")
    view = whole[shift:].view(t.shape[0], t.shape[1] + gap)[:, :t.shape[1]]
    view.copy_(t)
    return view


def moved(t, shift):
    """the same contiguous tensor, `shift` elements behind an aligned address"""
    whole = torch.zeros(t.numel() + shift, dtype=t.dtype, device="cuda")
    view = whole[shift:].view(t.shape)
    view.copy_(t)
    return view


class Call:
    """a case's tensors"""

    def __init__(self, c):
        self.c, seed = c, c["N"] + c["K"]
        self.offsets, self.counts, n = plain.groups(c["counts"], align=4, ahead=2)
        assert n == M.rows_of(c["counts"])
        self.wc, ws = plain.random_weights(len(c["counts"]), c["N"], c["K"], seed)
        self.ws = moved(ws, c["ws_shift"])
        self.grad, self.scales = c["op"] == "grad", None
        self.sum, self.width = (c["N"], c["K"]) if self.grad else (c["K"], c["N"])
        if c["mx"]:
            x, xs = (t[0] for t in plain.random_weights(1, n, c["K"], seed + 1))
            self.values = plain.values(x, xs)
            self.rows, self.scales = apart(x, c["gap"], c["shift"], 0x77), apart(xs, c["scale_gap"], 0, 255)
        else:
            x = torch.randn(n, self.sum, generator=torch.Generator(device="cuda").manual_seed(seed + 2), device="cuda").to(BF16)
            self.values = x.cpu().double()
            self.rows = apart(x, c["gap"], c["shift"], math.nan)

    def run(self, out_type):
        out = torch.full((self.rows.shape[0], self.width), 7.0, dtype=out_type, device="cuda")
        if self.grad:
            X.product_grad(self.rows, self.offsets, self.counts, self.wc, self.ws, out)
        else:
            X.product(self.rows, self.offsets, self.counts, self.wc, self.ws, out, row_scales=self.scales)
        return out

    def check(self, out):
        """on every so many outputs, the last ones among them"""
        E, eps = len(self.c["counts"]), torch.finfo(out.dtype).eps / 2
        step = next(s for s in (1, 7, 61) if s == 61 or E * self.sum * self.width / s <= 5e6)
        cols = torch.unique(torch.cat([torch.arange(0, self.width, step), torch.arange(max(0, self.width - 5), self.width)]))
        if self.grad:
            w = plain.values(self.wc, self.ws)[..., cols]
        else:
            w = plain.values(self.wc[:, cols.cuda()], self.ws[:, cols.cuda()])
        want, size = plain.products(self.values, self.offsets, self.counts, w, transposed=self.grad)
        got, none = out.cpu(), torch.isnan(want).all(dim=1)
        assert bool((got[none] == 7.0).all())
        far = ((got[:, cols].double() - want).abs() - (eps * want.abs() + self.sum * U * size * (1 + eps)))[~none]
        assert float(far.max()) <= 0, float(far.max())


@pytest.mark.parametrize("out_type", [BF16, F32])
@pytest.mark.parametrize("c", M.CASES, ids=M.name)
def test_cases(choose, c, out_type):
    assert M.taken_by(choose, c) == (c["op"], c["mx"]) + c["takes"]
    call = Call(c)
    out = call.run(out_type)
    call.check(out)
    assert torch.equal(call.run(out_type), out)


ALIKE = [c for i, c in enumerate(M.CASES) if c["K"] >= 160 and c["N"] >= 37 and c["takes"] not in [d["takes"] for d in M.CASES[:i] if d["K"] >= 160 and d["N"] >= 37
                                                                                                  and (d["op"], d["mx"]) == (c["op"], c["mx"])]]


@pytest.mark.parametrize("c", ALIKE, ids=M.name)
def test_nan_stays_with_its_row(c):
    """NaN in a row of no expert and in one of an expert's, in the last block of both sides, and in one output's weights"""
    call = Call(c)
    clean = call.run(F32)
    e = max(range(len(c["counts"])), key=lambda e: c["counts"][e])
    bad = int(call.offsets[e]) + c["counts"][e] - 1
    other = next(i for i in reversed(range(len(c["counts"]))) if i != e and c["counts"][i])
    o, n = int(call.offsets[other]), c["counts"][other]
    for row in (0, bad):
        if c["mx"]:
            call.scales[row, c["K"] // 32 - 1] = 255
        else:
            call.rows[row, call.sum - 1] = math.nan
    call.ws[other, c["N"] - 1, c["K"] // 32 - 1] = 255
    out, want = call.run(F32), torch.zeros_like(clean, dtype=torch.bool)
    want[bad] = True
    if call.grad:
        want[o:o + n, c["K"] - 32:] = True
    else:
        want[o:o + n, c["N"] - 1] = True
    assert torch.equal(torch.isnan(out), want)
    assert torch.equal(out[~want], clean[~want])


@pytest.mark.parametrize("c", ALIKE, ids=M.name)
def test_counts_that_do_not_fit_the_matrix(c):
    """what lies outside is not done, and nothing outside is touched"""
    call = Call(c)
    n, E = call.rows.shape[0], len(c["counts"])
    i32 = dict(dtype=torch.int32, device="cuda")
    call.offsets, call.counts = torch.full((E + 1,), n, **i32), torch.full((E,), 5, **i32)
    call.offsets[:3], call.counts[:3] = torch.tensor([0, -5, n - 3], **i32), torch.tensor([2, 400, 2 ** 31 - 1], **i32)
    whole = torch.full((n + 600, call.width), 7.0, device="cuda")
    out = whole[300:300 + n]
    if call.grad:
        X.product_grad(call.rows, call.offsets, call.counts, call.wc, call.ws, out)
    else:
        X.product(call.rows, call.offsets, call.counts, call.wc, call.ws, out, row_scales=call.scales)
    done = torch.zeros(n + 600, dtype=torch.bool, device="cuda")
    done[300:302], done[300 + n - 3:300 + n] = True, True
    assert bool((whole[~done] == 7.0).all()) and not bool((whole[done] == 7.0).all(dim=1).any())


@pytest.mark.parametrize("out_type", [BF16, F32])
@pytest.mark.parametrize("gap,shift", [(1, 0), (0, 1), (8, 0)])
@pytest.mark.parametrize("c", ALIKE, ids=M.name)
def test_outputs_at_any_stride(c, gap, shift, out_type):
    """the kernel is the same wherever its outputs go, and so are their bits; what lies between rows is left"""
    call = Call(c)
    want = call.run(out_type)
    whole = torch.full((want.shape[0] * (call.width + gap) + shift,), 7.0, dtype=out_type, device="cuda")
    out = whole[shift:].view(want.shape[0], call.width + gap)[:, :call.width]
    if call.grad:
        X.product_grad(call.rows, call.offsets, call.counts, call.wc, call.ws, out)
    else:
        X.product(call.rows, call.offsets, call.counts, call.wc, call.ws, out, row_scales=call.scales)
    assert torch.equal(out, want)
    out.fill_(7.0)
    assert bool((whole == 7.0).all())
