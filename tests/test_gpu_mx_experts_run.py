"""The operators of experts in 4 bits together, as a block uses them: router within groups, rows by expert, first product, SwiGLU, second
product, rows back by token; served with rows in BF16 and in 4 bits, trained beside frozen experts, captured into a graph.

Tolerances: every BF16 array between two operators is off by half a step, 2^-8 of each number, and the sums over columns average
them; five such arrays one after the other are at most 5 * 2^-8 of the norm, and twice that with what SwiGLU's slope (at most 1.1 per factor)
makes of them.  With rows in 4 bits the plain form takes the operators' own 4-bit rows at both places, as a rounding that falls the
other way there is a whole code."""
import pytest
import torch

from paper_2604_02715_amd import moe_block as M
from paper_2604_02715_amd import mx_experts as X
from tests import mx_plain as plain

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
NORM = 10 * 2.0 ** -8


class Layer:
    """Experts [2 F][H] and [H][F] in 4 bits, and the buffers of one batch"""

    def __init__(self, T, E, K, H, F, seed, align=1):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")
        dev, i32, u8 = dict(device="cuda"), dict(device="cuda", dtype=torch.int32), dict(device="cuda", dtype=torch.uint8)
        self.T, self.E, self.K, self.H, self.F, self.align = T, E, K, H, F, align
        self.x, self.logits, self.bias, self.d_out = rand(T, H).to(BF16), rand(T, E), 0.01 * rand(E), rand(T, H)
        self.w = []
        for n, k in ((2 * F, H), (H, F)):
            codes, scales = torch.empty(E, n, k // 2, **u8), torch.empty(E, n, k // 32, **u8)
            X.quantize(rand(E, n, k) / k ** 0.5, codes, scales)
            self.w += [codes, scales]
        n = M.sorted_rows(T, K, E, align)
        z = lambda *s, **kw: torch.zeros(*s, **(kw or dict(dtype=BF16, device="cuda")))
        self.b = dict(ids=z(T, K, **i32), gates=z(T, K, **dev), offsets=z(E + 1, **i32), counts=z(E, **i32), pair_row=z(T, K, **i32), row_pair=z(n, **i32),
                      rows=z(n, H), gate_up=z(n, 2 * F), h=z(n, F), y=z(n, H), out=z(T, H, **dev), rows4=z(n, H // 2, **u8), rows4s=z(n, H // 32, **u8),
                      h4=z(n, F // 2, **u8), h4s=z(n, F // 32, **u8), d_y=z(n, H), d_gates=z(T, K, **dev), d_h=z(n, F), d_gate_up=z(n, 2 * F),
                      d_rows=z(n, H), d_x=z(T, H, **dev), d_logits=z(T, E, **dev),
                      ws=torch.empty(M.sort_workspace_bytes(T, K, E), **u8))
        self.kw = dict(score="sigmoid", renormalize=True, scale=2.5)

    def forward(self, b, mx):
        M.route(self.logits, b["ids"], b["gates"], bias=self.bias, groups=4, top_groups=2, group_score="top2", **self.kw)
        M.sort_tokens(b["ids"], self.E, b["offsets"], b["counts"], b["pair_row"], b["row_pair"], b["ws"], align=self.align)
        M.dispatch(self.x, b["pair_row"], b["row_pair"], b["rows"])
        by = b["offsets"], b["counts"]
        if mx:
            X.quantize(b["rows"], b["rows4"], b["rows4s"])
            X.product(b["rows4"], *by, *self.w[:2], b["gate_up"], row_scales=b["rows4s"])
        else:
            X.product(b["rows"], *by, *self.w[:2], b["gate_up"])
        X.swiglu(b["gate_up"], b["h"])
        if mx:
            X.quantize(b["h"], b["h4"], b["h4s"])
            X.product(b["h4"], *by, *self.w[2:], b["y"], row_scales=b["h4s"])
        else:
            X.product(b["h"], *by, *self.w[2:], b["y"])
        M.combine(b["y"], b["pair_row"], b["gates"], b["out"])

    def backward(self, b):
        by = b["offsets"], b["counts"]
        M.combine_grad(self.d_out, b["y"], b["pair_row"], b["row_pair"], b["gates"], b["d_y"], b["d_gates"])
        X.product_grad(b["d_y"], *by, *self.w[2:], b["d_h"])
        X.swiglu_grad(b["gate_up"], b["d_h"], b["d_gate_up"])
        X.product_grad(b["d_gate_up"], *by, *self.w[:2], b["d_rows"])
        M.combine(b["d_rows"], b["pair_row"], None, b["d_x"])
        M.route_grad(self.logits, b["ids"], b["d_gates"], b["d_logits"], **self.kw)

    def plain(self, x, logits, ids, mx):
        """The block in 64 bits with these experts chosen; with mx the rows ahead of the products are the ones that b holds in 4 bits."""
        w1, w2 = plain.values(*self.w[:2]), plain.values(*self.w[2:])
        p = torch.gather(torch.sigmoid(logits), 1, ids)
        gates = 2.5 * p / p.sum(dim=1, keepdim=True)
        out = torch.zeros(self.T, self.H, dtype=torch.float64)
        pair_row = self.b["pair_row"].cpu().long()
        for e in range(self.E):
            t, k = (ids == e).nonzero(as_tuple=True)
            if t.numel() == 0:
                continue
            at = pair_row[t, k]
            rows = plain.values(self.b["rows4"].cpu()[at], self.b["rows4s"].cpu()[at]) if mx else x[t]
            g, u = (rows @ w1[e].t()).chunk(2, dim=1)
            h = plain.values(self.b["h4"].cpu()[at], self.b["h4s"].cpu()[at]) if mx else torch.nn.functional.silu(g) * u
            out = out.index_add(0, t, gates[t, k][:, None] * (h @ w2[e].t()))
        return out


def off(got, want):
    return float((got.cpu().double() - want).norm() / want.norm())


SHAPES = [(1, 16, 2, 256, 512, 1), (64, 8, 2, 256, 512, 16), (40, 16, 4, 160, 96, 1), (300, 8, 2, 256, 128, 8)]


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("T,E,K,H,F,align", SHAPES)
def test_served(T, E, K, H, F, align, mx):
    L = Layer(T, E, K, H, F, T, align)
    L.forward(L.b, mx)
    ids = L.b["ids"].cpu().long()
    assert bool((ids >= 0).all())
    assert off(L.b["out"], L.plain(L.x.cpu().double(), L.logits.cpu().double(), ids, mx)) <= NORM


@pytest.mark.parametrize("T,E,K,H,F,align", SHAPES[1:])
def test_trained_beside_frozen_experts(T, E, K, H, F, align):
    L = Layer(T, E, K, H, F, T, align)
    L.forward(L.b, False)
    L.backward(L.b)
    x, logits = L.x.cpu().double().requires_grad_(True), L.logits.cpu().double().requires_grad_(True)
    (L.plain(x, logits, L.b["ids"].cpu().long(), False) * L.d_out.cpu().double()).sum().backward()
    assert off(L.b["d_x"], x.grad) <= 2 * NORM               # back through the same arrays
    assert off(L.b["d_logits"], logits.grad) <= 2 * NORM


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("T,E,K,H,F,align", SHAPES)
def test_captured_and_replayed(T, E, K, H, F, align, mx):
    L = Layer(T, E, K, H, F, T, align)
    captured = {k: torch.zeros_like(v) for k, v in L.b.items()}

    def calls(b):
        L.forward(b, mx)
        L.backward(b)

    calls(L.b)
    torch.cuda.synchronize()
    graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        calls(captured)
    for turn in range(4):
        L.x.copy_(torch.randn(T, H, device="cuda"))           # eager work and new inputs between the replays
        L.logits.copy_(torch.randn(T, E, device="cuda"))
        for b in (L.b, captured):                             # rows of no pair are left as they were: the same in both
            for name in ("gate_up", "h", "y", "d_h", "d_gate_up", "d_rows"):
                b[name].zero_()
        calls(L.b)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name in L.b:
            if name != "ws":
                assert torch.equal(L.b[name], captured[name]), (turn, name)
