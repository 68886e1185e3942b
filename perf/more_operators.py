"""Experts in 4-bit floating point with shared scales, and the operators they are used with, as operators, and the cases they
are measured on.

  route         router logits -> experts chosen within the best groups of experts, and their gates
  quantize      rows -> 4-bit codes and a scale for each 32 of them, and back to numbers
  product       rows sorted by expert times their expert's 4-bit weights; rows in BF16 or in 4 bits themselves
  product_grad  its gradient to the rows, the experts being frozen
  swiglu        silu(gate) * up between an expert's two products
  swiglu_grad   its gradient

Shapes are those of paper_2604_02715_amd/inputs.py: hidden 4096 / ffn 14336 / 8 experts / top-2, hidden 2048 / ffn 512 / 512 experts /
top-10, hidden 5120 / ffn 1536 / 160 experts / top-8, and its tiny layer (hidden 256 / ffn 512 / 8 experts / top-2).

A row of numbers in 4 bits (microscaling format MXFP4) is uint8 [columns / 2] codes, an even column in the low half of a byte, and
uint8 [columns / 32] scales.  A code is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6; scale s stands for 2^(s - 127).

The plain forms below are the definitions: elementary operations in 32 bits, each output rounded once.  exact() says the same
again in 64 bits.
"""
import math

import torch

own = False          # True: run() calls the library's operators, otherwise the plain forms
DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
BLOCK = 32           # columns that share a scale
MX = 0.5 + 1 / 32    # bytes of a number in 4 bits, its share of the scale included
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # -- router
        # one decode token over 512 experts in eight groups, sigmoid scores with a balance bias: all launch and latency
        dict(name="route_token", kind="route", tokens=1, experts=512, top_k=10, groups=8, top_groups=4, by="top2", logits="f32",
             score="sigmoid", renormalize=True, masked=0.0),
        # a long prompt's tokens over 160 experts in groups of 20, softmax scores, a few experts switched off
        dict(name="route_prefill", kind="route", tokens=8191, experts=160, top_k=8, groups=8, top_groups=3, by="max", logits="bf16",
             score="softmax", renormalize=True, masked=0.03),
        # -- quantisation, and back
        # a decode batch's activations ahead of a product of two 4-bit operands
        dict(name="quantize_rows", kind="quantize", rows=512, columns=5120, type="bf16"),
        # the down projections of a layer of eight large experts
        dict(name="quantize_weights", kind="quantize", rows=32768, columns=14336, type="bf16"),
        # -- products
        # one decode token's ten experts of 512, gate and up projections: two megabytes of weights are latency
        dict(name="product_token", kind="product", tokens=1, experts=512, top_k=10, out_columns=1024, columns=2048, mx_rows=False,
             out="bf16", align=1, dropped=0.0, law="zipf"),
        # a prompt over few large experts, gate and up projections: bound by matrix products
        dict(name="product_prefill", kind="product", tokens=2048, experts=8, top_k=2, out_columns=28672, columns=4096, mx_rows=False,
             out="bf16", align=1, dropped=0.0, law="uniform"),
        # a decode batch over 160 experts, down projections, groups at multiples of 16 rows: every weight once for three rows
        dict(name="product_mx_decode", kind="product", tokens=64, experts=160, top_k=8, out_columns=5120, columns=1536, mx_rows=True,
             out="f32", align=16, dropped=0.05, law="uniform"),
        # a long prompt over few large experts, down projections, both operands in 4 bits
        dict(name="product_mx_prefill", kind="product", tokens=8191, experts=8, top_k=2, out_columns=4096, columns=14336, mx_rows=True,
             out="bf16", align=1, dropped=0.0, law="uniform"),
        # the gradient of a small training batch through the down projections of 512 experts
        dict(name="product_grad_small", kind="product_grad", tokens=100, experts=512, top_k=10, out_columns=2048, columns=512,
             out="bf16", align=1, dropped=0.0, law="zipf"),
        # the same of a large batch and few large experts
        dict(name="product_grad_large", kind="product_grad", tokens=4096, experts=8, top_k=2, out_columns=4096, columns=14336,
             out="bf16", align=1, dropped=0.0, law="uniform"),
        # -- between the products
        # a prompt's rows
        dict(name="swiglu_prefill", kind="swiglu", rows=4097, columns=14336, type="bf16", out="bf16"),
        # the gradient for a training batch's rows over many experts, 32-bit sums in
        dict(name="swiglu_grad", kind="swiglu_grad", rows=32768, columns=1536, type="f32", out="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _within(case, what):
    """`case` with fewer tokens or rows until it needs no more than the largest listed ones."""
    most = {k: max(work(c)[k] for c in listed()) for k in ("bytes", "flops")}
    while case[what] > 1 and any(work(case)[k] > most[k] for k in most):
        case[what] = max(1, int(case[what] * 0.9))
    return case


def draw(rng):
    kind = rng.choice(["route", "route", "quantize", "product", "product", "product", "product", "product_grad", "product_grad", "swiglu",
                       "swiglu_grad"])
    case = dict(kind=kind)
    if kind == "route":
        experts, top_k, groups, top_groups = rng.choice([(512, 10, 8, 4), (160, 8, 8, 3), (256, 8, 8, 4), (0, 0, 0, 0), (0, 0, 0, 0)])
        if not experts:
            groups = rng.randint(2, 16)
            size = _log_int(rng, 1, 64)
            experts, top_groups = groups * size, rng.randint(1, groups)
            top_k = _log_int(rng, 1, min(16, top_groups * size))
        score = rng.choice(["softmax", "sigmoid"])
        case.update(tokens=_log_int(rng, 1, 16384), experts=experts, top_k=top_k, groups=groups, top_groups=top_groups,
                    by=rng.choice(["max", "top2"]) if score == "sigmoid" else "max", logits=rng.choice(["f32", "bf16"]), score=score,
                    renormalize=rng.random() < 0.6, masked=rng.choice([0.0, 0.0, 0.05]))
        return _within(case, "tokens")
    if kind in ("quantize", "swiglu", "swiglu_grad"):
        columns = rng.choice([256, 512, 1536, 2048, 4096, 5120, 14336, 0, 0, 0])
        if not columns:
            columns = BLOCK * _log_int(rng, 1, 448) if kind == "quantize" else _log_int(rng, 1, 14336)
        case.update(rows=_log_int(rng, 1, 32768), columns=columns, type=rng.choice(["bf16", "f32"]))
        if kind != "quantize":
            case["out"] = rng.choice(["bf16", "f32"])
        return _within(case, "rows")
    # experts, top-k, and outputs and columns of one of their projections
    experts, top_k, n, k = rng.choice([(8, 2, 28672, 4096), (8, 2, 4096, 14336), (512, 10, 1024, 2048), (512, 10, 2048, 512),
                                       (160, 8, 5120, 1536), (160, 8, 5120, 1536), (8, 2, 1024, 256), (8, 2, 256, 512),
                                       (0, 0, 0, 0), (0, 0, 0, 0)])
    if not experts:
        experts = _log_int(rng, 1, 128)
        top_k = _log_int(rng, 1, min(8, experts))
        n, k = _log_int(rng, 1, 4096), BLOCK * _log_int(rng, 1, 128)
    # an odd count of outputs now and then
    case.update(tokens=_log_int(rng, 1, 8192), experts=experts, top_k=top_k, out_columns=max(1, n - rng.choice([0, 0, 0, 1, 7])), columns=k)
    if kind == "product":
        case["mx_rows"] = rng.random() < 0.5
    case.update(out=rng.choice(["bf16", "bf16", "f32"]), align=rng.choice([1, 1, 16]), dropped=rng.choice([0.0, 0.0, 0.1]),
                law=rng.choice(["zipf", "uniform"]))
    return _within(case, "tokens")


# ------------------------------------------------------------------------------------------ inputs
def _generator(seed, what):
    g = torch.Generator(device=DEVICE)
    g.manual_seed((seed * 1000003 + sum(ord(c) * 257 ** i for i, c in enumerate(what))) & 0x7FFFFFFFFFFFFFFF)
    return g


def _randn(seed, what, *shape):
    return torch.randn(*shape, generator=_generator(seed, what), device=DEVICE)


def _rand(seed, what, *shape):
    return torch.rand(*shape, generator=_generator(seed, what), device=DEVICE)


class State:
    def __init__(self, **kw):
        self.__dict__.update(kw)


def prepare(case, seed):
    return globals()["_prepare_" + case["kind"].replace("_grad", "")](case, seed)


def run(state):
    return globals()[("_own_" if own else "_plain_") + state.kind](state)


def _prepare_route(case, seed):
    T, E, K = case["tokens"], case["experts"], case["top_k"]
    # what a router gives: N(0, 1) around a popularity of its own for each expert; switched-off experts at minus infinity
    logits = _randn(seed, "logits", T, E) + 0.7 * _randn(seed, "popularity", E)
    off = _rand(seed, "masked", E) < case["masked"]
    off[0] = False
    # balance biases move in steps of 0.001
    bias = (_randn(seed, "bias", E) * 30).round() * 0.001 if case["score"] == "sigmoid" else None
    return State(kind="route", logits=logits.masked_fill_(off, -math.inf).to(TYPES[case["logits"]]), bias=bias, K=K, score=case["score"],
                 groups=case["groups"], top_groups=case["top_groups"], by=case["by"], renormalize=case["renormalize"],
                 scale=2.5 if bias is not None else 1.0, ids=torch.empty(T, K, dtype=torch.int32, device=DEVICE),
                 gates=torch.empty(T, K, device=DEVICE))


def _rows(seed, what, rows, columns):
    """Activations: some columns are much larger than the others."""
    channels = torch.exp(0.5 * _randn(seed, what + " channels", columns)) * (1.0 + 20.0 * (_rand(seed, what + " large", columns) < 2e-3))
    return _randn(seed, what, rows, columns).mul_(channels)


def _mx(x):
    """uint8 [..., columns / 2] codes and uint8 [..., columns / 32] scales of FP32 rows"""
    values, scale, _ = _to_mx(x)
    size = values.abs()
    code = torch.where(size < 2, size * 2, torch.where(size < 4, size + 2, size / 2 + 4)).to(torch.uint8)
    code += 8 * torch.signbit(values).to(torch.uint8)
    code = code.flatten(-2).unflatten(-1, (-1, 2))
    return code[..., 0] + 16 * code[..., 1], scale


def _mx_weights(case, seed):
    """[experts][outputs] rows of weights in 4 bits: N(0, 0.02^2), a size of its own to each output; made some experts at a time"""
    E, N, K = case["experts"], case["out_columns"], case["columns"]
    codes = torch.empty(E, N, K // 2, dtype=torch.uint8, device=DEVICE)
    scales = torch.empty(E, N, K // BLOCK, dtype=torch.uint8, device=DEVICE)
    some = max(1, (1 << 27) // (N * K))
    for e in range(0, E, some):
        n = min(some, E - e)
        w = _randn(seed, "weights %d" % e, n, N, K).mul_(0.02 * torch.exp(0.5 * _randn(seed, "outputs %d" % e, n, N, 1)))
        codes[e:e + n], scales[e:e + n] = _mx(w)
    return codes, scales


def _prepare_quantize(case, seed):
    R, C, dtype = case["rows"], case["columns"], TYPES[case["type"]]
    u8 = dict(dtype=torch.uint8, device=DEVICE)
    return State(kind="quantize", x=_rows(seed, "x", R, C).to(dtype), codes=torch.empty(R, C // 2, **u8),
                 scales=torch.empty(R, C // BLOCK, **u8), values=torch.empty(R, C, dtype=dtype, device=DEVICE))


def _prepare_product(case, seed):
    T, K, E = case["tokens"], case["top_k"], case["experts"]
    # distinct experts of each token, drawn evenly or by popularity rank^-1.1; pairs that are dropped have none
    key = -torch.log(-torch.log(_rand(seed, "pairs", T, E).clamp_(1e-7, 1 - 1e-6)))
    if case["law"] == "zipf":
        rank = torch.empty(E, device=DEVICE)
        rank[torch.argsort(_rand(seed, "ranks", E))] = torch.arange(1, E + 1, device=DEVICE, dtype=torch.float32)
        key -= 1.1 * torch.log(rank)
    ids = torch.topk(key, K, dim=1).indices
    ids = ids[_rand(seed, "dropped", T, K) >= case["dropped"]]
    # the order that sort_tokens gives them: each expert's rows together, its first row at a multiple of `align`
    counts = torch.bincount(ids, minlength=E)
    ends = torch.cumsum((counts + case["align"] - 1) // case["align"] * case["align"], 0)
    offsets = torch.cat([ends.new_zeros(1), ends])
    n = T * K + min(E, T * K) * (case["align"] - 1)
    w_codes, w_scales = _mx_weights(case, seed)
    s = State(kind=case["kind"], offsets=offsets.to(torch.int32), counts=counts.to(torch.int32), w_codes=w_codes, w_scales=w_scales,
              row_scales=None)
    # for the plain form: the experts that have rows, and where their rows are (n: a place that no row has)
    s.used = counts.nonzero().squeeze(1)
    at = torch.arange(int(counts.max()), device=DEVICE)[None]
    s.place = torch.where(at < counts[s.used][:, None], offsets[s.used][:, None] + at, n)
    if case["kind"] == "product_grad":
        s.d_out = _randn(seed, "d_out", n, case["out_columns"]).to(torch.bfloat16)
        s.d_rows = torch.zeros(n, case["columns"], dtype=TYPES[case["out"]], device=DEVICE)
        return s
    s.rows = _rows(seed, "rows", n, case["columns"])
    if case["mx_rows"]:
        s.rows, s.row_scales = _mx(s.rows)
    else:
        s.rows = s.rows.to(torch.bfloat16)
    s.out = torch.zeros(n, case["out_columns"], dtype=TYPES[case["out"]], device=DEVICE)
    return s


def _prepare_swiglu(case, seed):
    R, F, dtype, out = case["rows"], case["columns"], TYPES[case["type"]], TYPES[case["out"]]
    s = State(kind=case["kind"], gate_up=(2.0 * _randn(seed, "gate_up", R, 2 * F)).to(dtype))
    if case["kind"] == "swiglu":
        s.h = torch.empty(R, F, dtype=out, device=DEVICE)
    else:
        s.d_h = _randn(seed, "d_h", R, F).to(out)
        s.d_gate_up = torch.empty_like(s.gate_up)
    return s


# ------------------------------------------------------------------------------------------ the library's operators
def _own_route(s):
    from paper_2604_02715_amd import moe_block as M
    M.route(s.logits, s.ids, s.gates, bias=s.bias, scale=s.scale, score=s.score, renormalize=s.renormalize, groups=s.groups,
            top_groups=s.top_groups, group_score=s.by)
    return {"ids": s.ids, "gates": s.gates}


def _own_quantize(s):
    from paper_2604_02715_amd import mx_experts as X
    X.quantize(s.x, s.codes, s.scales)
    X.dequantize(s.codes, s.scales, s.values)
    return {"values": s.values}


def _own_product(s):
    from paper_2604_02715_amd import mx_experts as X
    X.product(s.rows, s.offsets, s.counts, s.w_codes, s.w_scales, s.out, row_scales=s.row_scales)
    return {"out": s.out}


def _own_product_grad(s):
    from paper_2604_02715_amd import mx_experts as X
    X.product_grad(s.d_out, s.offsets, s.counts, s.w_codes, s.w_scales, s.d_rows)
    return {"d_rows": s.d_rows}


def _own_swiglu(s):
    from paper_2604_02715_amd import mx_experts as X
    X.swiglu(s.gate_up, s.h)
    return {"h": s.h}


def _own_swiglu_grad(s):
    from paper_2604_02715_amd import mx_experts as X
    X.swiglu_grad(s.gate_up, s.d_h, s.d_gate_up)
    return {"d_gate_up": s.d_gate_up}


# ------------------------------------------------------------------------------------------ plain forms
def _plain_route(s):
    logits = s.logits.float()
    off = torch.isneginf(logits)
    scores = 1.0 / (1.0 + torch.exp(-logits)) if s.score == "sigmoid" else logits
    key = (scores if s.bias is None else scores + s.bias).masked_fill(off, -math.inf)
    # a group's score: its best key, or the sum of its two best (of one where there is no second)
    by_group = torch.sort(key.unflatten(1, (s.groups, -1)), dim=2, descending=True).values
    group = by_group[..., 0]
    if s.by == "top2" and by_group.shape[2] > 1:
        second = by_group[..., 1]
        group = group + torch.where(torch.isneginf(second), 0.0, second)
    best = torch.sort(group, dim=1, descending=True, stable=True).indices[:, :s.top_groups]   # equal scores: the lower group first
    kept = torch.zeros_like(group, dtype=torch.bool).scatter_(1, best, True)
    key = key.masked_fill(kept.logical_not().repeat_interleave(key.shape[1] // s.groups, dim=1), -math.inf)
    order = torch.sort(key, dim=1, descending=True, stable=True)
    ids = order.indices[:, :s.K]
    chosen = torch.isneginf(order.values[:, :s.K]).logical_not()
    if s.score == "softmax":
        scores = torch.exp(logits - logits.amax(dim=1, keepdim=True))
    gates = torch.where(chosen, torch.gather(scores, 1, ids), 0.0)
    if s.renormalize:
        total = gates.sum(dim=1, keepdim=True)
        gates = gates / torch.where(total == 0, 1.0, total)
    elif s.score == "softmax":
        gates = gates / scores.sum(dim=1, keepdim=True)
    return {"ids": torch.where(chosen, ids, -1).to(torch.int32), "gates": gates * s.scale}


def _power(scale):
    """2^(scale - 127) of integers 0 to 255 (255: not a number), from the bits"""
    bits = torch.where(scale == 0, 1 << 22, torch.where(scale == 255, 0x7FC00000, scale << 23))
    return bits.view(torch.float32)


def _to_mx(x):
    """(the codes' values [..., blocks][32], scales uint8 [..., blocks], what the scales stand for)"""
    x = x.float().unflatten(-1, (-1, BLOCK))
    top = x.abs().amax(dim=-1)
    exponent = torch.frexp(top).exponent - 1                             # floor of the logarithm
    exponent = torch.where(top > 0, exponent, -127).to(torch.int32)
    scale = torch.where(torch.isfinite(top), (exponent - 2 + 127).clamp_(min=0), 255)
    x = x * _power(254 - scale.clamp(max=254))[..., None]
    size = x.abs()
    step = torch.where(size < 2, 0.5, torch.where(size < 4, 1.0, 2.0))
    size = (torch.round(size / step) * step).clamp_(max=6.0)             # halves go to the even code
    return torch.copysign(size, x), scale.to(torch.uint8), _power(scale)


def _plain_quantize(s):
    values, _, power = _to_mx(s.x)
    return {"values": (values * power[..., None]).flatten(-2).to(s.values.dtype)}


def _from_mx(codes, scales):
    """FP32 rows of codes and scales"""
    table = torch.tensor([sign * m for sign in (1.0, -1.0) for m in MAGNITUDES], device=codes.device)
    codes = codes.to(torch.int32)
    values = table[torch.stack([codes & 15, codes >> 4], dim=-1)].flatten(-2)
    return (values.unflatten(-1, (-1, BLOCK)) * _power(scales.to(torch.int32))[..., None]).flatten(-2)


def _at(rows, s):
    """[used experts][most rows of one][columns]: each expert's rows, 0 where it has fewer"""
    return torch.cat([rows, rows.new_zeros(1, rows.shape[1])])[s.place]


def _back(y, s, like):
    """rows of `like` with each expert's results in their places, the others 0"""
    out = y.new_zeros(like.shape[0] + 1, y.shape[2])
    out[s.place.flatten()] = y.flatten(0, 1)
    return out[:-1].to(like.dtype)


def _plain_product(s):
    rows = s.rows.float() if s.row_scales is None else _from_mx(s.rows, s.row_scales)
    w = _from_mx(s.w_codes[s.used], s.w_scales[s.used])
    return {"out": _back(torch.matmul(_at(rows, s), w.transpose(1, 2)), s, s.out)}


def _plain_product_grad(s):
    w = _from_mx(s.w_codes[s.used], s.w_scales[s.used])
    return {"d_rows": _back(torch.matmul(_at(s.d_out.float(), s), w), s, s.d_rows)}


def _plain_swiglu(s):
    gate, up = s.gate_up.float().chunk(2, dim=1)
    return {"h": (gate / (1.0 + torch.exp(-gate)) * up).to(s.h.dtype)}


def _plain_swiglu_grad(s):
    gate, up = s.gate_up.float().chunk(2, dim=1)
    d_h = s.d_h.float()
    p = 1.0 / (1.0 + torch.exp(-gate))
    d_gate = d_h * up * p * (1.0 + gate * (1.0 - p))
    return {"d_gate_up": torch.cat([d_gate, d_h * gate * p], dim=1).to(s.gate_up.dtype)}


# ------------------------------------------------------------------------------------------ what a pass needs, and how exact it is
def _used(case):
    """Experts that have rows: all that the pairs can reach, or about as many as even draws reach."""
    E, pairs = case["experts"], case["tokens"] * case["top_k"] * (1.0 - case["dropped"])
    return min(pairs, E * (1.0 - math.exp(-pairs / E)) if pairs > case["top_k"] else pairs)


def work(case):
    """Each input read once and each output written once; of the weights those of the experts that have rows."""
    kind = case["kind"]
    if kind == "route":
        T, E = case["tokens"], case["experts"]
        return {"bytes": T * E * BYTES[case["logits"]] + 8 * T * case["top_k"] + (4 * E if case["score"] == "sigmoid" else 0), "flops": 5 * T * E}
    if kind == "quantize":
        el = case["rows"] * case["columns"]
        return {"bytes": el * (2 * BYTES[case["type"]] + MX), "flops": 6 * el}
    if kind.startswith("swiglu"):
        el, t, o = case["rows"] * case["columns"], BYTES[case["type"]], BYTES[case["out"]]
        return {"bytes": el * (2 * t + o), "flops": 8 * el} if kind == "swiglu" else {"bytes": el * (4 * t + o), "flops": 15 * el}
    N, K, out = case["out_columns"], case["columns"], BYTES[case["out"]]
    rows = case["tokens"] * case["top_k"] * (1.0 - case["dropped"])
    moved = N * 2 + K * out if kind == "product_grad" else K * (MX if case["mx_rows"] else 2) + N * out
    return {"bytes": rows * moved + _used(case) * N * K * MX + 8 * case["experts"], "flops": 2 * rows * N * K}


def exact(case, seed):
    s = prepare(case, seed)
    return globals()["_exact_" + case["kind"]](s)


def _exact_route(s):
    # which experts are chosen is decided on scores held in 32 bits
    l = s.logits.float()
    T, E = l.shape
    key = l if s.score == "softmax" else (1.0 + torch.exp(-l)).reciprocal() + s.bias
    key = torch.where(l == -math.inf, torch.full_like(key, -math.inf), key)
    kept = []
    for g in range(s.groups):
        part = torch.topk(key[:, g * (E // s.groups):(g + 1) * (E // s.groups)], min(2, E // s.groups), dim=1).values
        of_two = s.by == "top2" and part.shape[1] > 1
        kept.append(part[:, 0] + torch.where(part[:, 1] > -math.inf, part[:, 1], 0.0) if of_two else part[:, 0])
    order = torch.argsort(torch.argsort(-torch.stack(kept, 1), dim=1, stable=True), dim=1)      # a group's place
    key = torch.where((order < s.top_groups)[:, torch.arange(E, device=DEVICE) // (E // s.groups)], key, -math.inf)
    ids = torch.argsort(-key, dim=1, stable=True)[:, :s.K]
    p = torch.sigmoid(l.double()) if s.score == "sigmoid" else torch.softmax(l.double(), dim=1)
    taken = torch.take_along_dim(p, ids, dim=1) * (torch.take_along_dim(key, ids, dim=1) != -math.inf)
    if s.renormalize:
        taken = taken / taken.sum(dim=1, keepdim=True).clamp(min=1e-300)
    return {"ids": None, "gates": taken * s.scale}


def _exact_quantize(s):
    """Each number's nearest code by the borders between them; a number on a border goes to the even code."""
    size = torch.tensor(MAGNITUDES, dtype=torch.float64, device=DEVICE)
    border = (size[1:] + size[:-1]) / 2
    out = torch.empty(s.x.shape, dtype=torch.float64, device=DEVICE)
    for r in range(0, s.x.shape[0], 2048):
        x = s.x[r:r + 2048].double().view(-1, BLOCK)
        top = x.abs().amax(dim=1, keepdim=True)
        unit = torch.exp2(torch.floor(torch.log2(top.clamp(min=2.0 ** -149))) - 2)
        unit = torch.where(unit * 8 <= top, unit * 2, torch.where(unit * 4 > top, unit / 2, unit)).clamp(min=2.0 ** -127)
        v = (x / unit).abs()
        low, high = torch.bucketize(v, border), torch.bucketize(v, border, right=True)
        code = torch.where(low % 2 == 0, low, high)
        out[r:r + 2048] = (size[code] * torch.sign(x) * unit).view(-1, s.x.shape[1])
    return {"values": out}


def _values_64(codes, scales):
    codes = codes.long()
    sign = 1.0 - 2.0 * torch.stack([codes >> 3 & 1, codes >> 7], dim=-1)
    m = torch.stack([codes & 7, codes >> 4 & 7], dim=-1)
    size = torch.where(m < 2, m * 0.5, (1.0 + 0.5 * (m & 1)) * torch.exp2((m >> 1) - 1.0))
    return (sign * size).double().flatten(-2) * torch.exp2(scales.double() - 127).repeat_interleave(BLOCK, dim=-1)


def _by_expert(s, rows, columns, transposed):
    """64-bit products of the rows (rows.get gives a slice of rows.n) with their experts' weights"""
    offsets, counts = s.offsets.tolist(), s.counts.tolist()
    out = torch.zeros(rows.n, columns, dtype=torch.float64, device=DEVICE)
    for e, c in enumerate(counts):
        if c:
            w = _values_64(s.w_codes[e], s.w_scales[e])
            at = slice(offsets[e], offsets[e] + c)
            out[at] = rows.get(at) @ (w if transposed else w.t().contiguous())
    return out


class _Slices:
    def __init__(self, n, get):
        self.n, self.get = n, get


def _exact_product(s):
    if s.row_scales is None:
        rows = _Slices(s.rows.shape[0], lambda at: s.rows[at].double())
    else:
        rows = _Slices(s.rows.shape[0], lambda at: _values_64(s.rows[at], s.row_scales[at]))
    return {"out": _by_expert(s, rows, s.out.shape[1], False)}


def _exact_product_grad(s):
    return {"d_rows": _by_expert(s, _Slices(s.d_out.shape[0], lambda at: s.d_out[at].double()), s.d_rows.shape[1], True)}


def _exact_swiglu(s):
    F = s.h.shape[1]
    gate, up = s.gate_up[:, :F].double(), s.gate_up[:, F:].double()
    return {"h": torch.sigmoid(gate) * gate * up}


def _exact_swiglu_grad(s):
    """By differentiation, some rows at a time."""
    F, out = s.d_h.shape[1], torch.empty(s.gate_up.shape, dtype=torch.float64, device=DEVICE)
    for r in range(0, out.shape[0], 4096):
        x = s.gate_up[r:r + 4096].double().requires_grad_(True)
        h = x[:, :F] / (1.0 + torch.exp(-x[:, :F])) * x[:, F:]
        (h * s.d_h[r:r + 4096].double()).sum().backward()
        out[r:r + 4096] = x.grad
    return {"d_gate_up": out}
