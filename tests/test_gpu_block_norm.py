"""fluxmoe_block_norm and fluxmoe_block_norm_grad against plain forms in 64 bits, and the gradients against differences.

Tolerances: u = 2^-24.  The mean of squares over H columns is off by at most d = 8 + log2(H) + 4 roundings (eight columns one
after the other, the rest in a tree; H / threads where a column is taken at a time), its root by half of that, and each
factor adds one: (d + 8) u of r's terms and of n.  A gradient is a difference of two such terms, so its tolerance is taken of
their absolute values.  Sums over T tokens: a workgroup adds up its rows one after the other, then 32 partial sums at a time:
2 T / 256 + 64 roundings at most.  BF16 outputs add 2^-9 of the value (2^-8 here, for values at a tie)."""
import math

import pytest
import torch

from paper_2604_02715_amd import moe_block as M

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def rounding(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else U


def depth(H, vec):
    return 12 + math.log2(H + 1) if vec and H <= 8192 else H / 64 + 16


def strided(t, pad):
    wide = torch.full((t.shape[0], t.shape[1] + pad), 9.0, dtype=t.dtype, device=t.device)
    view = wide[:, pad // 2:pad // 2 + t.shape[1]]
    view.copy_(t)
    return view, wide


def make(T, H, y, residual, weight, gate, post, seed):
    g = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g)
    channels = torch.exp(0.5 * rand(H))
    channels[::97] *= 20
    d = dict(residual=(rand(T, H) * channels).to(TYPES[residual]), y=None if y is None else (0.5 * rand(T, H)).to(TYPES[y]),
             w_pre=(1 + 0.2 * rand(H)).to(TYPES[weight]), w_post=(1 + 0.2 * rand(H)).to(TYPES[weight]) if post else None,
             gate={None: None, "token": rand(T, 1), "channel": 0.5 + 0.2 * rand(H)}[gate])
    if T > 2 and y is not None:
        d["y"][1] = 0.0                                      # rows without anything in them: only eps under the root
        d["residual"][2] = 0.0
        d["y"][2] = 0.0
    return d


def cuda(t):
    return None if t is None else t.cuda()


def double(t):
    return None if t is None else t.double()


def forward_64(d, scale, sigmoid, zero_centred):
    """(r, n, the sum of r's absolute terms)"""
    one = 1.0 if zero_centred else 0.0
    residual, y, gate, w_pre, w_post = (double(d[k]) if not torch.is_tensor(d[k]) or d[k].dtype != torch.float64 else d[k]
                                        for k in ("residual", "y", "gate", "w_pre", "w_post"))
    r, size = residual, residual.abs()
    if y is not None:
        if w_post is not None:
            y = y * (y.square().mean(1, keepdim=True) + EPS).rsqrt() * (w_post + one)
        g = 1.0 if gate is None else torch.sigmoid(gate) if sigmoid else gate
        added = scale * g * y
        r, size = residual + added, residual.abs() + added.abs()
    n = r * (r.square().mean(1, keepdim=True) + EPS).rsqrt() * (w_pre + one)
    return r, n, size


SHAPES = [(1, 2048), (3, 8), (5, 64), (130, 256), (67, 512), (33, 520), (19, 1032), (9, 1544), (40, 4096), (7, 5120), (5, 8192), (3, 8200), (6, 250), (4, 1),
          (3, 2051)]
KINDS = [("f32", "bf16", "bf16", None, False), ("bf16", "f32", "f32", "token", True), ("f32", "f32", "bf16", "channel", True),
         ("bf16", "bf16", "f32", "channel", False), ("bf16", "bf16", "bf16", "token", False), (None, "bf16", "bf16", None, False),
         (None, "f32", "f32", None, False), ("f32", "bf16", "f32", None, True)]


@pytest.mark.parametrize("T,H", SHAPES)
@pytest.mark.parametrize("y,residual,weight,gate,post", KINDS)
@pytest.mark.parametrize("sigmoid,zero_centred,pad", [(False, False, 0), (True, True, 0), (False, False, 7), (True, False, 16)])
def test_forward(T, H, y, residual, weight, gate, post, sigmoid, zero_centred, pad):
    sigmoid = sigmoid and gate is not None
    d = make(T, H, y, residual, weight, gate, post, H + T)
    dev = {k: cuda(v) for k, v in d.items()}
    rt = TYPES[residual]
    out, wide = strided(torch.full((T, H), math.nan, dtype=rt, device="cuda"), pad)
    normed, wide_n = strided(torch.full((T, H), math.nan, dtype=torch.bfloat16, device="cuda"), pad)
    has = y is not None
    M.block_norm(strided(dev["residual"], pad)[0], dev["w_pre"], normed, y=strided(dev["y"], pad)[0] if has else None, gate=dev["gate"],
                 w_post=dev["w_post"], residual_out=out if has else None, eps=EPS, scale=0.7, gate_sigmoid=sigmoid, zero_centred=zero_centred)
    r, n, size = forward_64(d, 0.7, sigmoid, zero_centred)
    tol = (depth(H, pad != 7 and H % 8 == 0) + 8) * U
    if has:
        assert bool(((out.cpu().double() - r).abs() <= tol * size + rounding(rt) * r.abs()).all())
        # in the residual's own place
        again, _ = strided(dev["residual"], pad)
        M.block_norm(again, dev["w_pre"], torch.empty_like(normed), y=dev["y"], gate=dev["gate"], w_post=dev["w_post"], residual_out=again, eps=EPS,
                     scale=0.7, gate_sigmoid=sigmoid, zero_centred=zero_centred)
        if pad == 0:
            assert torch.equal(again, out)
        else:
            assert bool(((again.cpu().double() - r).abs() <= tol * size + rounding(rt) * r.abs()).all())
    # n's error: r's own, relative to r's size, times n / r
    factor = (n / torch.where(r == 0, 1.0, r)).abs()
    rms = (r.square().mean(1, keepdim=True) + EPS).sqrt()
    moved = ((size * size).mean(1, keepdim=True)).sqrt() / rms                 # how the row's mean of squares feels r's errors
    assert bool(((normed.cpu().double() - n).abs() <= 2 * tol * (size * factor + n.abs() * moved) + (2.0 ** -8 + tol) * n.abs()).all())
    if pad:
        assert bool((wide[:, :pad // 2] == 9.0).all()) and bool((wide_n[:, pad // 2 + H:] == 9.0).all())


def gradients_64(d, d_n, d_r, scale, sigmoid, zero_centred):
    """by differentiation at the r that residual_out says"""
    v = {k: None if t is None else t.double().requires_grad_(True) for k, t in d.items()}
    with torch.no_grad():
        added = forward_64(dict(v, residual=torch.zeros_like(v["residual"])), scale, sigmoid, zero_centred)[0]
    v["residual"] = (d["residual"].double() - added).requires_grad_(True)
    r, n, _ = forward_64(v, scale, sigmoid, zero_centred)
    (n * d_n.double()).sum().backward() if d_r is None else ((n * d_n.double()).sum() + (r * d_r.double()).sum()).backward()
    return {k: None if t is None else t.grad for k, t in v.items()}


def run_gradient(d, d_n, d_r, scale, sigmoid, zero_centred, pad=0):
    dev = {k: cuda(v) for k, v in d.items()}
    T, H = d["residual"].shape
    nan = lambda t: None if t is None else torch.full(t.shape, math.nan, dtype=t.dtype, device="cuda")
    nan32 = lambda t: None if t is None else torch.full(t.shape, math.nan, device="cuda")
    put = lambda t: None if t is None else strided(t.cuda(), pad)[0]
    got = dict(residual=put(nan(d["residual"])), y=put(nan(d["y"])), gate=nan32(d["gate"]), w_pre=nan32(d["w_pre"]), w_post=nan32(d["w_post"]))
    ws = torch.full((M.block_norm_grad_workspace_bytes(T, H),), 0xFF, dtype=torch.uint8, device="cuda")
    M.block_norm_grad(put(d["residual"]), dev["w_pre"], put(d_n), got["residual"], got["w_pre"], ws, d_residual_out=put(d_r), y=put(d["y"]),
                      gate=dev["gate"], w_post=dev["w_post"], d_y=got["y"], d_gate=got["gate"], d_w_post=got["w_post"], eps=EPS, scale=scale,
                      gate_sigmoid=sigmoid, zero_centred=zero_centred)
    return got


@pytest.mark.parametrize("T,H", SHAPES + [(1500, 264), (700, 2048), (300, 4100)])
@pytest.mark.parametrize("y,residual,weight,gate,post", KINDS)
@pytest.mark.parametrize("sigmoid,zero_centred,pad", [(False, False, 0), (True, True, 0), (True, False, 7)])
def test_gradient_against_the_formula(T, H, y, residual, weight, gate, post, sigmoid, zero_centred, pad):
    sigmoid = sigmoid and gate is not None
    d = make(T, H, y, residual, weight, gate, post, 7 * H + T)
    g = torch.Generator().manual_seed(T)
    d_n = torch.randn(T, H, generator=g).to(torch.bfloat16)
    d_r = None if zero_centred else torch.randn(T, H, generator=g).to(TYPES[residual])
    got = run_gradient(d, d_n, d_r, 0.7, sigmoid, zero_centred, pad)
    want = gradients_64(d, d_n, d_r, 0.7, sigmoid, zero_centred)
    one = 1.0 if zero_centred else 0.0
    tol = (depth(H, pad != 7 and H % 8 == 0) + 8) * U
    over_t = 2 * T / 256 + 64
    # the sizes of the terms whose sums and differences the gradients are
    r, w = d["residual"].double(), (d["w_pre"].double() + one).abs()
    rstd = (r.square().mean(1, keepdim=True) + EPS).rsqrt()
    h = (r * rstd).abs()
    dn = d_n.double().abs()
    dr = (0.0 if d_r is None else d_r.double().abs()) + rstd * (dn * w + h * (dn * w * h).mean(1, keepdim=True))
    close = lambda name, size, extra=0.0: bool(((got[name].cpu().double() - want[name]).abs() <= 2 * tol * size + extra + 1e-30).all())
    bits = lambda name: rounding(got[name].dtype) * want[name].abs()
    assert close("residual", dr, bits("residual"))
    assert close("w_pre", (dn * h).sum(0) * (1 + over_t * U / tol))
    if y is None:
        return
    v = d["y"].double()
    rstd_y = (v.square().mean(1, keepdim=True) + EPS).rsqrt() if post else torch.ones(T, 1, dtype=torch.float64)
    hy = (v * rstd_y).abs()
    wy = (d["w_post"].double() + one).abs() if post else 1.0
    gv = 1.0 if gate is None else (torch.sigmoid(d["gate"].double()) if sigmoid else d["gate"].double().abs())
    dy = 0.7 * gv * dr
    assert close("y", 2 * (rstd_y * (dy * wy + hy * (dy * wy * hy).mean(1, keepdim=True)) if post else dy), bits("y"))
    if post:
        assert close("w_post", 2 * (dy * hy).sum(0) * (1 + over_t * U / tol))
    if gate == "token":
        assert close("gate", 2 * (dr * hy * wy).sum(1, keepdim=True))
    if gate == "channel":
        assert close("gate", 2 * (dr * hy * wy).sum(0) * (1 + over_t * U / tol))


@pytest.mark.parametrize("gate,post", [(None, False), ("token", True), ("channel", True)])
def test_gradient_against_differences(gate, post):
    """every input moved a little in 64 bits: the slope along a random direction"""
    T, H, step = 4, 24, 1e-5
    d = make(T, H, "f32", "f32", "f32", gate, post, 11)
    g = torch.Generator().manual_seed(3)
    d_n, d_r = torch.randn(T, H, generator=g).to(torch.bfloat16), torch.randn(T, H, generator=g)
    d = {k: (None if v is None else v + 0.05 * torch.sign(v) + 0.01) for k, v in d.items()}      # no empty rows: their slope changes within a step
    r0 = forward_64(d, 0.7, gate is not None, False)[0]
    got = run_gradient(dict(d, residual=r0.float()), d_n, d_r, 0.7, gate is not None, False)

    def value(v):
        r, n, _ = forward_64(v, 0.7, gate is not None, False)
        return ((n * d_n.double()).sum() + (r * d_r.double()).sum()).item()

    for k in d:
        if d[k] is None:
            continue
        way = torch.randn(d[k].shape, generator=g).double()
        up, down = (dict(d, **{k: d[k].double() + s * step * way}) for s in (1, -1))
        slope = (value(up) - value(down)) / (2 * step)
        mine = (got[k].cpu().double() * way).sum().item()
        # residual_out is rounded to 32 bits and the kernel's sums are off by less than 40 u of their terms, of which there are T H, below 100 each
        assert abs(mine - slope) <= 64 * U * 100 * T * H + 1e-5 * abs(slope)


def test_no_tokens():
    empty = torch.empty(0, 64, device="cuda")
    w, n = torch.ones(64, device="cuda"), torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    M.block_norm(empty, w, n, y=empty, residual_out=empty)
    d_w = torch.full((64,), math.nan, device="cuda")
    M.block_norm_grad(empty, w, n, empty, d_w, torch.empty(0, dtype=torch.uint8, device="cuda"))
    assert d_w.abs().sum().item() == 0.0                     # a sum over no tokens


@pytest.mark.parametrize("T,H", [(1, 64), (5, 256), (3, 1000), (2, 4096)])
@pytest.mark.parametrize("gate,post", [(None, False), ("token", True), ("channel", True)])
def test_eps_of_zero(T, H, gate, post):
    """A workgroup's places without a row add nothing to the sums over the tokens, though the root of their mean square is 0."""
    d = make(T, H, "f32", "f32", "f32", gate, post, T)
    d = {k: (None if v is None else v + 0.01 + 0.1 * (v == 0)) for k, v in d.items()}           # no empty rows
    g = torch.Generator().manual_seed(H)
    d_n, d_r = torch.randn(T, H, generator=g).to(torch.bfloat16), torch.randn(T, H, generator=g)
    got = {}
    for eps in (0.0, 1e-12):
        dev = {k: cuda(v) for k, v in d.items()}
        out = {k: None if v is None else torch.full_like(cuda(v), math.nan) for k, v in d.items()}
        ws = torch.full((M.block_norm_grad_workspace_bytes(T, H),), 0xFF, dtype=torch.uint8, device="cuda")
        M.block_norm_grad(dev["residual"], dev["w_pre"], d_n.cuda(), out["residual"], out["w_pre"], ws, d_residual_out=d_r.cuda(), y=dev["y"],
                          gate=dev["gate"], w_post=dev["w_post"], d_y=out["y"], d_gate=out["gate"], d_w_post=out["w_post"], eps=eps)
        r, n = torch.empty(T, H, device="cuda"), torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
        M.block_norm(dev["residual"], dev["w_pre"], n, y=dev["y"], gate=dev["gate"], w_post=dev["w_post"], residual_out=r, eps=eps)
        got[eps] = dict(out, r=r, n=n)
    for k, v in got[0.0].items():
        if v is not None:
            # 1e-12 beside a mean square above 1e-4 moves nothing by more than 1e-8, less than a rounding
            assert bool(torch.isfinite(v).all()), k
            assert bool(((v.float() - got[1e-12][k].float()).abs() <= 2.0 ** -7 * v.float().abs() + 1e-5).all()), k


def test_infinities_stay_in_their_row():
    T, H = 6, 512
    d = {k: cuda(v) for k, v in make(T, H, "f32", "f32", "f32", None, False, 1).items()}
    out, n = torch.empty(T, H, device="cuda"), torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
    M.block_norm(d["residual"], d["w_pre"], n, y=d["y"], residual_out=out)
    d["y"][3, 5], d["y"][4, 6] = math.inf, math.nan
    out2, n2 = torch.empty_like(out), torch.empty_like(n)
    M.block_norm(d["residual"], d["w_pre"], n2, y=d["y"], residual_out=out2)
    rows = [0, 1, 2, 5]
    assert torch.equal(out[rows], out2[rows]) and torch.equal(n[rows], n2[rows])
    assert not bool(torch.isfinite(n2[3, 5])) and bool(torch.isnan(n2[4]).all())


def test_rows_far_apart_pass_32_bit_offsets():
    H, T = 64, 2100
    wide = torch.empty(T, 1 << 20, device="cuda")            # 8.8 GB
    residual = wide[:, :H]
    residual.copy_(torch.randn(T, H, device="cuda"))
    w, y = torch.ones(H, device="cuda"), torch.randn(T, H, device="cuda")
    n, n2 = (torch.empty(T, H, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    out = torch.empty(T, H, device="cuda")
    M.block_norm(residual.contiguous(), w, n, y=y, residual_out=out)
    M.block_norm(residual, w, n2, y=y, residual_out=residual)
    assert torch.equal(n, n2) and torch.equal(out, residual)


def test_the_same_call_gives_the_same_bits_on_any_stream():
    T, H = 2000, 2048
    d = make(T, H, "bf16", "bf16", "bf16", "channel", True, 1)
    dn, dr = torch.randn(T, H).to(torch.bfloat16), torch.randn(T, H).to(torch.bfloat16)
    first = run_gradient(d, dn, dr, 0.7, True, False)
    side = torch.cuda.Stream()
    for s in (torch.cuda.current_stream(), side):
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            again = run_gradient(d, dn, dr, 0.7, True, False)
        s.synchronize()
        assert all(torch.equal(first[k], again[k]) for k in first)


@pytest.mark.parametrize("name", ["residual", "y", "residual_out", "normed"])
def test_expanded_rows_are_refused(name):
    T, H = 4, 64
    t = {k: torch.zeros(T, H, device="cuda") for k in ("residual", "y", "residual_out")}
    t["normed"] = torch.zeros(T, H, dtype=torch.bfloat16, device="cuda")
    t[name] = t[name][:1].expand(T, H)
    with pytest.raises(ValueError, match="rows of %s overlap" % name):
        M.block_norm(t["residual"], torch.zeros(H, device="cuda"), t["normed"], y=t["y"], residual_out=t["residual_out"])
