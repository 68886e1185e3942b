"""fluxmoe_sort_tokens, fluxmoe_dispatch, fluxmoe_combine and fluxmoe_combine_grad against plain forms: the order exactly, sums
and gradients in 64 bits.

Tolerances: u = 2^-24.  A sum of K products has K roundings of its own and K of the products, each at most u of the sum of
absolute terms; a dot product over H columns at most (8 + log2(H)) + 1 of them, as eight columns are added one after the other
and the rest in a tree.  A BF16 output adds 2^-9 of the value (2^-8 here, for sums at a tie)."""
import math

import pytest
import torch

from paper_2604_02715_amd import moe_block as M

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def rounding(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else U


def make_ids(T, K, E, seed, dropped=0.0, skew=False):
    g = torch.Generator().manual_seed(seed)
    key = torch.rand(T, E, generator=g)
    if skew:
        key = key - torch.log(torch.arange(1, E + 1))[None] * 0.5
    ids = torch.topk(key, K, dim=1).indices.to(torch.int32)
    ids[torch.rand(T, K, generator=g) < dropped] = -1
    return ids


def plain_order(ids, E, align, cap):
    """offsets, counts, pair_row, row_pair as Python lists"""
    flat = ids.reshape(-1).tolist()
    groups = [[] for _ in range(E)]
    for p, e in enumerate(flat):
        if 0 <= e < E:
            groups[e].append(p)
    offsets, pair_row, row_pair, at = [], [-1] * len(flat), [-1] * cap, 0
    for g in groups:
        offsets.append(at)
        for i, p in enumerate(g):
            pair_row[p], row_pair[at + i] = at + i, p
        at += -(-len(g) // align) * align
    return offsets + [at], [len(g) for g in groups], pair_row, row_pair


def run_order(ids, E, align=1, more=0):
    T, K = ids.shape
    cap = M.sorted_rows(T, K, E, align) + more
    i32 = dict(dtype=torch.int32, device="cuda")
    o = dict(offsets=torch.full((E + 1,), -9, **i32), counts=torch.full((E,), -9, **i32), pair_row=torch.full((T, K), -9, **i32),
             row_pair=torch.full((cap,), -9, **i32))
    ws = torch.full((M.sort_workspace_bytes(T, K, E),), 0xA5, dtype=torch.uint8, device="cuda")
    M.sort_tokens(ids.cuda(), E, workspace=ws, align=align, **o)
    return o


@pytest.mark.parametrize("T,K,E", [(1, 1, 1), (1, 10, 512), (3, 2, 8), (64, 4, 64), (65, 4, 64), (100, 10, 512), (127, 8, 160), (512, 8, 160),
                                   (1024, 4, 5), (410, 10, 1024), (400, 10, 1025), (256, 16, 2048), (33, 8, 2049), (500, 8, 4096),
                                   (513, 8, 160), (4097, 1, 3), (2049, 2, 8), (6000, 10, 512), (3000, 8, 513), (1111, 64, 300), (70000, 1, 2)])
@pytest.mark.parametrize("align,dropped", [(1, 0.0), (16, 0.0), (1, 0.3), (7, 0.1)])
def test_order(T, K, E, align, dropped):
    ids = make_ids(T, K, E, T + K + E, dropped, skew=T % 2 == 0)
    o = run_order(ids, E, align)
    want = plain_order(ids, E, align, o["row_pair"].numel())
    for name, w in zip(("offsets", "counts", "pair_row", "row_pair"), want):
        assert o[name].reshape(-1).cpu().tolist() == w, name


@pytest.mark.parametrize("T,K", [(40, 3), (3000, 3)])
def test_order_of_odd_batches(T, K):
    """everything to one expert, everything dropped, ids out of range, a larger row_pair than needed"""
    E = 9
    odd = make_ids(T, K, E, 1)
    odd[::3, 0], odd[1::3, 1] = 1 << 30, -5
    for ids in (torch.full((T, K), 4, dtype=torch.int32), torch.full((T, K), -1, dtype=torch.int32), odd):
        o = run_order(ids, E, 16, more=37)
        want = plain_order(ids, E, 16, o["row_pair"].numel())
        for name, w in zip(("offsets", "counts", "pair_row", "row_pair"), want):
            assert o[name].reshape(-1).cpu().tolist() == w, name


def test_no_tokens():
    o = run_order(torch.empty(0, 4, dtype=torch.int32), 6, 1, more=3)
    assert o["offsets"].tolist() == [0] * 7 and o["counts"].tolist() == [0] * 6 and o["row_pair"].tolist() == [-1] * 3
    rows = torch.full((3, 64), 2.0, device="cuda")
    M.dispatch(torch.empty(0, 64, device="cuda"), o["pair_row"], o["row_pair"], rows)
    assert rows.abs().sum().item() == 0.0
    M.combine(rows, o["pair_row"], None, torch.empty(0, 64, device="cuda"))


def strided(t, pad):
    """the same values in rows that are further apart and (pad odd) not aligned"""
    wide = torch.full((t.shape[0], t.shape[1] + pad), 9.0, dtype=t.dtype, device=t.device)
    view = wide[:, pad // 2:pad // 2 + t.shape[1]]
    view.copy_(t)
    return view, wide


SHAPES = [(1, 10, 512, 2048), (5, 2, 8, 8), (37, 3, 8, 250), (64, 8, 160, 520), (130, 10, 64, 1032), (33, 4, 16, 5120), (9, 2, 8, 8192), (5, 3, 8, 8200),
          (7, 2, 4, 1), (300, 1, 12, 264), (3, 64, 100, 96)]


@pytest.mark.parametrize("T,K,E,H", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("align,dropped,pad", [(1, 0.0, 0), (16, 0.25, 0), (1, 0.1, 7), (4, 0.0, 16)])
def test_dispatch_and_its_gradient(T, K, E, H, dtype, align, dropped, pad):
    g = torch.Generator().manual_seed(H + T)
    ids = make_ids(T, K, E, H, dropped)
    o = run_order(ids, E, align)
    pair = o["row_pair"].cpu().long()
    x = torch.randn(T, H, generator=g).to(dtype)
    x_dev, _ = strided(x.cuda(), pad)
    rows, wide = strided(torch.full((pair.numel(), H), math.nan, dtype=dtype, device="cuda"), pad)
    M.dispatch(x_dev, o["pair_row"], o["row_pair"], rows)
    want = torch.where((pair >= 0)[:, None], x[pair.clamp(min=0) // K], torch.zeros((), dtype=dtype))
    assert torch.equal(rows.cpu(), want)
    if pad:
        assert bool((wide[:, :pad // 2] == 9.0).all()) and bool((wide[:, pad // 2 + H:] == 9.0).all())
    # the gradient: the rows' gradients added up by token
    d_rows = torch.randn(pair.numel(), H, generator=g).to(dtype)
    d_x, _ = strided(torch.full((T, H), math.nan, device="cuda"), pad)
    M.combine(strided(d_rows.cuda(), pad)[0], o["pair_row"], None, d_x)
    at = o["pair_row"].cpu().long()
    terms = torch.where((at >= 0)[..., None], d_rows.double()[at.clamp(min=0)], 0.0)
    assert bool(((d_x.cpu().double() - terms.sum(1)).abs() <= 2 * K * U * terms.abs().sum(1)).all())


@pytest.mark.parametrize("T,K,E,H", SHAPES)
@pytest.mark.parametrize("rows_type,out_type", [(torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32),
                                                (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("align,dropped,pad", [(1, 0.0, 0), (16, 0.25, 0), (1, 0.5, 7)])
def test_combine_and_its_gradient(T, K, E, H, rows_type, out_type, align, dropped, pad):
    g = torch.Generator().manual_seed(3 * H + T)
    ids = make_ids(T, K, E, H + 1, dropped)
    if T > 2:
        ids[1] = -1                                          # a token without experts
    o = run_order(ids, E, align)
    n, at = o["row_pair"].numel(), o["pair_row"].cpu().long()
    here = (at >= 0)[..., None]
    rows = torch.randn(n, H, generator=g).to(rows_type)
    rows[o["row_pair"].cpu() < 0] = math.nan                 # nothing reads rows of no pair
    gates = torch.rand(T, K, generator=g)
    gates[~here[..., 0]] = math.inf                          # nor the gates of dropped pairs
    rows_dev = strided(rows.cuda(), pad)[0]
    out, _ = strided(torch.full((T, H), math.nan, dtype=out_type, device="cuda"), pad)
    M.combine(rows_dev, o["pair_row"], gates.cuda(), out)
    terms = torch.where(here, rows.double()[at.clamp(min=0)] * gates.double()[..., None], 0.0)
    want, size = terms.sum(1), terms.abs().sum(1)
    tol = 2 * K * U * size + rounding(out_type) * want.abs()
    assert bool(((out.cpu().double() - want).abs() <= tol).all())
    if T > 2:
        assert out[1].abs().sum().item() == 0.0
    before = torch.randn(T, H, generator=g).to(out_type)
    out.copy_(before)
    M.combine(rows_dev, o["pair_row"], gates.cuda(), out, accumulate=True)
    total = want + before.double()
    assert bool(((out.cpu().double() - total).abs() <= tol + (2 * K * U + rounding(out_type)) * (total.abs() + before.double().abs())).all())

    d_out = torch.randn(T, H, generator=g).to(out_type)
    d_rows, wide = strided(torch.full((n, H), math.nan, dtype=rows_type, device="cuda"), pad)
    d_gates = torch.full((T, K), math.nan, device="cuda")
    M.combine_grad(strided(d_out.cuda(), pad)[0], rows_dev, o["pair_row"], o["row_pair"], gates.cuda(), d_rows, d_gates)
    want_rows = torch.zeros(n, H, dtype=torch.float64)
    full = gates.double()[..., None] * d_out.double()[:, None, :]
    want_rows[at[at >= 0]] = full[at >= 0]
    assert bool(((d_rows.cpu().double() - want_rows).abs() <= rounding(rows_type) * want_rows.abs()).all())
    terms = torch.where(here, rows.double()[at.clamp(min=0)] * d_out.double()[:, None, :], 0.0)
    tol = (9 + math.log2(H + 1)) * U * terms.abs().sum(2) if pad == 0 and H % 8 == 0 and H <= 8192 else (H / 64 + 16) * U * terms.abs().sum(2)
    assert bool(((d_gates.cpu().double() - terms.sum(2)).abs() <= tol).all())
    if pad:
        assert bool((wide[:, :pad // 2] == 9.0).all()) and bool((wide[:, pad // 2 + H:] == 9.0).all())


def test_gradient_against_differences():
    """out is linear in rows and in gates, so a step of any size gives the slope itself."""
    T, K, E, H = 6, 3, 5, 40
    g = torch.Generator().manual_seed(4)
    o = run_order(make_ids(T, K, E, 2, 0.2), E)
    n = o["row_pair"].numel()
    rows, gates, d_out = torch.randn(n, H, generator=g), torch.rand(T, K, generator=g), torch.randn(T, H, generator=g)
    d_rows, d_gates = torch.empty(n, H, device="cuda"), torch.empty(T, K, device="cuda")
    M.combine_grad(d_out.cuda(), rows.cuda(), o["pair_row"], o["row_pair"], gates.cuda(), d_rows, d_gates)

    def value(rows, gates):
        at = o["pair_row"].cpu().long()
        out = torch.where((at >= 0)[..., None], rows[at.clamp(min=0)] * gates[..., None], 0.0).sum(1)
        return (out * d_out.double()).sum()

    rows, gates = rows.double(), gates.double()
    base = value(rows, gates)
    for t in range(T):
        for k in range(K):
            step = gates.clone()
            step[t, k] += 1.0
            assert abs(float(value(rows, step) - base) - float(d_gates[t, k])) <= 16 * U * H * 9
    for r in range(n):
        step = rows.clone()
        step[r, r % H] += 1.0
        assert abs(float(value(step, gates) - base) - float(d_rows[r, r % H])) <= 1e-6


def test_infinite_rows_stay_with_their_token():
    o = run_order(torch.tensor([[0, 1], [1, 0], [0, -1]], dtype=torch.int32), 2)
    rows = torch.ones(6, 64, device="cuda")
    rows[int(o["pair_row"][1, 0])] = math.inf
    rows[5] = math.nan                                       # the row that the dropped pair leaves over
    out = torch.empty(3, 64, device="cuda")
    M.combine(rows, o["pair_row"], torch.ones(3, 2, device="cuda"), out)
    assert bool((out[0] == 2).all()) and bool(torch.isinf(out[1]).all()) and bool((out[2] == 1).all())


def test_rows_behind_two_gigabytes_of_elements():
    """offsets of rows and elements past 32 bits: 4.3 GB of BF16 rows 1 MiB apart"""
    H, n = 64, 4100
    wide = torch.empty(n, 1 << 20, dtype=torch.bfloat16, device="cuda")
    rows = wide[:, :H]
    x = torch.randn(n, H, device="cuda").to(torch.bfloat16)
    order = torch.arange(n, dtype=torch.int32, device="cuda").flip(0).contiguous()
    M.dispatch(x, order.view(n, 1), order, rows)
    assert torch.equal(rows, x.flip(0))
    out = torch.empty(n, H, dtype=torch.bfloat16, device="cuda")
    M.combine(rows, order.view(n, 1), None, out)
    assert torch.equal(out, x)


def test_the_same_call_gives_the_same_bits_on_any_stream():
    ids = make_ids(3001, 8, 160, 5, 0.1, skew=True)
    first = run_order(ids, 160, 16)
    rows = torch.randn(first["row_pair"].numel(), 512, device="cuda").to(torch.bfloat16)
    gates, d_out = torch.rand(3001, 8, device="cuda"), torch.randn(3001, 512, device="cuda")
    outs = []
    streams = [torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.current_stream()]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        out, d_rows, d_gates = torch.empty(3001, 512, device="cuda"), torch.empty_like(rows), torch.empty_like(gates)
        torch.cuda.synchronize()
        M.combine(rows, first["pair_row"], gates, out, stream=s)
        M.combine_grad(d_out, rows, first["pair_row"], first["row_pair"], gates, d_rows, d_gates, stream=s)
        s.synchronize()
        outs.append((out, d_rows, d_gates))
        again = run_order(ids, 160, 16)
        assert all(torch.equal(first[k], again[k]) for k in first)
    for other in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], other))


@pytest.mark.parametrize("H", [1, 8])
def test_more_empty_rows_than_a_launch_has_workgroups_for(H):
    """16 rows to each of 2^20 workgroups, and some more; a column at a time and 16 bytes at a time."""
    T, cap = 3, (1 << 24) + 1000
    row_pair = torch.full((cap,), -1, dtype=torch.int32, device="cuda")
    pair_row = torch.tensor([[5], [cap - 2], [(1 << 24) + 7]], dtype=torch.int32, device="cuda")
    row_pair[pair_row.flatten().long()] = torch.arange(T, dtype=torch.int32, device="cuda")
    x = torch.randn(T, H, device="cuda").to(torch.bfloat16)
    rows = torch.full((cap, H), 7.0, dtype=torch.bfloat16, device="cuda")
    M.dispatch(x, pair_row, row_pair, rows)
    want = torch.zeros_like(rows)
    want[pair_row.flatten().long()] = x
    assert torch.equal(rows, want)
    d_rows, d_gates = torch.full_like(rows, 7.0), torch.empty(T, 1, device="cuda")
    M.combine_grad(x, rows, pair_row, row_pair, torch.ones(T, 1, device="cuda"), d_rows, d_gates)
    assert torch.equal(d_rows, want)
    assert torch.allclose(d_gates[:, 0], x.float().square().sum(1), rtol=1e-6)


@pytest.mark.parametrize("T,K,E", [(3, 2, 8), (100, 10, 512), (300, 8, 160), (3000, 3, 9), (6000, 10, 512)])
@pytest.mark.parametrize("align,first,more", [(1, 1, 0), (128, 1, 2), (128, 2, 5), (100, 3, 3), (1024, 0, 1)])
def test_rows_of_no_pair(T, K, E, align, first, more):
    """Long gaps between the groups; row_pair at any 4-byte address and of any length, and nothing beside it is written."""
    ids = make_ids(T, K, E, 3, 0.1)
    cap = M.sorted_rows(T, K, E, align) + more
    i32 = dict(dtype=torch.int32, device="cuda")
    whole = torch.full((first + cap + 8,), -9, **i32)
    row_pair = whole[first:first + cap]
    o = [torch.empty(E + 1, **i32), torch.empty(E, **i32), torch.empty(T, K, **i32), row_pair]
    M.sort_tokens(ids.cuda(), E, *o, torch.empty(M.sort_workspace_bytes(T, K, E), dtype=torch.uint8, device="cuda"), align=align)
    for got, want in zip(o, plain_order(ids, E, align, cap)):
        assert got.reshape(-1).cpu().tolist() == want
    assert bool((whole[:first] == -9).all()) and bool((whole[first + cap:] == -9).all())
