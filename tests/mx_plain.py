"""Plain forms, in 64 bits, of the operators on rows in 4-bit floating point, for the tests."""
import torch

SIZES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def values(codes, scales):
    """float64 [..., columns] of codes [..., columns / 2] and scales [..., columns / 32]"""
    codes, scales = codes.cpu().long(), scales.cpu()
    nibbles = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2)
    v = SIZES[nibbles & 7] * (1 - 2 * (nibbles >> 3)).double()
    power = torch.where(scales == 255, torch.nan, torch.exp2(scales.double() - 127))
    return (v.unflatten(-1, (-1, 32)) * power[..., None]).flatten(-2)


def quantize(x):
    """(codes, scales) uint8 of x [..., columns]: each number's nearest size, by its distances to all of them"""
    x = x.cpu().double().unflatten(-1, (-1, 32))
    top = x.abs().amax(dim=-1)
    fine = torch.isfinite(top)
    exponent = torch.frexp(torch.where(fine & (top > 0), top, 2.0 ** -140)).exponent - 1 - 2
    exponent = exponent.clamp(min=-127)
    scales = torch.where(fine, exponent + 127, 255)
    v = torch.where(fine[..., None], x, 0.0) * torch.exp2(-exponent.double())[..., None]
    far = (v.abs()[..., None] - SIZES).abs()
    near = far.amin(dim=-1, keepdim=True)
    # of two sizes as near as each other the even one
    code = torch.where(far == near, torch.arange(8) + 8 * (torch.arange(8) % 2), 99).amin(dim=-1) % 8
    code = torch.where(torch.signbit(x) & fine[..., None], code + 8, code).flatten(-2).unflatten(-1, (-1, 2))
    return (code[..., 0] + 16 * code[..., 1]).to(torch.uint8), scales.to(torch.uint8)


def random_weights(E, N, K, seed, spread=3):
    """codes and scales of weights about 2^-5, on the GPU"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 256, (E, N, K // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.randint(121 - spread, 122 + spread, (E, N, K // 32), generator=g, device="cuda", dtype=torch.uint8)
    return codes, scales


def groups(counts, align=1, ahead=0):
    """(offsets int32 [E + 1], counts int32 [E], rows) of groups of these sizes, the first at row `ahead`"""
    offsets = [ahead]
    for c in counts:
        offsets.append(offsets[-1] + -(-c // align) * align)
    i32 = dict(dtype=torch.int32, device="cuda")
    return torch.tensor(offsets, **i32), torch.tensor(counts, **i32), offsets[-1]


def products(x, offsets, counts, w, transposed=False):
    """(products, sums of their terms' magnitudes), 64 bits: rows of x times their expert's w [E][N][K]; other rows are NaN"""
    out = torch.full((x.shape[0], w.shape[2 if transposed else 1]), torch.nan, dtype=torch.float64)
    size = out.clone()
    for e, (o, c) in enumerate(zip(offsets.tolist(), counts.tolist())):
        m = w[e] if transposed else w[e].t()
        out[o:o + c] = x[o:o + c] @ m
        size[o:o + c] = x[o:o + c].abs() @ m.abs()
    return out, size
