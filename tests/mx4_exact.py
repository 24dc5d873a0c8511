"""Operands of microscaled products whose sums are exact in 32 bits, whatever their order, so that a product has one right answer: bf16 of the exact sum.  A block or a
unit that is left out, taken twice or scaled wrongly changes nearly every result; a bound on what rounded sums may be off would let it pass on long rows."""
import torch

VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]


def operand(g, rows, K, middle=127):
    """codes[rows, 128 U], scales[U, rows, 8] of random codes (zeros beyond K) and scale bytes middle - 1 .. middle + 1, on g's device."""
    U = -(-K // 256)
    code = torch.randint(0, 16, (rows, U * 256), generator=g, device=g.device, dtype=torch.uint8)
    code[:, K:] = 0
    return code[:, 0::2] | (code[:, 1::2] << 4), torch.randint(middle - 1, middle + 2, (U, rows, 8), generator=g, device=g.device, dtype=torch.uint8)


def values(codes, scales):
    """Their values in 64 bits."""
    rows, U = codes.shape[0], scales.shape[0]
    table = torch.tensor(VALUES, dtype=torch.float64, device=codes.device)
    v = table[torch.stack([codes & 15, codes >> 4], dim=-1).view(rows, U * 256).long()].view(rows, U * 8, 32)
    return (v * torch.exp2(scales.transpose(0, 1).reshape(rows, U * 8).double() - 127)[..., None]).view(rows, U * 256)


def sums_are_exact(x, w, middle_x=127, middle_w=127):
    """Every product is a whole multiple of the product of the smallest codes and scales, 2^-4 where both middles are 127; any partial sum is at most |x| |w| (norms)."""
    step = 2.0 ** (middle_x + middle_w - 2 * 127 - 4)
    return float(x.norm(dim=1).max() * w.norm(dim=1).max()) < 2 ** 24 * step


def wrong(Y, sums):
    """Where Y is not bf16 of the exact sums."""
    return Y != sums.float().to(torch.bfloat16)


def wrong_gated(Y, gate, up):
    """Where Y is off silu(gate) up by more than bf16's rounding, half a step of its 8 bits or 2^-8, and what the exponential, the sum, the quotient and the product in 32 bits add, each
    a few 2^-24: 2^-18 in all.  Below minus 88 the exponential passes the range of 32 bits and silu is 0, off by less than 2^-118 |up|."""
    ref = gate * torch.sigmoid(gate) * up
    return ~((Y.double() - ref).abs() <= (2.0 ** -8 + 2.0 ** -18) * ref.abs() + 2.0 ** -118 * up.abs())
