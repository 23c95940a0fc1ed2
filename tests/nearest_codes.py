"""Which codes and scales an append to pages of 8 bits has to write for keys that are normed or rotated: the nearest ones to the formula's values.

Values are computed in 64 bits here as in the library, both with errors of a few 2^-53, so a code or scale may be either of two only where the value lies within such
an error of the border between them."""
import torch

import pages_reference as pages

U64 = 2.0 ** -53


def keys(x, weight, table, positions, eps, interleaved=False):
    """(value, bound) of the keys [n, heads, d].  A sum of d squares is off by at most d u of itself, the root by half of that; mean, eps, root, division, two
    products, and two more products and a sum where the key is rotated are 9 roundings; all of them twice (here and in the library), and a factor of two for higher
    orders.  Without a norm, elements that are not rotated, or by an angle whose cosine is 1 and whose sine is 0, are what they were: no bound."""
    x, d = x.double(), x.shape[-1]
    y = x
    if weight is not None:
        y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + float(torch.tensor(eps, dtype=torch.float32))) * weight.double()
    z, size = y.clone(), y.abs() if weight is not None else torch.zeros_like(y)
    if table is not None:
        half = table.shape[1] // 2
        rows = table.double()[positions.long()]
        cos, sin = rows[:, None, :half], rows[:, None, half:]
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
        z[..., a], z[..., b] = y[..., a] * cos - y[..., b] * sin, y[..., b] * cos + y[..., a] * sin
        turned = (sin != 0) | (cos != 1) if weight is None else torch.ones_like(sin, dtype=torch.bool)
        size[..., a], size[..., b] = turned * ((y[..., a] * cos).abs() + (y[..., b] * sin).abs()), turned * ((y[..., b] * cos).abs() + (y[..., a] * sin).abs())
    return z, 2 * 2 * (d / 2 + 9) * U64 * size


def scales_for(top):
    """The smallest e from LEAST on with 448 * 2^e >= top."""
    share, power = torch.frexp(top)  # 448 = 0.875 * 2^9
    return (power - 9 + (share > 0.875).int()).clamp(min=pages.LEAST).where(top > 0, torch.full_like(power, pages.LEAST))


def compare(codes, scales, y, bound, dtype):
    """(wrong scales, wrong codes, codes that either of two values may have) of whole blocks: codes [blocks, 16, heads, d], scales [blocks, heads], y and bound
    [blocks * 16, heads, d], all finite."""
    blocks, _, heads, d = codes.shape
    most = pages.most_of(dtype)
    y, bound = y.view(blocks, 16, heads, d).clamp(-most, most), bound.view(blocks, 16, heads, d)
    e = pages.exponents(scales)
    lo, hi = (scales_for((y.abs() + s * bound).clamp(0, most).amax((1, 3))) for s in (-1, 1))
    wrong_scales = int(((e < lo) | (e > hi)).sum())
    by = pages.two_to(-e)[:, None, :, None]
    y, bound, got = (y * by).clamp(-448, 448), bound * by, codes.float().double()  # (a wrong scale is counted above)
    unit = pages.step(y.abs())
    at = y.abs() / unit
    either = ((at - at.floor() - 0.5).abs() * unit <= bound) & (bound > 0)
    return wrong_scales, int(((got != pages.codes_of(y)) & ~either).sum()), int(either.sum())


def written(y, dtype):
    """Codes and scales [blocks, 16, heads, d] and [blocks, heads] of values [blocks * 16, heads, d] in 64 bits, as compare takes them."""
    n, heads, d = y.shape
    y = y.view(n // 16, 16, heads, d).clamp(-pages.most_of(dtype), pages.most_of(dtype))
    e = scales_for(y.abs().amax((1, 3)))
    codes = pages.codes_of(y * pages.two_to(-e)[:, None, :, None]).float().to(pages.E4M3)
    return codes, (e + 127).to(torch.uint8).view(pages.E8M0)


def next_to_borders():
    """(keys, table): with cosines of 1 and sines of +-2^-30 the first elements of pairs become values next to the border between two codes at scale 1, which 32
    bits round onto it; the largest is 448 in the first two blocks, and just above or below it in the others, where that decides the scale.
    32 keys of each sign of the sine, [64, 1, 128]; key i is at position i // 32."""
    x = torch.zeros(64, 1, 128, dtype=torch.float64)
    border = (1 + (2 * torch.arange(8) + 1) / 16)[None, :] * 2.0 ** torch.arange(8)[:, None]  # 64 of them, between 1 and 480
    border = border.flatten().double()
    border = border[border < 440]
    x[:, 0, :border.shape[0]], x[:, 0, 64:] = border, 1.0
    x[:, 0, 63] = torch.tensor([448.0, 1.0]).repeat_interleave(16).repeat(2)   # 448 -+ 2^-30 in blocks 0 and 2
    x[:, 0, 127] = torch.tensor([1.0, 448.0]).repeat_interleave(16).repeat(2)  # 448 +- 2^-30 in blocks 1 and 3
    table = torch.cat([torch.ones(2, 64), torch.tensor([[1.0], [-1.0]]).expand(2, 64) * 2.0 ** -30], 1)
    return x, table
