"""Which codes and scales an append to pages of 8 bits has to write for keys that are normed or rotated: the nearest ones to the formula's values.

Values are computed in 64 bits here as in the library, both with errors of a few 2^-53, so a code or scale may be either of two only where the value lies within such
an error of the border between them."""
import torch

import pages_reference as pages

U64 = 2.0 ** -53


def keys(x, weight, table, positions, eps, interleaved=False):
    """(value, bound) of the keys [n, heads, d].  A sum of d squares is off by at most d u of itself, the root by half of that; mean, eps, root, division, two
    products, and two more products and a sum where the key is rotated are 9 roundings; all of them twice (here and in the library), and a factor of two for higher orders."""
    x, d = x.double(), x.shape[-1]
    y = x
    if weight is not None:
        y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + float(torch.tensor(eps, dtype=torch.float32))) * weight.double()
    z, size = y.clone(), y.abs()
    if table is not None:
        half = table.shape[1] // 2
        rows = table.double()[positions.long()]
        cos, sin = rows[:, None, :half], rows[:, None, half:]
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
        z[..., a], z[..., b] = y[..., a] * cos - y[..., b] * sin, y[..., b] * cos + y[..., a] * sin
        size[..., a], size[..., b] = (y[..., a] * cos).abs() + (y[..., b] * sin).abs(), (y[..., b] * cos).abs() + (y[..., a] * sin).abs()
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
    either = (at - at.floor() - 0.5).abs() * unit <= bound
    return wrong_scales, int(((got != pages.codes_of(y)) & ~either).sum()), int(either.sum())
