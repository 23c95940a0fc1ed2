"""The comparison of tests/nearest_codes.py, on plain implementations in 64 and in 32 bits: it accepts the former and not the latter."""
import torch

import nearest_codes as nearest
import pages_reference as pages


def in_32_bits(x, weight, table, positions, eps, interleaved):
    y = x.float()
    if weight is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + eps) * weight.float()
    rows = table[positions.long()][:, None]
    half = table.shape[1] // 2
    cos, sin = rows[..., :half], rows[..., half:]
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    z = y.clone()
    z[..., a], z[..., b] = y[..., a] * cos - y[..., b] * sin, y[..., b] * cos + y[..., a] * sin
    return z.double()


def test_32_bits_are_told_from_64():
    wrong = 0
    for norm, interleaved in ((True, True), (True, False), (False, True), (False, False)):
        gen = torch.Generator().manual_seed(1)
        n, heads, d = 8192, 4, 128
        x, w = torch.randn((n, heads, d), generator=gen).to(torch.bfloat16), (1 + 0.2 * torch.randn(d, generator=gen)).to(torch.bfloat16) if norm else None
        angle = torch.arange(4096).double()[:, None] * 10000.0 ** (-torch.arange(d // 2).double() / (d // 2))
        table, positions = torch.cat([angle.cos(), angle.sin()], 1).float(), torch.randint(0, 4096, (n,), generator=gen)
        y, bound = nearest.keys(x, w, table, positions, 1e-6, interleaved)
        scales, codes, either = nearest.compare(*nearest.written(y, x.dtype), y, bound, x.dtype)
        assert (scales, codes) == (0, 0) and either <= 1  # one in 10^10 may be either of two
        wrong += nearest.compare(*nearest.written(in_32_bits(x, w, table, positions, 1e-6, interleaved), x.dtype), y, bound, x.dtype)[1]
    assert wrong > 5  # of 16 million, one to three in a million


def test_values_rounded_twice_are_told_from_values_rounded_once():
    x, table = nearest.next_to_borders()
    y, bound = nearest.keys(x, None, table, torch.arange(64) // 32, 0.0)
    assert nearest.compare(*nearest.written(y, torch.float32), y, bound, torch.float32) == (0, 0, 0)
    codes, scales = nearest.written(y, torch.float32)
    assert sorted(set(pages.exponents(scales).flatten().tolist())) == [0, 1]
    # to 32 bits first: onto the border, and to the even code of the two from there
    wrong_scales, wrong_codes, _ = nearest.compare(*nearest.written(y.float().double(), torch.float32), y, bound, torch.float32)
    assert wrong_scales == 2 and wrong_codes > 500
