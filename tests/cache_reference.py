"""Plain 64-bit implementations of the paged-cache operators on the CPU, with how far a result may be off.

Bounds count every rounding: a value rounded to type t is off by at most u(t) = eps(t) / 2 of itself, a sum of n terms in 32 bits by
at most n * 2^-24 of the sum of their magnitudes (to first order; factors of two stand for the higher ones)."""
import math

import torch

U32 = 2.0 ** -24


def u(dtype):
    return torch.finfo(dtype).eps / 2


def rotate(x, weight, table, positions, eps=1e-6, interleaved=False):
    """(value, bound) of norm and rotation of [n, heads, d]; table float32 [positions, rot] or None, weight [d] or None."""
    dtype, x = x.dtype, x.double()
    d = x.shape[-1]
    y = x
    if weight is not None:
        y = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    z, size = y.clone(), y.abs()
    if table is not None:
        rot = table.shape[1]
        half = rot // 2
        ok = (positions >= 0) & (positions < table.shape[0])
        rows = table.double()[positions.clamp(0, table.shape[0] - 1).long()]
        rows = torch.where(ok[:, None], rows, torch.full_like(rows, math.nan))
        cos, sin = rows[:, None, :half], rows[:, None, half:]
        a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, half), slice(half, rot))
        z[..., a], z[..., b] = y[..., a] * cos - y[..., b] * sin, y[..., b] * cos + y[..., a] * sin
        both = y[..., a].abs() + y[..., b].abs()
        size = size.clone()
        size[..., a], size[..., b] = both, both
    # norm: a sum of d squares (relative d u, halved by the root), root, division, two products; rotation: two products and a sum
    bound = u(dtype) * z.abs() + (d / 2 + 16) * U32 * size + (torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps)
    return z, bound


def attention(q, k_pages, v_pages, group_offsets, prefix_tables, prefix_lens, q_offsets, own_tables, own_lens, scale=None):
    """(out, lse, bound of out, bound of lse); everything on the CPU."""
    dtype = q.dtype
    n_pages, page, kv_heads, d = k_pages.shape
    tokens, heads, _ = q.shape
    share = heads // kv_heads
    scale = d ** -0.5 if scale is None else scale
    out, lse = torch.zeros(tokens, heads, d, dtype=torch.float64), torch.full((tokens, heads), -math.inf, dtype=torch.float64)
    out_b, lse_b = torch.zeros_like(out), torch.zeros_like(lse)

    def held(table, length):
        """(keys, values, which of the positions there are) of the first `length` tokens of a table."""
        length = max(0, min(int(length), table.shape[0] * page))
        ks, vs = torch.zeros(length, kv_heads, d, dtype=torch.float64), torch.zeros(length, kv_heads, d, dtype=torch.float64)
        there = torch.zeros(length, dtype=torch.bool)
        for first in range(0, length, page):
            n, p = min(page, length - first), int(table[first // page])
            if 0 <= p < n_pages:
                ks[first:first + n], vs[first:first + n] = k_pages[p, :n].double(), v_pages[p, :n].double()
                there[first:first + n] = True
        return ks, vs, there

    for g in range(prefix_tables.shape[0]):
        head_k, head_v, head_there = held(prefix_tables[g], prefix_lens[g])
        for r in range(int(group_offsets[g]), int(group_offsets[g + 1])):
            t0, t1 = int(q_offsets[r]), int(q_offsets[r + 1])
            own_k, own_v, own_there = held(own_tables[r], own_lens[r])
            for t in range(t0, t1):
                seen = max(0, own_k.shape[0] - (t1 - t0) + (t - t0) + 1)
                k = torch.cat([head_k[head_there], own_k[:seen][own_there[:seen]]])
                v = torch.cat([head_v[head_there], own_v[:seen][own_there[:seen]]])
                n = k.shape[0]
                if n == 0:
                    continue
                for h in range(heads):
                    x, kh, vh = q[t, h].double(), k[:, h // share], v[:, h // share]
                    s = (kh @ x) * scale
                    w = torch.softmax(s, 0)
                    out[t, h], lse[t, h] = w @ vh, torch.logsumexp(s, 0)
                    # a score: a product over d in 32 bits, then scaled, the maximum taken off, exponent of two (itself good to 2^-22)
                    off = 2 * ((d + 8) * U32 * float((kh.abs() @ x.abs()).max()) * scale + 8 * U32 * float(s.abs().max())) + 2.0 ** -21
                    # weights rounded to the type of the values; sums over n keys, twice (weights, and products with the values), and the joins
                    size = w @ vh.abs()
                    out_b[t, h] = u(dtype) * out[t, h].abs() + size * (u(dtype) + 2 * off + 4 * (n + 64) * U32) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
                    lse_b[t, h] = 2 * off + 2 * (n + 64) * U32 + 8 * U32 * abs(float(lse[t, h]))
    return out, lse, out_b, lse_b


def assert_within(got, want, bound, what):
    got = got.detach().cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan), f"{what}: NaN in other places"
    same = nan | (got == want)
    off = torch.where(same, torch.zeros_like(want), (got - want).abs() - bound)
    assert not torch.isnan(off).any() and float(off.max() if off.numel() else 0.0) <= 0.0, f"{what}: {float(off.max())} over its bound at {int(off.argmax())}"
