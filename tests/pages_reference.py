"""Plain 64-bit implementations of the paged-cache operators for pages of 8 bits, windows and moving pages, on the CPU.

Bounds count every rounding, as cache_reference.py has them."""
import math

import torch

import cache_reference as ref

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
BLOCK = 16
LEAST = -100


def exponents(scales):
    return scales.view(torch.uint8).to(torch.int64) - 127


def two_to(e):
    """2^e in 64 bits."""
    return torch.ldexp(torch.ones((), dtype=torch.float64), e.to(torch.int32) if torch.is_tensor(e) else torch.tensor(e))


def decode(pages, scales):
    """Values, in 64 bits, of codes [n_pages, page, heads, d] with scales [n_pages, page / 16, heads]; exponent 128 (byte 255) is NaN."""
    e = exponents(scales)
    by = torch.where(e == 128, torch.full((), math.nan, dtype=torch.float64), two_to(e))
    return pages.float().double() * by.repeat_interleave(BLOCK, 1)[..., None]


def step(size):
    """The distance of neighbouring codes around a magnitude (in units of the scale)."""
    return two_to(torch.floor(torch.log2(size.clamp(min=2.0 ** -6))) - 3)


def codes_of(x):
    """The nearest codes, ties to even, as values; x in 64 bits, magnitudes up to 448."""
    unit = step(x.abs())
    return torch.round(x / unit) * unit  # torch.round goes to even


def scale_for(top):
    """The smallest e from LEAST on with 448 * 2^e >= top."""
    e = LEAST
    while 448.0 * 2.0 ** e < top:
        e += 1
    return e


def most_of(dtype):
    return 61440.0 if dtype == torch.float16 else 1.875 * 2.0 ** 127


def places(q_offsets, own_tables, own_lens, n_pages, page, n_tokens):
    """(token, page, row of it) of every new token that has a place."""
    out = []
    for r in range(own_tables.shape[0]):
        t0, t1 = (max(0, min(int(q_offsets[r + i]), n_tokens)) for i in (0, 1))
        for t in range(t0, t1):
            at = int(own_lens[r]) - (t1 - t0) + (t - t0)
            if 0 <= at < own_tables.shape[1] * page and 0 <= int(own_tables[r, at // page]) < n_pages:
                out.append((t, int(own_tables[r, at // page]), at % page))
    return out


def check_append8(before, scales_before, after, scales_after, x, bound, where, dtype):
    """That codes and scales [n_pages, page, heads, d] went from before to after by an append of x [n_tokens, heads, d], known to `bound`, to the places `where`."""
    page, heads = before.shape[1], before.shape[2]
    old_e, new_e = exponents(scales_before), exponents(scales_after)
    touched = {}
    for t, p, row in where:
        touched.setdefault((p, row // BLOCK), []).append((t, row % BLOCK))
    want_bytes = before.view(torch.uint8).clone()
    got_bytes = after.view(torch.uint8)
    same_scale = torch.ones_like(old_e, dtype=torch.bool)
    limit = most_of(dtype)
    for (p, b), rows in touched.items():
        first = min(row for _, row in rows)
        tokens = [t for t, _ in rows]
        same_scale[p, b] = False
        span = slice(b * BLOCK, (b + 1) * BLOCK)
        for h in range(heads):
            y, off = x[tokens, h], bound[tokens, h]
            finite = torch.isfinite(y)
            size = torch.where(finite, y.abs(), torch.zeros_like(y)).clamp(max=limit)
            fuzz = torch.where(finite, off, torch.zeros_like(y))
            lo, hi = (scale_for(float((size + s * fuzz).max().clamp(max=limit))) for s in (-1, 1))
            e = int(new_e[p, b, h])
            if first > 0:
                lo, hi = max(lo, int(old_e[p, b, h])), max(hi, int(old_e[p, b, h]))
            assert lo <= e <= hi, (p, b, h, e, lo, hi)
            if first > 0 and e != int(old_e[p, b, h]) and int(old_e[p, b, h]) != 128:
                # codes before the first new row, brought to the new scale: exactly
                held = before[p, span][:first, h].float().double() * 2.0 ** (int(old_e[p, b, h]) - e)
                got = after[p, span][:first, h].float().double()
                want = torch.where(torch.isnan(held), held, codes_of(held))
                assert torch.equal(torch.isnan(want), torch.isnan(got)) and torch.equal(want.nan_to_num(9e9), got.nan_to_num(9e9)), (p, b, h)
                want_bytes[p, span][:first, h] = got_bytes[p, span][:first, h]
            for t, row in rows:
                got = after[p, b * BLOCK + row, h].float().double()
                want_bytes[p, b * BLOCK + row, h] = got_bytes[p, b * BLOCK + row, h]
                if e == 128:
                    continue
                assert torch.equal(torch.isnan(got), ~torch.isfinite(x[t, h])), (t, h)
                ok = torch.isfinite(x[t, h])
                y, off = (x[t, h].clamp(-limit, limit) * 2.0 ** -e)[ok], (bound[t, h] * 2.0 ** -e)[ok]
                if not bool((bound[t, h][ok] > 0).any()):
                    assert torch.equal(got[ok], codes_of(y)), (t, h)
                # at most half a step of the largest magnitude that it may be, and what it is known to
                assert bool(((got[ok] - y).abs() <= step(y.abs() + off) / 2 + off).all()), (t, h)
    assert torch.equal(want_bytes, got_bytes), "bytes were written that belong to no new token"
    assert torch.equal(old_e[same_scale], new_e[same_scale]), "scales were written of blocks without new tokens"


def attention(q, k_pages, v_pages, group_offsets, prefix_tables, prefix_lens, q_offsets, own_tables, own_lens, scale=None, window=0, sinks=0):
    """(out, lse, bound of out, bound of lse) of attention with a window; pages hold values of q's type."""
    dtype = q.dtype
    n_pages, page, kv_heads, d = k_pages.shape
    tokens, heads, _ = q.shape
    share = heads // kv_heads
    scale = d ** -0.5 if scale is None else scale
    out, lse = torch.zeros(tokens, heads, d, dtype=torch.float64), torch.full((tokens, heads), -math.inf, dtype=torch.float64)
    out_b, lse_b = torch.zeros_like(out), torch.zeros_like(lse)

    def held(table, length):
        length = max(0, min(int(length), table.shape[0] * page))
        at = torch.arange(length)
        pages = table.long()[at // page]
        there = (pages >= 0) & (pages < n_pages)
        pages = pages.clamp(0, max(0, n_pages - 1))
        return k_pages[pages, at % page].double(), v_pages[pages, at % page].double(), there

    for g in range(prefix_tables.shape[0]):
        head = held(prefix_tables[g], prefix_lens[g])
        for r in range(int(group_offsets[g]), int(group_offsets[g + 1])):
            t0, t1 = int(q_offsets[r]), int(q_offsets[r + 1])
            own = held(own_tables[r], own_lens[r])
            k, v, there = (torch.cat([a, b]) for a, b in zip(head, own))
            prefix, length = head[0].shape[0], own[0].shape[0]
            place = torch.arange(prefix + length)
            for t in range(t0, t1):
                me = prefix + length - (t1 - t0) + (t - t0)
                sees = there & ((place < prefix) | (place <= me))
                if window:
                    sees &= (place < sinks) | (place > me - window)
                n = int(sees.sum())
                if n == 0:
                    continue
                for kv in range(kv_heads):
                    mine = slice(kv * share, (kv + 1) * share)
                    x, kh, vh = q[t, mine].double(), k[sees, kv], v[sees, kv]
                    s = x @ kh.T * scale
                    w = torch.softmax(s, 1)
                    out[t, mine], lse[t, mine] = w @ vh, torch.logsumexp(s, 1)
                    # as cache_reference.attention has them
                    off = 2 * ((d + 8) * ref.U32 * (x.abs() @ kh.abs().T).amax(1) * scale + 8 * ref.U32 * s.abs().amax(1)) + 2.0 ** -21
                    size = w @ vh.abs()
                    out_b[t, mine] = ref.u(dtype) * out[t, mine].abs() + size * (ref.u(dtype) + 2 * off + 4 * (n + 64) * ref.U32)[:, None] + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
                    lse_b[t, mine] = 2 * off + 2 * (n + 64) * ref.U32 + 8 * ref.U32 * lse[t, mine].abs()
    return out, lse, out_b, lse_b


def compact(n_pages, page_tokens, tables, lens):
    """(new tables, moved, n_live) as lists."""
    holds = [[[j * page_tokens < int(n) and 0 <= int(p) < n_pages for j, p in enumerate(row)] for row, n in zip(t, ls)] for t, ls in zip(tables, lens)]
    live = sorted({int(p) for t, h in zip(tables, holds) for row, hr in zip(t, h) for p, held in zip(row, hr) if held})
    n = len(live)
    moved = [-1] * n_pages
    for p in live:
        moved[p] = p
    holes = [p for p in range(n) if moved[p] < 0]
    for p, hole in zip([p for p in live if p >= n], holes):
        moved[p] = hole
    return [[[moved[int(p)] if held else int(p) for p, held in zip(row, hr)] for row, hr in zip(t, h)] for t, h in zip(tables, holds)], moved, n
