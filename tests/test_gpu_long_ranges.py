"""Attention over pages of 8 bits, and with a window, where one workgroup goes over more keys than it looks up pages for at a time (1,024 of a wide tile, 4,096 of a
narrow one), against 64 bits.

Keys are +-1 and every row's query is one of the keys that it sees, so that its result is that key's value, whatever else there is: a tile with another's keys,
values or scales is off by the whole of a value."""
import pytest
import torch

import cache_reference as ref
import pages_reference as pages

pytestmark = pytest.mark.gpu

BF16, FP16 = torch.bfloat16, torch.float16
SHARP = 60.0  # the score of a row's own key; others' are normal with SHARP / sqrt(d)


@pytest.fixture(scope="module")
def lsm():
    import paper_2511_16138_amd as lsm
    return lsm


def ints(v):
    return torch.tensor(v, dtype=torch.int32)


def offsets(v):
    return ints([sum(v[:i]) for i in range(len(v) + 1)])


def make_pages(gen, n, page, hkv, d, dtype, in_8_bits):
    """(held, scales, values): keys of +-1, as codes of +-2^-e and scales of 2^e, and normal values, likewise."""
    keys = torch.randint(0, 2, (n, page, hkv, d), generator=gen).float() * 2 - 1
    vals = torch.randn((n, page, hkv, d), generator=gen)
    if not in_8_bits:
        held = torch.stack([keys, vals], 1).to(dtype)
        return held, None, held
    e = torch.randint(-3, 4, (n, 2, page // 16, hkv), generator=gen)
    by = pages.two_to(e).float().repeat_interleave(16, 2)[..., None]
    codes = (torch.stack([keys, vals], 1) / by).to(pages.E4M3)
    scales = (e + 127).to(torch.uint8).view(pages.E8M0)
    return codes, scales, torch.stack([pages.decode(codes[:, i], scales[:, i]) for i in (0, 1)], 1).to(dtype)


def check(lsm, gen, groups, prefix, q_lens, own, hq, hkv, d, page, dtype, *, in_8_bits, window=0, sinks=0, parts_of_work):
    """All prefixes lie in the same pages, and so do all requests' own tokens.  parts_of_work: into how many parts the plan has to cut the keys (0: one range, nothing to join)."""
    widths = -(-max(prefix) // page), -(-max(own) // page)
    total = sum(widths)
    held, scales, values = make_pages(gen, total + 2, page, hkv, d, dtype, in_8_bits)
    order = torch.randperm(total + 2, generator=gen).tolist()

    prefix_tables, own_tables = (ints([order.pop() for _ in range(w)]).expand(n, w).contiguous() for w, n in zip(widths, (len(prefix), len(own))))
    cuts = offsets(groups)
    tokens, share = sum(q_lens), hq // hkv
    q = torch.zeros((tokens, hq, d), dtype=dtype)
    # each row's query: a key that it sees
    t = 0
    for r, n in enumerate(q_lens):
        g = int((cuts[1:-1] <= r).sum())
        for j in range(n):
            me = prefix[g] + own[r] - n + j
            first = max(0, me + 1 - window) if window else 0
            for h in range(hq):
                seen = me + 1 - first + min(sinks, first)
                at = int(torch.randint(0, seen, (1,), generator=gen))
                at = at if at < min(sinks, first) else first + at - min(sinks, first)
                row, at = (prefix_tables[g], at) if at < prefix[g] else (own_tables[r], at - prefix[g])
                q[t, h] = values[int(row[at // page]), 0, at % page, h // share]
            t += 1
    parts = (cuts, prefix_tables, ints(prefix), offsets(q_lens), own_tables, ints(own))
    want, want_lse, bound, lse_bound = pages.attention(q, values[:, 0], values[:, 1], *parts, scale=SHARP / d, window=window, sinks=sinks)
    assert float(bound.max()) < 0.5 and float(want.abs().mean()) > 0.5  # what a mistake is off by, and what is let pass
    dev, batch, qd = held.cuda(), lsm.PrefixBatch(*(p.cuda() for p in parts)), q.cuda()
    more = {} if scales is None else dict(zip(("k_scales", "v_scales"), (s for s in scales.cuda().unbind(1))))
    call = lambda **x: lsm.lsm_prefix_attention(qd, dev[:, 0], dev[:, 1], batch, scale=SHARP / d, window=window, sinks=sinks, **more, **x)  # noqa: E731
    space = torch.empty(parts_of_work * tokens * hq * (d * 4 + 8), dtype=torch.uint8, device="cuda")
    call(workspace=space)
    if parts_of_work:
        with pytest.raises(lsm.LsmError):
            call(workspace=space[:-1])
    out, lse = call(with_lse=True)
    ref.assert_within(out, want, bound, "out")
    ref.assert_within(lse, want_lse, lse_bound, "lse")
    assert torch.equal(out.view(torch.int16), call().view(torch.int16))


WIDE = [(8, 8, 64, BF16, 16), (8, 8, 128, FP16, 64), (8, 4, 256, BF16, 32)]  # share, KV heads, head's elements, type, page


@pytest.mark.parametrize("share, hkv, d, dtype, page", WIDE)
@pytest.mark.parametrize("kind", ["8 bits", "8 bits, window", "16 bits, window"])
def test_wide_tiles(lsm, kind, share, hkv, d, dtype, page):
    """About 2,600 keys for each tile, half of the requests' behind a prefix; 256 tiles and more, so that nothing is cut."""
    gen = torch.Generator().manual_seed(d + len(kind))
    n = 256 // hkv
    q_lens = [7] * n
    prefix, own = [1100 + 16 * 3 + 5 if r % 2 else 0 for r in range(n)], [2600 - 29 * (r % 5) - (1150 if r % 2 else 0) for r in range(n)]
    window = dict(window=1500, sinks=70) if "window" in kind else {}
    check(lsm, gen, [1] * n, prefix, q_lens, own, share * hkv, hkv, d, page, dtype, in_8_bits=kind.startswith("8"), parts_of_work=0, **window)


@pytest.mark.parametrize("share, hkv, d, dtype, page", WIDE)
def test_narrow_tiles_of_two_stages(lsm, share, hkv, d, dtype, page):
    """Own tokens beyond 4,096 behind short shared prefixes."""
    gen = torch.Generator().manual_seed(d)
    n = 520 // hkv
    own = [4000 + 97 * (r % 7) for r in range(n)]
    check(lsm, gen, [n - 3, 3], [40, 16], [1] * n, own, 2 * hkv, hkv, d, page, dtype, in_8_bits=True, parts_of_work=2)


@pytest.mark.parametrize("share, hkv, d, dtype, page", WIDE)
def test_narrow_tiles_of_prefixes(lsm, share, hkv, d, dtype, page):
    """Prefixes beyond 4,096 tokens, two requests behind each."""
    gen = torch.Generator().manual_seed(d + 1)
    groups = 168 // hkv
    check(lsm, gen, [2] * groups, [4300 - 13 * (g % 4) for g in range(groups)], [1] * (2 * groups), [300 + 16 * (r % 2) for r in range(2 * groups)], 2 * hkv, hkv, d, page, dtype, in_8_bits=True, parts_of_work=2)


@pytest.mark.parametrize("d, dtype", [(64, BF16), (128, FP16)])
@pytest.mark.parametrize("kind", ["8 bits", "8 bits, window", "16 bits, window"])
def test_narrow_tiles_of_very_long_requests(lsm, kind, d, dtype):
    """300,000 tokens: 64 ranges are the most that there are, of more than 4,096 keys each.  Requests with the same pages and lengths."""
    gen = torch.Generator().manual_seed(d + 2)
    window = dict(window=290001, sinks=100) if "window" in kind else {}
    check(lsm, gen, [1] * 4, [0] * 4, [1] * 4, [300001] * 4, 32, 1, d, 64, dtype, in_8_bits=kind.startswith("8"), parts_of_work=64, **window)
