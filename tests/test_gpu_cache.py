"""The paged-cache operators on the GPU against plain 64-bit implementations (tests/cache_reference.py)."""
import math

import pytest
import torch

import cache_reference as ref

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def lsm():
    import paper_2511_16138_amd as lsm
    return lsm


def normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(dtype)


# ---------------------------------------------------------------------------------------------------------------------
# rotation
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("theta, rot, n", [(10000.0, 128, 1000), (10000.0, 2, 3), (500000.0, 64, 1 << 18), (1.5, 6, 1), (10000.0, 256, 0)])
def test_rope_table(lsm, theta, rot, n):
    got = lsm.lsm_rope_table(n, rot, theta).cpu().double()
    i = torch.arange(rot // 2, dtype=torch.float64)
    angle = torch.arange(n, dtype=torch.float64)[:, None] * theta ** (-2 * i / rot)
    want = torch.cat([angle.cos(), angle.sin()], 1)
    # one rounding of a value of at most 1, and an angle off by 2^-50 of itself
    assert got.shape == want.shape and (n == 0 or float((got - want).abs().max()) <= ref.U32 + max(1, n) * 2.0 ** -50)


ROTATE = [
    # tokens, hq, hkv, d, rot, interleaved, dtype
    (1, 32, 2, 128, 128, False, BF16),
    (7, 32, 8, 128, 64, True, FP16),
    (3, 5, 1, 64, 64, False, FP32),
    (130, 12, 12, 80, 40, False, BF16),    # half of the rotated part is no whole number of lanes
    (33, 3, 2, 80, 20, True, FP16),
    (9, 8, 1, 256, 256, False, BF16),
    (17, 2, 2, 8, 2, False, FP32),
    (5000, 4, 2, 64, 32, False, BF16),     # a wave per token
    (2, 1, 1, 248, 96, False, FP16),
    (4, 70, 3, 96, 96, True, BF16),
]


@pytest.mark.parametrize("tokens, hq, hkv, d, rot, interleaved, dtype", ROTATE)
@pytest.mark.parametrize("norm", [False, True])
def test_rotate_heads(lsm, tokens, hq, hkv, d, rot, interleaved, dtype, norm):
    gen = torch.Generator().manual_seed(tokens * 1000 + d)
    fused = normal(gen, (tokens, hq + 2 * hkv, d), dtype, 3.0)
    q, k = fused[:, :hq], fused[:, hq:hq + hkv]
    positions = torch.randint(0, 777, (tokens,), generator=gen, dtype=torch.int32)
    weights = [normal(gen, (d,), FP32 if hq % 2 else dtype) if norm else None for _ in range(2)]
    table = lsm.lsm_rope_table(777, rot, 10000.0)
    dev = fused.cuda()
    wq, wk = (None if w is None else w.cuda() for w in weights)
    got = lsm.lsm_rotate_heads(dev[:, :hq], dev[:, hq:hq + hkv], positions.cuda(), table, q_weight=wq, k_weight=wk, eps=1e-5, interleaved=interleaved)
    for x, w, y, what in ((q, weights[0], got[0], "q"), (k, weights[1], got[1], "k")):
        want, bound = ref.rotate(x, w, table.cpu(), positions, 1e-5, interleaved)
        ref.assert_within(y, want, bound, what)
    assert torch.equal(dev.cpu(), fused)  # inputs are as they were


@pytest.mark.parametrize("offset, head_pad, dtype", [(1, 0, BF16), (0, 3, BF16), (8, 8, FP16), (3, 1, FP32)])
def test_rotate_heads_of_any_alignment_and_in_place(lsm, offset, head_pad, dtype):
    gen = torch.Generator().manual_seed(5)
    n, h, d = 37, 6, 64
    positions = torch.arange(n, dtype=torch.int32)
    table = lsm.lsm_rope_table(n, 48)
    flat = normal(gen, (offset + n * h * (d + head_pad),), dtype)
    for rot_table in (table, table[:, :20].contiguous()):  # halves of 24 and of 10
        dev = flat.cuda()
        view = dev[offset:].view(n, h, d + head_pad)[:, :, :d]
        want, bound = ref.rotate(flat[offset:].view(n, h, d + head_pad)[:, :, :d], None, rot_table.cpu(), positions)
        out, _ = lsm.lsm_rotate_heads(view, None, positions.cuda(), rot_table)
        ref.assert_within(out, want, bound, "out of place")
        lsm.lsm_rotate_heads(view, None, positions.cuda(), rot_table, q_out=view)
        ref.assert_within(view, want, bound, "in place")
        rest = dev.cpu()[offset:].view(n, h, d + head_pad)[:, :, d:]
        assert torch.equal(rest, flat[offset:].view(n, h, d + head_pad)[:, :, d:])


def test_rotate_heads_without_rotation_or_tokens_and_with_far_positions(lsm):
    gen = torch.Generator().manual_seed(6)
    q = normal(gen, (5, 4, 64), BF16)
    same, none = lsm.lsm_rotate_heads(q.cuda(), None, None, None)
    assert none is None and torch.equal(same.cpu(), q)
    w = normal(gen, (64,), BF16)
    normed, _ = lsm.lsm_rotate_heads(q.cuda(), None, None, None, q_weight=w.cuda())
    ref.assert_within(normed, *ref.rotate(q, w, None, None), "norm alone")
    empty, _ = lsm.lsm_rotate_heads(q[:0].cuda(), None, torch.zeros(0, dtype=torch.int32).cuda(), lsm.lsm_rope_table(4, 64))
    assert empty.shape == (0, 4, 64)
    # positions without an angle: NaN where it would be rotated, the rest as it is
    positions = torch.tensor([0, -1, 9, 10, 2 ** 31 - 1], dtype=torch.int32)
    table = lsm.lsm_rope_table(10, 32)
    got, _ = lsm.lsm_rotate_heads(q.cuda(), None, positions.cuda(), table)
    ref.assert_within(got, *ref.rotate(q, None, table.cpu(), positions), "positions out of range")
    # zeros stay zeros, infinities and NaN stay in their head
    x = torch.zeros(2, 3, 64, dtype=FP16)
    x[0, 1, 5], x[1, 2, 40] = math.inf, math.nan
    got, _ = lsm.lsm_rotate_heads(x.cuda(), None, torch.tensor([0, 3], dtype=torch.int32).cuda(), table, q_weight=torch.ones(64, dtype=FP16).cuda())
    finite = torch.isfinite(got.cpu()).all(-1)
    assert finite.tolist() == [[True, False, True], [True, True, False]] and float(got[0, 0].abs().max()) == 0.0


# ---------------------------------------------------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("tokens, hq, hkv, d, rot, page, dtype, norm, interleaved", [
    (1, 32, 2, 128, 128, 16, BF16, True, False),
    (64, 0, 8, 128, 64, 16, FP16, False, True),
    (333, 12, 12, 64, 64, 32, BF16, True, False),
    (50, 8, 1, 256, 128, 64, BF16, False, False),
    (21, 3, 3, 40, 20, 24, FP32, True, False),   # a page of no power of two
    (5000, 4, 2, 64, 64, 16, FP16, True, False),
])
def test_kv_append(lsm, tokens, hq, hkv, d, rot, page, dtype, norm, interleaved):
    gen = torch.Generator().manual_seed(tokens + d)
    fused = normal(gen, (tokens, hq + 2 * hkv, d), dtype)
    pages = -(-tokens // page) + 3
    blocks = normal(gen, (pages, 2, page, hkv, d), dtype)
    positions = torch.randint(0, 500, (tokens,), generator=gen, dtype=torch.int32)
    slots = torch.randperm(pages * page, generator=gen)[:tokens]
    if tokens > 20:
        slots[3], slots[7], slots[11] = -1, pages * page, 2 ** 62  # nothing is written for these
        slots[13] = -2 ** 63
    table = lsm.lsm_rope_table(500, rot)
    wq, wk = (normal(gen, (d,), dtype) if norm else None for _ in range(2))
    dev, held = fused.cuda(), blocks.cuda()
    q, k, v = dev[:, :hq], dev[:, hq:hq + hkv], dev[:, hq + hkv:]
    queries = dict(q=q, q_weight=None if wq is None else wq.cuda()) if hq else {}
    got_q = lsm.lsm_kv_append(k, v, positions.cuda(), slots.cuda(), held[:, 0], held[:, 1], table, k_weight=None if wk is None else wk.cuda(),
                              interleaved=interleaved, **queries)
    want, bound = ref.rotate(fused[:, hq:hq + hkv], wk, table.cpu(), positions, interleaved=interleaved)
    k_want, k_bound = blocks[:, 0].double().reshape(pages * page, hkv, d).clone(), torch.zeros(pages * page, hkv, d, dtype=torch.float64)
    v_want = blocks[:, 1].reshape(pages * page, hkv, d).clone()
    ok = (slots >= 0) & (slots < pages * page)
    k_want[slots[ok]], k_bound[slots[ok]], v_want[slots[ok]] = want[ok], bound[ok], fused[:, hq + hkv:][ok]
    ref.assert_within(held[:, 0].reshape(pages * page, hkv, d), k_want, k_bound, "keys")
    assert torch.equal(held[:, 1].reshape(pages * page, hkv, d).cpu(), v_want)
    if hq:
        ref.assert_within(got_q, *ref.rotate(fused[:, :hq], wq, table.cpu(), positions, interleaved=interleaved), "queries")
    else:
        assert got_q is None


def test_kv_append_beyond_four_gigabytes(lsm):
    """Pages whose offsets pass 32 bits, in bytes and in elements."""
    page, hkv, d = 16, 8, 128
    pages = (1 << 32) // (page * hkv * d) + 64          # elements past 2^32, bytes past 2^33
    k_pages = torch.empty((pages, page, hkv, d), dtype=BF16, device="cuda")
    gen = torch.Generator().manual_seed(8)
    k = normal(gen, (3, hkv, d), BF16)
    slots = torch.tensor([pages * page - 1, 5, (1 << 32) // (hkv * d) + 17])
    k_pages[(slots // page).cuda()] = 0
    lsm.lsm_kv_append(k.cuda(), k.cuda(), None, slots.cuda(), k_pages, k_pages, None)  # the values are the keys
    flat = k_pages.view(-1, hkv, d)
    assert torch.equal(flat[slots.cuda()].cpu(), k)
    # and attention over them
    tables = (slots // page).to(torch.int32)
    q = normal(gen, (3, 16, d), BF16)
    batch = lsm.PrefixBatch(*(t.cuda() for t in (torch.tensor([0, 3], dtype=torch.int32), torch.zeros(1, 0, dtype=torch.int32), torch.zeros(1, dtype=torch.int32),
                                                 torch.arange(4, dtype=torch.int32), tables[:, None].contiguous(), (slots % page + 1).to(torch.int32))))
    few = k_pages[tables.long().cuda()].cpu()
    out = lsm.lsm_prefix_attention(q.cuda(), k_pages, k_pages, batch)
    want, _, bound, _ = ref.attention(q, few, few, torch.tensor([0, 3]), torch.zeros(1, 0), torch.zeros(1), torch.arange(4), torch.arange(3)[:, None], slots % page + 1)
    ref.assert_within(out, want, bound, "out")


# ---------------------------------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------------------------------
def make_batch(gen, groups, prefix, q_lens, own_lens, hq, hkv, d, page, dtype, holes=0, garbage=None, scale=1.0, spare=0):
    """groups: requests of each; garbage: what lies behind lengths and in pages that nobody uses."""
    counts = [-(-x // page) for x in list(prefix) + list(own_lens)]
    total = sum(counts) + 4
    shape = (total, 2, page, hkv, d)
    blocks = normal(gen, shape, dtype, scale)
    order = torch.randperm(total, generator=gen).tolist()
    used = torch.zeros(total, page, dtype=torch.bool)
    rows, at = [], 0
    for length, c in zip(list(prefix) + list(own_lens), counts):
        mine = order[at:at + c]
        at += c
        for i, p in enumerate(mine):
            used[p, :min(page, length - i * page)] = True
        rows.append(mine)
    if garbage is not None:
        blocks.permute(0, 2, 1, 3, 4)[~used] = garbage
    n_groups = len(prefix)

    def table(rows):
        width = max([len(r) for r in rows] + [0]) + spare
        t = torch.full((len(rows), width), 0x7FFFFFF0, dtype=torch.int32)
        for i, r in enumerate(rows):
            t[i, :len(r)] = torch.tensor(r, dtype=torch.int32)
            for _ in range(holes if len(r) > 1 else 0):
                t[i, int(torch.randint(0, len(r), (1,), generator=gen))] = [-1, total, -2 ** 31][int(torch.randint(0, 3, (1,), generator=gen))]
        return t

    ints = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    offsets = lambda v: ints([sum(v[:i]) for i in range(len(v) + 1)])  # noqa: E731
    q = normal(gen, (sum(q_lens), hq, d), dtype, scale)
    return q, blocks, [offsets(list(groups)), table(rows[:n_groups]), ints(list(prefix)), offsets(list(q_lens)), table(rows[n_groups:]), ints(list(own_lens))]


def check(lsm, q, blocks, parts, scale=None, twice=True):
    want, want_lse, bound, lse_bound = ref.attention(q, blocks[:, 0], blocks[:, 1], *parts, scale=scale)
    held, dev = blocks.cuda(), [p.cuda() for p in parts]
    out, lse = lsm.lsm_prefix_attention(q.cuda(), held[:, 0], held[:, 1], lsm.PrefixBatch(*dev), scale=scale, with_lse=True)
    ref.assert_within(out, want, bound, "out")
    ref.assert_within(lse, want_lse, lse_bound, "lse")
    if twice:
        again = lsm.lsm_prefix_attention(q.cuda(), held[:, 0], held[:, 1], lsm.PrefixBatch(*dev), scale=scale)
        assert torch.equal(out, again)
    return out


ATTEND = [
    # groups, prefix, q_lens, own_lens, hq, hkv, d, page, dtype
    ("one token", [1], [0], [1], [1], 1, 1, 64, 16, BF16),
    ("one request, one group", [1], [33], [1], [7], 4, 1, 128, 16, FP16),
    ("decode behind one prefix", [5], [100], [1] * 5, [1, 17, 64, 65, 3], 32, 2, 128, 16, BF16),
    ("decode behind three", [2, 1, 4], [64, 0, 129], [1] * 7, [16, 1, 300, 31, 33, 128, 2], 8, 2, 128, 16, BF16),
    ("heads of 64", [3, 3], [70, 1], [1] * 6, [5, 200, 64, 63, 1, 129], 20, 5, 64, 32, FP16),
    ("heads of 256", [4], [90], [1] * 4, [40, 1, 33, 70], 8, 1, 256, 16, BF16),
    ("heads of 256, no prefix", [1, 1], [0, 0], [1, 40], [300, 50], 8, 1, 256, 64, FP16),
    ("a share of seven", [6], [50], [1] * 6, [9, 10, 11, 100, 1, 64], 28, 4, 128, 64, FP16),
    ("a share of 24", [4], [40], [2, 1, 1, 3], [9, 10, 11, 100], 48, 2, 128, 16, BF16),
    ("every head its own", [5], [65], [1] * 5, [1, 2, 3, 4, 130], 6, 6, 64, 16, BF16),
    ("no prefix at all", [1, 1, 1], [0, 0, 0], [1, 1, 1], [1, 130, 700], 8, 2, 128, 256, BF16),
    ("few new tokens", [3, 2], [31, 97], [3, 1, 7, 2, 4], [3, 50, 80, 2, 65], 8, 2, 128, 16, FP16),
    ("prompts", [2, 1], [64, 30], [100, 37, 130], [100, 60, 190], 8, 2, 128, 16, BF16),
    ("prompts, heads of 64", [2], [33], [70, 129], [75, 129], 4, 4, 64, 64, FP16),
    ("prompts, heads of 256", [2], [33], [70, 33], [75, 40], 4, 1, 256, 16, BF16),
    ("requests without tokens", [3, 0, 2], [20, 50, 10], [0, 2, 0, 1, 0], [9, 30, 0, 1, 100], 4, 2, 64, 16, BF16),
    ("rows that see nothing", [2, 2], [0, 5], [3, 1, 2, 1], [1, 0, 0, 0], 4, 2, 128, 16, FP16),
    ("prompts that see nothing at first", [1, 1], [0, 0], [150, 40], [20, 0], 8, 1, 128, 16, BF16),
    ("mixed prompts and decode", [4], [80], [1, 90, 1, 1], [70, 95, 1, 33], 16, 4, 128, 16, BF16),
    ("many requests", [40, 1, 70], [48, 17, 0], [1] * 111, [1 + (i * 7) % 40 for i in range(111)], 4, 2, 64, 16, FP16),
    ("a long prefix", [2], [5000], [1, 2], [3, 900], 8, 1, 128, 16, BF16),
]


@pytest.mark.parametrize("case", ATTEND, ids=[c[0] for c in ATTEND])
def test_prefix_attention(lsm, case):
    _, groups, prefix, q_lens, own, hq, hkv, d, page, dtype = case
    gen = torch.Generator().manual_seed(len(case[0]) * 100 + d)
    check(lsm, *make_batch(gen, groups, prefix, q_lens, own, hq, hkv, d, page, dtype))


@pytest.mark.parametrize("garbage", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("q_lens", [[1, 1, 1, 1], [40, 33, 5, 60]])
def test_prefix_attention_never_uses_what_no_length_reaches(lsm, garbage, q_lens):
    gen = torch.Generator().manual_seed(11)
    check(lsm, *make_batch(gen, [3, 1], [70, 18], q_lens, [100, 33, 70, 61], 8, 2, 128, 32, BF16, garbage=garbage, spare=3))


@pytest.mark.parametrize("q_lens, hq, hkv, d, dtype", [([40, 33, 5, 70], 8, 2, 128, BF16), ([130, 1, 2, 64], 4, 4, 64, FP16), ([3, 2, 1, 5], 4, 2, 128, FP16),
                                                         ([40, 2, 90, 1], 4, 1, 256, BF16), ([9, 4, 2, 7], 2, 1, 64, BF16)])
@pytest.mark.parametrize("in_keys", [False, True])
def test_prefix_attention_keeps_what_is_not_finite_from_tokens_before_it(lsm, q_lens, hq, hkv, d, dtype, in_keys):
    """Infinities and NaN in the values (NaN in the keys) of new tokens: they reach the tokens that see them, in their columns, and no others."""
    gen = torch.Generator().manual_seed(18)
    page = 16
    own = [n + extra for n, extra in zip(q_lens, (37, 0, 64, 15))]
    q, blocks, parts = make_batch(gen, [3, 1], [70, 18], q_lens, own, hq, hkv, d, page, dtype)
    for r, n in enumerate(q_lens):
        for i, j in enumerate(sorted({n - 1, n // 2, 1} & set(range(1, n)))):  # not the first new token, which all others see
            at = own[r] - n + j
            where = blocks[int(parts[4][r, at // page]), 0 if in_keys else 1, at % page, (r + i) % hkv]
            where[(7 * j + r) % d] = math.nan if in_keys else (math.inf, math.nan, -math.inf)[i]
    out = check(lsm, q, blocks, parts, twice=False)
    finite = torch.isfinite(out.cpu()).all(-1).all(-1)
    first = [sum(q_lens[:r]) for r in range(4)]
    assert all(bool(finite[t]) for t in first) and not bool(finite.all())


@pytest.mark.parametrize("q_lens, d", [([1, 1, 1, 1], 128), ([40, 33, 5, 70], 64), ([1, 2, 1, 3], 256)])
def test_prefix_attention_with_holes(lsm, q_lens, d):
    """Page numbers out of range: their tokens are not seen."""
    gen = torch.Generator().manual_seed(12)
    check(lsm, *make_batch(gen, [3, 1], [170, 100], q_lens, [100, 233, 70, 161], 8, 2, d, 16, FP16, holes=3))


def test_prefix_attention_with_lengths_beyond_the_tables(lsm):
    gen = torch.Generator().manual_seed(13)
    q, blocks, parts = make_batch(gen, [2, 1], [64, 32], [1, 1, 2], [64, 64, 32], 4, 2, 64, 16, BF16)
    parts[2] = torch.tensor([2 ** 31 - 1, -5], dtype=torch.int32)
    parts[5] = torch.tensor([64, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)
    check(lsm, q, blocks, parts)


@pytest.mark.parametrize("scale, size", [(None, 30.0), (3.0, 1.0), (1e-6, 1.0), (0.05, 0.0)])
def test_prefix_attention_of_large_and_zero_scores(lsm, scale, size):
    gen = torch.Generator().manual_seed(14)
    q, blocks, parts = make_batch(gen, [4], [130], [1, 1, 40, 2], [40, 100, 90, 7], 8, 2, 128, 16, BF16, scale=1.0)
    check(lsm, (q.float() * size).to(BF16), blocks, parts, scale=scale)


@pytest.mark.parametrize("groups, prefix, hq", [([33, 31], [12400, 3001], 64), ([40], [8200], 64), ([30, 10], [6000, 6000], 32)])
def test_prefix_attention_of_many_requests_behind_long_prefixes(lsm, groups, prefix, hq):
    """Wide first stages, their keys dealt to different numbers of workgroups, beside narrow second ones."""
    gen = torch.Generator().manual_seed(19)
    n = sum(groups)
    check(lsm, *make_batch(gen, groups, prefix, [1] * n, [1 + (i * 5) % 37 for i in range(n)], hq, 1, 64, 256, BF16))


def test_prefix_attention_of_strided_tensors(lsm):
    gen = torch.Generator().manual_seed(15)
    q, blocks, parts = make_batch(gen, [2, 2], [50, 20], [1, 3, 1, 2], [40, 33, 1, 90], 8, 2, 64, 16, BF16)
    want, _, bound, _ = ref.attention(q, blocks[:, 0], blocks[:, 1], *parts)
    dev = [p.cuda() for p in parts]
    # heads before tokens in a page, keys and values in tensors of their own, queries and output inside wider rows, heads first
    k = blocks[:, 0].permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3)
    v = torch.nn.functional.pad(blocks[:, 1], (0, 16)).cuda()[..., :64]
    wide = torch.zeros(8, q.shape[0], 72, dtype=BF16, device="cuda")
    qd = wide.permute(1, 0, 2)[:, :, 8:]
    qd.copy_(q)
    out = torch.full((q.shape[0], 9, 64), 7.0, dtype=BF16, device="cuda")
    got = lsm.lsm_prefix_attention(qd, k, v, lsm.PrefixBatch(*dev), out=out[:, 1:])
    ref.assert_within(got, want, bound, "out")
    assert float((out[:, 0] - 7).abs().max()) == 0.0


def test_prefix_attention_of_no_tokens(lsm):
    gen = torch.Generator().manual_seed(16)
    q, blocks, parts = make_batch(gen, [1], [16], [0], [5], 4, 2, 64, 16, BF16)
    held = blocks.cuda()
    out, lse = lsm.lsm_prefix_attention(q.cuda(), held[:, 0], held[:, 1], lsm.PrefixBatch(*(p.cuda() for p in parts)), with_lse=True)
    assert out.shape == (0, 4, 64) and lse.shape == (0, 4)


def test_operators_on_another_stream_and_in_a_graph(lsm):
    """A decode step: append, then attention; on a side stream, then captured and replayed with new inputs in the same buffers."""
    gen = torch.Generator().manual_seed(17)
    hq, hkv, d, page = 8, 2, 128, 16
    q, blocks, parts = make_batch(gen, [3], [40], [1, 1, 1], [20, 33, 1], hq, hkv, d, page, BF16)
    dev, held = [p.cuda() for p in parts], blocks.cuda()
    table = lsm.lsm_rope_table(200, d)
    positions = (parts[5] + 40 - 1).to(torch.int32)
    slots = torch.tensor([int(parts[4][r, (int(n) - 1) // page]) * page + (int(n) - 1) % page for r, n in enumerate(parts[5])])
    fused = torch.zeros(3, hq + 2 * hkv, d, dtype=BF16, device="cuda")
    positions_d, slots_d = positions.cuda(), slots.cuda()

    def step():
        rotated = lsm.lsm_kv_append(fused[:, hq:hq + hkv], fused[:, hq + hkv:], positions_d, slots_d, held[:, 0], held[:, 1], table, q=fused[:, :hq])
        return rotated, lsm.lsm_prefix_attention(rotated, held[:, 0], held[:, 1], lsm.PrefixBatch(*dev))

    def verify(x, rotated, out):
        want_k, _ = ref.rotate(x[:, hq:hq + hkv], None, table.cpu(), positions)
        after = held.cpu()
        ref.assert_within(after[:, 0].reshape(-1, hkv, d)[slots], want_k, ref.rotate(x[:, hq:hq + hkv], None, table.cpu(), positions)[1], "keys")
        assert torch.equal(after[:, 1].reshape(-1, hkv, d)[slots], x[:, hq + hkv:])
        want, _, bound, _ = ref.attention(rotated.cpu(), after[:, 0], after[:, 1], *parts)
        ref.assert_within(out, want, bound, "out")

    side = torch.cuda.Stream()
    x = normal(gen, fused.shape, BF16)
    with torch.cuda.stream(side):
        fused.copy_(x)
        rotated, out = step()
    side.synchronize()
    verify(x, rotated, out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rotated, out = step()
    for _ in range(4):
        x = normal(gen, fused.shape, BF16)
        fused.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        verify(x, rotated, out)
        again_rotated, again = step()  # eager work of the same kind in between
        assert torch.equal(again, out) and torch.equal(again_rotated, rotated)
