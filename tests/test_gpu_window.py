"""Attention over pages of 8 bits and with a window on the GPU against plain 64-bit implementations (tests/cache_reference.py, tests/pages_reference.py)."""
import math
import re

import pytest
import torch

import cache_reference as ref
import pages_reference as pages
from test_gpu_cache import ATTEND, make_batch
from test_gpu_cache_joins import STAGES, kernels

pytestmark = pytest.mark.gpu

BF16, FP16 = torch.bfloat16, torch.float16
E4M3, E8M0 = pages.E4M3, pages.E8M0


@pytest.fixture(scope="module")
def lsm():
    import paper_2511_16138_amd as lsm
    return lsm


def to_8_bits(gen, blocks, least=-9, most=4):
    """Blocks [P, 2, page, heads, d] as codes and scales of any size (between the powers of two that the arguments are), with the magnitudes that come of it."""
    p, _, page, heads, d = blocks.shape
    x = blocks.float().reshape(p, 2, page // 16, 16, heads, d)
    size = torch.where(torch.isfinite(x), x.abs(), torch.zeros(())).amax((3, 5), keepdim=True).clamp(min=1e-3)
    e = torch.randint(least, most, (p, 2, page // 16, 1, heads, 1), generator=gen)
    codes = torch.where(torch.isfinite(x), x / size * 448, torch.full((), math.nan)).to(E4M3).view(p, 2, page, heads, d)
    return codes, (e - 8 + 127).to(torch.uint8).view(p, 2, page // 16, heads).view(E8M0)


def values(codes, scales, dtype):
    """What the pages hold, as dtype has it."""
    out = torch.stack([pages.decode(codes[:, i], scales[:, i]) for i in (0, 1)], 1).to(dtype)
    return out


def compare(lsm, q, held, parts, *, scales=None, window=0, sinks=0, scale=None, blocks=None, way=None, joined=None):
    """held: pages as they lie on the GPU, blocks: what they hold."""
    blocks = held if blocks is None else blocks
    reference = pages.attention if window else ref.attention
    more = dict(window=window, sinks=sinks) if window else {}
    want, want_lse, bound, lse_bound = reference(q, blocks[:, 0], blocks[:, 1], *parts, scale=scale, **more)
    dev, batch, qd = held.cuda(), lsm.PrefixBatch(*(p.cuda() for p in parts)), q.cuda()
    if scales is not None:
        s = scales.cuda()
        more.update(k_scales=s[:, 0], v_scales=s[:, 1])
    call = lambda **x: lsm.lsm_prefix_attention(qd, dev[:, 0], dev[:, 1], batch, scale=scale, **more, **x)  # noqa: E731
    out, lse = call(with_lse=True)
    ref.assert_within(out, want, bound, "out")
    ref.assert_within(lse, want_lse, lse_bound, "lse")
    assert torch.equal(out.view(torch.int16), call().view(torch.int16))
    if way is not None:
        names = kernels(call)
        flags = f"Lb{int(scales is not None)}ELb{int(window > 0)}E"
        assert re.search(rf"attention_kernelILi{0 if q.dtype == BF16 else 1}ELi{q.shape[2]}ELi{way}E.*WindowArgsI{flags}", names[0]), names
        assert joined is None or len(names) == (2 if joined else 1), names
    return out, lse


@pytest.mark.parametrize("case", ATTEND, ids=[c[0] for c in ATTEND])
def test_8_bits(lsm, case):
    _, groups, prefix, q_lens, own, hq, hkv, d, page, dtype = case
    gen = torch.Generator().manual_seed(len(case[0]) * 100 + d)
    q, blocks, parts = make_batch(gen, groups, prefix, q_lens, own, hq, hkv, d, page, dtype)
    codes, scales = to_8_bits(gen, blocks)
    compare(lsm, q, codes, parts, scales=scales, blocks=values(codes, scales, dtype))


@pytest.mark.parametrize("case", STAGES, ids=[c[0] for c in STAGES])
def test_8_bits_in_two_stages(lsm, case):
    name, groups, prefix, q_lens, own, hq, hkv, d, page, dtype, spare = case
    gen = torch.Generator().manual_seed(len(name) * 100 + d)
    q, blocks, parts = make_batch(gen, groups, prefix, q_lens, own, hq, hkv, d, page, dtype, spare=2 * spare)
    codes, scales = to_8_bits(gen, blocks)
    compare(lsm, q, codes, parts, scales=scales, blocks=values(codes, scales, dtype), way=0, joined=True)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("q_lens", [[1, 1, 1, 1], [40, 33, 5, 60]])
def test_8_bits_never_use_what_no_length_reaches(lsm, dtype, q_lens):
    """NaN codes behind every length and in pages that nobody uses, and NaN scales of blocks that nobody reaches."""
    gen = torch.Generator().manual_seed(11)
    q, blocks, parts = make_batch(gen, [3, 1], [70, 18], q_lens, [100, 33, 70, 61], 8, 2, 128, 32, dtype, garbage=math.nan, spare=3)
    codes, scales = to_8_bits(gen, blocks)
    unused = torch.isnan(codes.float()).all(-1).reshape(codes.shape[0], 2, 2, 16, 2).all(3)
    scales.view(torch.uint8)[unused] = 255
    compare(lsm, q, codes, parts, scales=scales, blocks=values(codes, scales, dtype))


@pytest.mark.parametrize("q_lens, hq, hkv, d, dtype", [([40, 33, 5, 70], 8, 2, 128, BF16), ([130, 1, 2, 64], 4, 4, 64, FP16), ([3, 2, 1, 5], 4, 2, 128, FP16),
                                                         ([40, 2, 90, 1], 4, 1, 256, BF16), ([9, 4, 2, 7], 2, 1, 64, BF16)])
@pytest.mark.parametrize("side", [0, 1])
def test_8_bits_keep_what_is_nan_from_tokens_before_it(lsm, q_lens, hq, hkv, d, dtype, side):
    gen = torch.Generator().manual_seed(18)
    page = 16
    own = [n + extra for n, extra in zip(q_lens, (37, 0, 64, 15))]
    q, blocks, parts = make_batch(gen, [3, 1], [70, 18], q_lens, own, hq, hkv, d, page, dtype)
    for r, n in enumerate(q_lens):
        for i, j in enumerate(sorted({n - 1, n // 2, 1} & set(range(1, n)))):
            at = own[r] - n + j
            blocks[int(parts[4][r, at // page]), side, at % page, (r + i) % hkv, (7 * j + r) % d] = math.nan
    codes, scales = to_8_bits(gen, blocks)
    out, _ = compare(lsm, q, codes, parts, scales=scales, blocks=values(codes, scales, dtype))
    finite = torch.isfinite(out.cpu()).all(-1).all(-1)
    assert all(bool(finite[sum(q_lens[:r])]) for r in range(4)) and not bool(finite.all())


def test_8_bits_scales_of_every_size(lsm):
    """The byte 255 makes a block NaN; scales that take values out of the type's range, below and above."""
    gen = torch.Generator().manual_seed(19)
    for dtype, least, most in ((FP16, -30, -8), (FP16, 0, 6), (BF16, -60, -40), (BF16, 20, 40)):
        q, blocks, parts = make_batch(gen, [2, 1], [64, 32], [1, 40, 2], [64, 64, 32], 4, 2, 64, 16, dtype)
        codes, scales = to_8_bits(gen, blocks, least, most)
        compare(lsm, q, codes, parts, scales=scales, blocks=values(codes, scales, dtype), scale=2.0 ** -(most + 3))
    q, blocks, parts = make_batch(gen, [1, 1], [64, 32], [1, 2], [64, 40], 4, 2, 64, 16, BF16)
    codes, scales = to_8_bits(gen, blocks)
    scales.view(torch.uint8)[int(parts[1][0, 1]), 1, 0, 1] = 255   # values of the first request's prefix, one head
    out, _ = compare(lsm, q, codes, parts, scales=scales, blocks=values(codes, scales, BF16))
    assert torch.isnan(out[0, 2:]).all() and not torch.isnan(out[0, :2]).any() and not torch.isnan(out[1:]).any()


def test_8_bits_of_strided_tensors(lsm):
    gen = torch.Generator().manual_seed(15)
    q, blocks, parts = make_batch(gen, [2, 2], [50, 20], [1, 3, 1, 2], [40, 33, 1, 90], 8, 2, 64, 32, BF16)
    codes, scales = to_8_bits(gen, blocks)
    held = values(codes, scales, BF16)
    want, _, bound, _ = ref.attention(q, held[:, 0], held[:, 1], *parts)
    k = codes[:, 0].permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3)
    v = torch.cat([codes[:, 1].view(torch.uint8), torch.zeros(codes.shape[0], 32, 2, 16, dtype=torch.uint8)], -1).cuda().view(E4M3)[..., :64]
    ks = scales[:, 0].permute(2, 1, 0).contiguous().cuda().permute(2, 1, 0)
    vs = torch.stack([scales[:, 1], scales[:, 1]], -1).cuda()[..., 1]
    got = lsm.lsm_prefix_attention(q.cuda(), k, v, lsm.PrefixBatch(*(p.cuda() for p in parts)), k_scales=ks, v_scales=vs)
    ref.assert_within(got, want, bound, "out")


# ---------------------------------------------------------------------------------------------------------------------
# windows
# ---------------------------------------------------------------------------------------------------------------------
WINDOWS = [(1, 0), (1, 1), (2, 4), (16, 0), (64, 4), (65, 63), (100, 64), (100, 65), (37, 200), (1000, 4), (1 << 29, 1 << 29)]

WINDOW_CASES = [
    # groups, prefix, q_lens, own_lens, hq, hkv, d, page, dtype
    ("one token", [1], [0], [1], [1], 1, 1, 64, 16, BF16),
    ("decode behind a prefix", [5], [100], [1] * 5, [1, 17, 64, 65, 3], 32, 2, 128, 16, BF16),
    ("decode, no prefix", [1, 1, 1], [0, 0, 0], [1, 1, 1], [1, 130, 700], 8, 2, 128, 256, FP16),
    ("decode, long", [2, 1], [1500, 20], [1, 1, 1], [3, 900, 2000], 8, 1, 64, 16, BF16),
    ("few new tokens", [3, 2], [31, 97], [3, 1, 7, 2, 4], [3, 50, 80, 2, 65], 8, 2, 128, 16, FP16),
    ("prompts", [2, 1], [64, 30], [100, 37, 130], [100, 60, 190], 8, 2, 128, 16, BF16),
    ("prompts, heads of 64", [2], [33], [70, 129], [75, 129], 4, 4, 64, 64, FP16),
    ("prompts, heads of 256", [2], [33], [70, 33], [75, 40], 4, 1, 256, 16, BF16),
    ("a long prompt", [1], [70], [700], [790], 4, 1, 128, 32, BF16),
    ("requests without tokens", [3, 0, 2], [20, 50, 10], [0, 2, 0, 1, 0], [9, 30, 0, 1, 100], 4, 2, 64, 16, BF16),
    ("rows that see nothing", [2, 2], [0, 5], [3, 1, 2, 1], [1, 0, 0, 0], 4, 2, 128, 16, FP16),
    ("prompts that see nothing at first", [1, 1], [0, 0], [150, 40], [20, 0], 8, 1, 128, 16, BF16),
    ("fewer own tokens than new ones, a prefix", [1, 1], [40, 90], [150, 3], [20, 0], 8, 1, 128, 16, BF16),
    ("heads of 256, decode", [4], [90], [1] * 4, [40, 1, 33, 300], 8, 1, 256, 16, FP16),
]


@pytest.mark.parametrize("in_8_bits", [False, True])
@pytest.mark.parametrize("case", WINDOW_CASES, ids=[c[0] for c in WINDOW_CASES])
def test_window(lsm, case, in_8_bits):
    _, groups, prefix, q_lens, own, hq, hkv, d, page, dtype = case
    gen = torch.Generator().manual_seed(len(case[0]) * 100 + d)
    q, blocks, parts = make_batch(gen, groups, prefix, q_lens, own, hq, hkv, d, page, dtype)
    more, held = {}, blocks
    if in_8_bits:
        held, scales = to_8_bits(gen, blocks)
        blocks, more = values(held, scales, dtype), dict(scales=scales)
    for window, sinks in WINDOWS:
        compare(lsm, q, held, parts, blocks=blocks, window=window, sinks=sinks, **more)


def test_a_window_that_hides_nothing_is_none(lsm):
    """The same rows as without a window."""
    gen = torch.Generator().manual_seed(20)
    q, blocks, parts = make_batch(gen, [2, 1], [64, 30], [100, 1, 130], [100, 60, 190], 8, 2, 128, 16, BF16)
    dev, batch = blocks.cuda(), lsm.PrefixBatch(*(p.cuda() for p in parts))
    plain, plain_lse = lsm.lsm_prefix_attention(q.cuda(), dev[:, 0], dev[:, 1], batch, with_lse=True)
    for window, sinks in ((300, 0), (1 << 29, 5), (100, 300)):
        out, lse = lsm.lsm_prefix_attention(q.cuda(), dev[:, 0], dev[:, 1], batch, with_lse=True, window=window, sinks=sinks)
        # each within its own bound of the same numbers
        want, want_lse, bound, lse_bound = ref.attention(q, blocks[:, 0], blocks[:, 1], *parts)
        ref.assert_within(out, want, bound, "out")
        assert bool(((out.cpu().double() - plain.cpu().double()).abs() <= 2 * bound).all()) and bool(((lse.cpu().double() - plain_lse.cpu().double()).abs() <= 2 * lse_bound).all())


@pytest.mark.parametrize("in_8_bits", [False, True])
@pytest.mark.parametrize("hkv, q_lens, own, way", [(1, [1], [9000], 1), (2, [1, 1], [5000, 300], 1), (1, [80], [4000], 2), (1, [3], [9000], 1)])
def test_a_window_dealt_to_several_workgroups(lsm, hkv, q_lens, own, way, in_8_bits):
    gen = torch.Generator().manual_seed(21)
    q, blocks, parts = make_batch(gen, [len(own)], [40], q_lens, own, 8, hkv, 64, 64, BF16)
    more, held = {}, blocks
    if in_8_bits:
        held, scales = to_8_bits(gen, blocks)
        blocks, more = values(held, scales, BF16), dict(scales=scales)
    for window, sinks, joined in ((3000, 500, True), (2100, 1, True), (1 << 20, 3, True), (150, 4, way == 2 and None)):
        # a window as long as the tables hides nothing: the kernels without one
        compare(lsm, q, held, parts, blocks=blocks, window=window, sinks=sinks, way=way if window < 1 << 20 else None, joined=joined, **more)


@pytest.mark.parametrize("in_8_bits", [False, True])
@pytest.mark.parametrize("q_lens", [[1, 1, 1, 1], [40, 33, 5, 90]])
def test_a_window_with_holes_and_garbage(lsm, q_lens, in_8_bits):
    """Pages that there are not, and NaN behind the lengths and in what no length reaches."""
    gen = torch.Generator().manual_seed(22)
    q, blocks, parts = make_batch(gen, [3, 1], [170, 100], q_lens, [100, 233, 70, 161], 8, 2, 128, 16, BF16, holes=3, garbage=math.nan, spare=2)
    more, held = {}, blocks
    if in_8_bits:
        held, scales = to_8_bits(gen, blocks)
        blocks, more = values(held, scales, BF16), dict(scales=scales)
    for window, sinks in ((1, 0), (20, 4), (64, 70), (200, 20)):
        compare(lsm, q, held, parts, blocks=blocks, window=window, sinks=sinks, **more)


@pytest.mark.parametrize("in_8_bits", [False, True])
@pytest.mark.parametrize("q_lens, own", [([1, 1], [200, 130]), ([50, 20], [200, 130]), ([150, 3], [200, 130]), ([5, 128], [90, 130])])
def test_what_is_not_finite_outside_a_window(lsm, q_lens, own, in_8_bits):
    """NaN and infinities in keys and values everywhere: they reach the tokens whose window or first tokens hold them, and no others."""
    gen = torch.Generator().manual_seed(23)
    q, blocks, parts = make_batch(gen, [2], [100], q_lens, own, 8, 2, 64, 16, BF16)
    for i, (segment, r, at) in enumerate([(1, 0, 2), (1, 0, 50), (1, 0, 99), (4, 0, 0), (4, 0, own[0] - q_lens[0] // 2 - 1), (4, 1, 33), (4, 1, own[1] - 1)]):
        page = int(parts[segment][r, at // 16])
        blocks[page, i % 2, at % 16, i % 2, 5 * i] = math.nan if i % 2 == 0 or in_8_bits else (math.inf, -math.inf)[i // 2 % 2]
    more, held = {}, blocks
    if in_8_bits:
        held, scales = to_8_bits(gen, blocks)
        blocks, more = values(held, scales, BF16), dict(scales=scales)
    some = []
    for window, sinks in ((1, 0), (10, 0), (20, 2), (20, 3), (64, 0), (130, 60)):
        out, _ = compare(lsm, q, held, parts, blocks=blocks, window=window, sinks=sinks, **more)
        some += torch.isfinite(out.cpu()).all(-1).all(-1).tolist()
    assert not all(some) and (any(some) or max(q_lens) == 1)  # both requests' last tokens hold some


@pytest.mark.parametrize("in_8_bits", [False, True])
def test_what_is_not_finite_between_first_tokens_and_window(lsm, in_8_bits):
    """Decode: NaN at every place but those that are seen."""
    gen = torch.Generator().manual_seed(24)
    q, blocks, parts = make_batch(gen, [2, 1], [100, 40], [1, 1, 1], [200, 3, 130], 8, 2, 64, 16, BF16)
    window, sinks, totals = 70, 5, [300, 103, 170]
    seen = torch.zeros(blocks.shape[0], 16, dtype=torch.bool)
    for r, total in enumerate(totals):
        prefix, table = (100, parts[1][0]) if r < 2 else (40, parts[1][1])
        for i in list(range(sinks)) + list(range(total - window, total)):
            page, row = (table[i // 16], i % 16) if i < prefix else (parts[4][r, (i - prefix) // 16], (i - prefix) % 16)
            seen[int(page), row] = True
    blocks.permute(0, 2, 1, 3, 4)[~seen] = math.nan
    more, held = {}, blocks
    if in_8_bits:
        held, scales = to_8_bits(gen, blocks)
        blocks, more = values(held, scales, BF16), dict(scales=scales)
    # the first two requests share a prefix, and one's window reaches where the other's does not: its tokens are all seen
    out, lse = compare(lsm, q, held, parts, blocks=blocks, window=window, sinks=sinks, **more)
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())


# ---------------------------------------------------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("window, sinks", [(0, 0), (40, 4)])
def test_a_cache_in_8_bits_from_append_to_compaction(lsm, window, sinks):
    """Two prompts, then decode steps; a request forks in its half-filled block; another one ends and the pages are moved together.  Every step's attention is that of
    the values that the appended blocks hold, and the moves change no bit of it."""
    gen = torch.Generator().manual_seed(30)
    hq, hkv, d, page, n_pages = 8, 2, 128, 16, 24
    codes = torch.zeros((n_pages, 2, page, hkv, d), dtype=torch.uint8, device="cuda").view(E4M3)
    scales = torch.zeros((n_pages, 2, 1, hkv), dtype=torch.uint8, device="cuda").view(E8M0)
    table, weight = lsm.lsm_rope_table(200, d), (1 + 0.1 * torch.randn(d, generator=gen)).to(BF16).cuda()
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731

    def batch(tables, lens, q_lens):
        n = len(lens)
        wide = max(len(t) for t in tables)
        return lsm.PrefixBatch(ints([0, n]), ints([]).reshape(1, 0), ints([0]), ints([sum(q_lens[:i]) for i in range(n + 1)]), ints([t + [-1] * (wide - len(t)) for t in tables]), ints(lens))

    def step(tables, lens, q_lens):
        b = batch(tables, lens, q_lens)
        x = torch.randn((sum(q_lens), hq + 2 * hkv, d), generator=gen).to(BF16)
        positions = ints([n - m + i for n, m in zip(lens, q_lens) for i in range(m)])
        dev = x.cuda()
        q = lsm.lsm_kv_append8(dev[:, hq:hq + hkv], dev[:, hq + hkv:], positions, b, codes[:, 0], codes[:, 1], scales[:, 0], scales[:, 1], table, k_weight=weight, q=dev[:, :hq], q_weight=weight)
        y, bound = ref.rotate(x[:, hq:hq + hkv].float(), weight.cpu(), table.cpu(), positions.cpu())
        held = values(codes.cpu(), scales.cpu(), BF16)
        e = pages.two_to(pages.exponents(scales.cpu()))
        t = 0
        for tab, n, m in zip(tables, lens, q_lens):
            for i in range(n - m, n):
                p = tab[i // page]
                for side, want, fuzz in ((0, y[t], bound[t]), (1, x[t, hq + hkv:].double(), 0.0)):
                    got = held[p, side, i % page].double()
                    assert bool(((got - want).abs() <= (want.abs() + fuzz) * 2.0 ** -4 + e[p, side, 0][:, None] * 2.0 ** -10 + fuzz).all())
                t += 1
        return q, b, attend(q, b)

    def attend(q, b):
        out = lsm.lsm_prefix_attention(q, codes[:, 0], codes[:, 1], b, k_scales=scales[:, 0], v_scales=scales[:, 1], window=window, sinks=sinks)
        held = values(codes.cpu(), scales.cpu(), BF16)
        parts = [t.cpu() for t in (b.group_offsets, b.prefix_tables, b.prefix_lens, b.q_offsets, b.own_tables, b.own_lens)]
        want, _, bound, _ = pages.attention(q.cpu(), held[:, 0], held[:, 1], *parts, window=window, sinks=sinks)
        ref.assert_within(out, want, bound, "out")
        return out

    tables, lens = [[20, 3, 9, 11], [5, 17, 2, 0]], [37, 18]
    step(tables, lens, [37, 18])
    for _ in range(3):
        lens = [n + 1 for n in lens]
        step(tables, lens, [1, 1])
    # the first request goes on in two ways: what is full is shared, the block under way is copied for the second
    tables, lens = tables + [[20, 3, 22, 23]], lens + [lens[0]]
    lsm.lsm_copy_pages([codes, scales], ints([9]), ints([22]))
    assert torch.equal(codes[22].view(torch.uint8), codes[9].view(torch.uint8)) and torch.equal(scales[22].view(torch.uint8), scales[9].view(torch.uint8))
    for _ in range(2):
        lens = [n + 1 for n in lens]
        q, b, before = step(tables, lens, [1, 1, 1])
    # the second request ends; the others' pages are moved together
    tables, lens, q = [tables[0], tables[2]], [lens[0], lens[2]], q[::2].contiguous()
    b = batch(tables, lens, [1, 1])
    (new,), moved, n_live = lsm.lsm_compact_pages([codes, scales], [b.own_tables], [b.own_lens], page)
    assert n_live.tolist() == [4] and sorted(p for p in moved.tolist() if p >= 0) == [0, 1, 2, 3] and int(new[:, :3].max()) < 4
    b.own_tables = new
    assert torch.equal(attend(q, b), before[::2])
    # and goes on
    lens = [n + 1 for n in lens]
    step([r[:3] + [i + 4] for i, r in enumerate(new.tolist())], lens, [1, 1])


def test_on_another_stream_and_in_a_graph(lsm):
    """Attention of both kinds recorded and replayed with new contents and lengths, eager work in between."""
    gen = torch.Generator().manual_seed(31)
    q, blocks, parts = make_batch(gen, [2, 1], [40, 17], [1, 1, 1], [300, 33, 170], 8, 2, 128, 16, BF16)
    codes, scales = to_8_bits(gen, blocks)
    dev, c, s, qd, batch = blocks.cuda(), codes.cuda(), scales.cuda(), q.cuda(), lsm.PrefixBatch(*(p.cuda() for p in parts))
    calls = [lambda **x: lsm.lsm_prefix_attention(qd, dev[:, 0], dev[:, 1], batch, window=50, sinks=4, **x),
             lambda **x: lsm.lsm_prefix_attention(qd, c[:, 0], c[:, 1], batch, k_scales=s[:, 0], v_scales=s[:, 1], **x),
             lambda **x: lsm.lsm_prefix_attention(qd, c[:, 0], c[:, 1], batch, k_scales=s[:, 0], v_scales=s[:, 1], window=70, sinks=20, **x)]
    for call in calls:
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = [call() for call in calls]
    side = torch.cuda.Stream()
    for i in range(4):
        qd.copy_(torch.randn(q.shape, generator=gen).to(BF16))
        batch.own_lens.copy_(torch.tensor([300 - 17 * i, 1 + i, 170 - i], dtype=torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        eager = [call() for call in calls]
        side.wait_stream(torch.cuda.current_stream())
        aside = [call(stream=side) for call in calls]
        torch.cuda.synchronize()
        for a, b, x in zip(outs, eager, aside):
            assert torch.equal(a, b) and torch.equal(a, x)
