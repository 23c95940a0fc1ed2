"""Append to pages of 8 bits on the GPU against plain 64-bit implementations (tests/pages_reference.py)."""
import math

import pytest
import torch

import cache_reference as ref
import pages_reference as pages

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
E4M3, E8M0 = pages.E4M3, pages.E8M0


@pytest.fixture(scope="module")
def lsm():
    import paper_2511_16138_amd as lsm
    return lsm


def ints(v):
    return torch.tensor(v, dtype=torch.int32)


def offsets(v):
    return ints([sum(v[:i]) for i in range(len(v) + 1)])


def pool(gen, n_pages, page, hkv, d, spread=3):
    """Codes and scales of keys and values side by side: [n_pages, 2, ...]."""
    codes = torch.randint(0, 127, (n_pages, 2, page, hkv, d), generator=gen, dtype=torch.uint8) | (torch.randint(0, 2, (n_pages, 2, page, hkv, d), generator=gen, dtype=torch.uint8) << 7)
    e = torch.randint(127 - 8 - spread, 127 - 8 + spread, (n_pages, 2, page // 16, hkv), generator=gen, dtype=torch.uint8)
    return codes.view(E4M3), e.view(E8M0)


def tables(gen, n_pages, page, lens, spare=1):
    """Page tables of requests of these lengths: pages in any order, each of one request, something else behind the lengths."""
    order = torch.randperm(n_pages, generator=gen).tolist()
    counts = [-(-max(0, n) // page) for n in lens]
    assert sum(counts) <= n_pages
    out = torch.full((len(lens), max(counts + [0]) + spare), 0x7FFFFFF0, dtype=torch.int32)
    for i, c in enumerate(counts):
        out[i, :c] = ints([order.pop() for _ in range(c)])
    return out


def batch_of(lsm, q_lens, own_tables, own_lens):
    n = len(q_lens)
    return lsm.PrefixBatch(*(t.cuda() for t in (ints([0, n]), ints([[]]).reshape(1, 0), ints([0]), offsets(q_lens), own_tables, ints(own_lens))))


def run(lsm, gen, fused, hq, hkv, d, q_lens, own_lens, page, *, table=None, positions=None, weights=(None, None), interleaved=False, eps=1e-6, held=None, spare_pages=3, own_tables=None):
    """Appends, and checks all of what was and was not written; (codes, scales, queries)."""
    n_pages = sum(-(-max(0, n) // page) for n in own_lens) + spare_pages
    codes, scales = pool(gen, n_pages, page, hkv, d) if held is None else held
    n_pages = codes.shape[0]
    own_tables = tables(gen, n_pages, page, own_lens) if own_tables is None else own_tables
    dev, c, s = fused.cuda(), codes.cuda(), scales.cuda()
    cuda = lambda t: None if t is None else t.cuda()  # noqa: E731
    queries = dict(q=dev[:, :hq], q_weight=cuda(weights[0])) if hq else {}
    got_q = lsm.lsm_kv_append8(dev[:, hq:hq + hkv], dev[:, hq + hkv:hq + 2 * hkv], cuda(positions), batch_of(lsm, q_lens, own_tables, own_lens), c[:, 0], c[:, 1], s[:, 0], s[:, 1],
                               cuda(table), k_weight=cuda(weights[1]), interleaved=interleaved, eps=eps, **queries)
    after, scales_after = c.cpu(), s.cpu()
    where = pages.places(offsets(q_lens), own_tables, own_lens, n_pages, page, fused.shape[0])
    k, v = fused[:, hq:hq + hkv], fused[:, hq + hkv:hq + 2 * hkv]
    if table is None and weights[1] is None:
        y, bound = k.double(), torch.zeros(k.shape, dtype=torch.float64)
    else:
        y, bound = ref.rotate(k.float(), weights[1], table, positions, eps, interleaved)
    pages.check_append8(codes[:, 0], scales[:, 0], after[:, 0], scales_after[:, 0], y, bound, where, fused.dtype)
    pages.check_append8(codes[:, 1], scales[:, 1], after[:, 1], scales_after[:, 1], v.double(), torch.zeros(v.shape, dtype=torch.float64), where, fused.dtype)
    assert torch.equal(dev.cpu().view(torch.uint8), fused.view(torch.uint8))  # inputs are as they were
    if hq:
        ref.assert_within(got_q, *ref.rotate(fused[:, :hq], weights[0], table, positions, eps, interleaved), "queries")
    else:
        assert got_q is None
    return after, scales_after, own_tables


def normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(dtype)


APPEND = [
    # q_lens, own_lens, hq, hkv, d, rot, page, dtype, norm, interleaved
    ([1], [1], 32, 2, 128, 128, 16, BF16, True, False),
    ([1] * 5, [1, 16, 17, 33, 48], 32, 2, 128, 64, 16, BF16, False, True),       # first and last rows of blocks
    ([40, 1, 100, 16, 31], [40, 9, 130, 32, 46], 12, 3, 64, 64, 32, FP16, True, False),
    ([3, 50], [70, 50], 0, 1, 256, 128, 64, BF16, True, False),
    ([21, 2], [25, 2], 3, 3, 40, 20, 48, FP32, True, True),                      # a page of three blocks
    ([7, 33], [20, 33], 5, 2, 80, 40, 16, BF16, True, False),                    # half of the rotated part is no whole number of lanes
    ([5, 17], [21, 30], 2, 2, 8, 2, 16, FP32, False, False),
    ([9], [40], 1, 1, 256, 256, 128, FP32, True, False),
    ([600, 1, 0, 77], [601, 5, 3, 200], 4, 2, 64, 32, 16, FP16, True, True),
    ([1] * 70, list(range(1, 71)), 8, 1, 128, 128, 16, BF16, True, False),       # more requests than lanes
    ([2, 30], [3, 60], 3, 2, 248, 96, 16, FP16, False, False),
]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: f"{len(c[0])}x{c[4]}-{str(c[7])[6:]}")
def test_append8(lsm, case):
    q_lens, own_lens, hq, hkv, d, rot, page, dtype, norm, interleaved = case
    gen = torch.Generator().manual_seed(sum(own_lens) + d)
    n = sum(q_lens)
    fused = normal(gen, (n, hq + 2 * hkv, d), dtype)
    fused[:, hq:] *= torch.exp2(torch.randint(-4, 4, (n, 2 * hkv, 1), generator=gen).to(dtype))
    table = lsm.lsm_rope_table(500, rot).cpu()
    positions = torch.randint(0, 500, (n,), generator=gen, dtype=torch.int32)
    weights = [normal(gen, (d,), FP32 if hq % 2 else dtype) if norm else None for _ in range(2)]
    run(lsm, gen, fused, hq, hkv, d, q_lens, own_lens, page, table=table, positions=positions, weights=weights, interleaved=interleaved, eps=1e-5)


@pytest.mark.parametrize("d, rot, dtype, interleaved", [(128, 128, BF16, False), (64, 32, FP16, True), (256, 64, FP16, False), (128, 64, BF16, True), (64, 64, BF16, False)])
def test_weights_of_32_bits(lsm, d, rot, dtype, interleaved):
    """Elements of 16 bits with weights of 32, rows aligned: kernels of their own, on every kind of pair."""
    gen = torch.Generator().manual_seed(d + rot)
    q_lens, own_lens, hq, hkv = [40, 1, 33, 0, 5], [47, 16, 33, 4, 70], 4, 2
    n = sum(q_lens)
    fused = normal(gen, (n, hq + 2 * hkv, d), dtype)
    table = lsm.lsm_rope_table(300, rot).cpu()
    positions = torch.randint(0, 300, (n,), generator=gen, dtype=torch.int32)
    run(lsm, gen, fused, hq, hkv, d, q_lens, own_lens, 16, table=table, positions=positions, weights=[normal(gen, (d,), FP32) for _ in range(2)], interleaved=interleaved)


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
def test_values_as_they_are_are_rounded_exactly(lsm, dtype):
    """No norm, no rotation: codes are the nearest ones, ties to even; magnitudes of every size, ties, subnormals, zeros."""
    gen = torch.Generator().manual_seed(3)
    n, hkv, d = 64, 2, 128
    x = normal(gen, (n, 2 * hkv, d), FP32) * torch.exp2(torch.randint(-14, 10, (n, 2 * hkv, d), generator=gen).float())
    grid = torch.arange(127, dtype=torch.uint8).view(E4M3).float()
    ties = (grid[1:] + grid[:-1]) / 2  # halfway between neighbouring codes, at scale 1 (the largest is 448)
    x[:16, 0, :126], x[0, 0, 126] = ties[:126], 448.0
    x[16:32, 1] = 0.0
    x[32:48, 2] *= 2.0 ** -9
    run(lsm, gen, x.to(dtype), 0, hkv, d, [64], [64], 16)


def test_what_is_not_finite_and_the_largest_and_smallest(lsm):
    gen = torch.Generator().manual_seed(4)
    for dtype, most, least in ((FP16, 65504.0, 2.0 ** -24), (BF16, 3.3895e38, 1.2e-38), (FP32, 3.4e38, 1e-40)):
        x = normal(gen, (64, 2, 64), dtype)
        x[0, 0, 3], x[1, 0, 5], x[2, 1, 7] = math.inf, math.nan, -math.inf
        x[16:32, 0] *= 0.0
        x[16, 0, 9], x[17, 1, 1], x[18, 1, 2] = most, -most, most
        x[32:48] = least
        x[48:64, 0] = math.nan  # nothing finite in the block
        run(lsm, gen, x, 0, 1, 64, [64], [64], 32)


def test_positions_without_an_angle_give_nan(lsm):
    gen = torch.Generator().manual_seed(5)
    fused = normal(gen, (5, 4, 64), BF16)
    positions = ints([0, -1, 9, 10, 2 ** 31 - 1])
    table = lsm.lsm_rope_table(10, 32)
    c, s = (t.cuda() for t in pool(gen, 4, 16, 1, 64))
    lsm.lsm_kv_append8(fused[:, 2:3].cuda(), fused[:, 3:].cuda(), positions.cuda(), batch_of(lsm, [5], ints([[2]]), [5]), c[:, 0], c[:, 1], s[:, 0], s[:, 1], table)
    nan = torch.isnan(c[2, 0, :5, 0].float()).cpu()
    assert nan[[1, 3, 4], :32].all() and not nan[[0, 2]].any() and not nan[:, 32:].any() and not torch.isnan(c[2, 1].float()).any()


@pytest.mark.parametrize("offset, head_pad, dtype, d", [(1, 0, BF16, 64), (0, 3, BF16, 128), (8, 8, FP16, 64), (3, 1, FP32, 40), (4, 4, BF16, 64)])
def test_any_alignment(lsm, offset, head_pad, dtype, d):
    """Inputs and pages at any address and stride."""
    gen = torch.Generator().manual_seed(offset + d)
    n, hkv, page = 37, 2, 32
    width = d + head_pad
    flat = normal(gen, (offset + n * 2 * hkv * width,), dtype)
    x = flat[offset:].view(n, 2 * hkv, width)[:, :, :d]
    codes, scales = pool(gen, 5, page, hkv, width)
    store, scale_store = codes.cuda(), torch.cat([scales, scales], -1).cuda()[..., ::2]  # scales with gaps
    before, scales_before = store.cpu(), scale_store.cpu()
    own_tables, own_lens, q_lens = tables(gen, 5, page, [50, 20]), [50, 20], [30, 7]
    table, positions = lsm.lsm_rope_table(100, 24), torch.randint(0, 100, (n,), generator=gen, dtype=torch.int32)
    dev = flat.cuda()[offset:].view(n, 2 * hkv, width)[:, :, :d]
    p = store[..., head_pad:] if head_pad else store
    lsm.lsm_kv_append8(dev[:, :hkv], dev[:, hkv:], positions.cuda(), batch_of(lsm, q_lens, own_tables, own_lens), p[:, 0], p[:, 1], scale_store[:, 0], scale_store[:, 1], table)
    where = pages.places(offsets(q_lens), own_tables, own_lens, 5, page, n)
    b, a = before[..., head_pad:], store.cpu()[..., head_pad:]
    pages.check_append8(b[:, 0], scales_before[:, 0], a[:, 0], scale_store.cpu()[:, 0], *ref.rotate(x[:, :hkv].float(), None, table.cpu(), positions), where, dtype)
    pages.check_append8(b[:, 1], scales_before[:, 1], a[:, 1], scale_store.cpu()[:, 1], x[:, hkv:].double(), torch.zeros(n, hkv, d, dtype=torch.float64), where, dtype)
    if head_pad:
        assert torch.equal(before[..., :head_pad].view(torch.uint8), store.cpu()[..., :head_pad].view(torch.uint8))


def test_tokens_without_a_place_are_not_written(lsm):
    """Lengths shorter than the new tokens, beyond the table or below 0, pages that there are not, requests without tokens, tokens of no request."""
    gen = torch.Generator().manual_seed(7)
    q_lens, own_lens = [20, 5, 6, 0, 4, 3, 40], [7, 70, 0, 9, 3, -5, 40]
    own_tables = ints([[0, 1, 9], [2, 3, 9], [4, 9, 9], [5, 9, 9], [-1, 9, 9], [6, 9, 9], [7, 10, 8]])  # pages of 16; 10 and 9 are none
    fused = normal(gen, (sum(q_lens) + 11, 2 + 2 * 2, 64), BF16)  # eleven tokens of no request
    held = pool(gen, 9, 16, 2, 64)
    run(lsm, gen, fused, 2, 2, 64, q_lens, own_lens, 16, held=held, own_tables=own_tables)


def test_a_block_filled_token_by_token(lsm):
    """Magnitudes that rise and fall: scales grow when they must and never shrink, older tokens keep their values within a step of the scale they end up with."""
    gen = torch.Generator().manual_seed(8)
    hkv, d = 2, 64
    held = pool(gen, 3, 32, hkv, d)
    x = normal(gen, (32, 2 * hkv, d), BF16) * torch.exp2(torch.tensor([-3, 0, 2, -9, 4, 4, 6, -12, 1, 0, 9, 3, 2, -2, 12, 0] * 2).to(BF16))[:, None, None]
    own_tables = ints([[1, 7]])
    c, s = held
    for i in range(32):
        c, s, _ = run(lsm, gen, x[i:i + 1], 0, hkv, d, [1], [i + 1], 32, held=(c, s), own_tables=own_tables)
    # each value: half a step of its own rounding, and, where its code became subnormal, half a step of 2^-9 for each of at most 16 raises
    got = pages.decode(c[:, 0], s[:, 0])[1]
    e = pages.two_to(pages.exponents(s[1, 0])).repeat_interleave(16, 0)[..., None]
    want = x[:, :hkv].double()
    assert bool(((got - want).abs() <= want.abs() * 2.0 ** -4 + 17 * e * 2.0 ** -10).all())


def test_a_scale_that_is_nan_stays(lsm):
    gen = torch.Generator().manual_seed(9)
    codes, scales = pool(gen, 2, 16, 1, 64)
    scales.view(torch.uint8)[0, :, 0, 0] = 255
    x = normal(gen, (3, 2, 64), BF16)
    c, s, _ = run(lsm, gen, x, 0, 1, 64, [3], [8], 16, held=(codes, scales), own_tables=ints([[0]]))
    assert s.view(torch.uint8)[0].flatten().tolist() == [255, 255]
    c, s, _ = run(lsm, gen, x, 0, 1, 64, [3], [3], 16, held=(c, s), own_tables=ints([[0]]))  # the block begins anew
    assert max(s.view(torch.uint8)[0].flatten().tolist()) < 255


def test_beyond_four_gigabytes(lsm):
    page, hkv, d = 16, 8, 128
    n_pages = (1 << 32) // (page * hkv * d) + 64
    codes = torch.empty((n_pages, page, hkv, d), dtype=E4M3, device="cuda")
    scales = torch.zeros((n_pages, 1, hkv), dtype=torch.uint8, device="cuda").view(E8M0)
    gen = torch.Generator().manual_seed(10)
    k = normal(gen, (3, hkv, d), BF16)
    own_tables = ints([[n_pages - 1], [5], [(1 << 32) // (page * hkv * d) + 1]])
    at = own_tables[:, 0].long().cuda()
    codes.view(torch.uint8)[at] = 0
    batch = batch_of(lsm, [1, 1, 1], own_tables, [1, 1, 1])
    lsm.lsm_kv_append8(k.cuda(), k.cuda(), None, batch, codes, codes, scales, scales, None)
    got = pages.decode(codes.view(torch.uint8)[at].cpu().view(E4M3), scales.view(torch.uint8)[at].cpu().view(E8M0))
    for i in range(3):
        e = pages.two_to(pages.exponents(scales.view(torch.uint8)[at[i]].cpu().view(E8M0)))[0][:, None]
        assert torch.equal(got[i, 0], pages.codes_of(k[i].double() / e) * e)
    q = normal(gen, (3, 16, d), BF16)
    out = lsm.lsm_prefix_attention(q.cuda(), codes, codes, batch, k_scales=scales, v_scales=scales)
    few = got.to(BF16)
    want, _, bound, _ = ref.attention(q, few, few, ints([0, 3]), torch.zeros(1, 0), torch.zeros(1), torch.arange(4), torch.arange(3)[:, None], torch.ones(3, dtype=torch.int32))
    ref.assert_within(out, want, bound, "out")


def test_on_another_stream_and_in_a_graph(lsm):
    """Recorded once and replayed on new tokens and lengths in the same memory; eager work and synchronizations in between."""
    gen = torch.Generator().manual_seed(11)
    hq, hkv, d, page, n = 4, 2, 128, 16, 6
    table, weights = lsm.lsm_rope_table(300, d), [normal(gen, (d,), BF16).cuda() for _ in range(2)]
    codes, scales = pool(gen, 30, page, hkv, d)
    x = torch.zeros(n, hq + 2 * hkv, d, dtype=BF16, device="cuda")
    own_tables = torch.randperm(30, generator=gen)[:n * 3].view(n, 3).to(torch.int32)
    positions, lens = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    q_out = torch.zeros(n, hq, d, dtype=BF16, device="cuda")
    batch = lsm.PrefixBatch(*(t.cuda() for t in (ints([0, n]), ints([[]]).reshape(1, 0), ints([0]), torch.arange(n + 1, dtype=torch.int32), own_tables)), lens)

    def call(c, s, **more):
        return lsm.lsm_kv_append8(x[:, hq:hq + hkv], x[:, hq + hkv:], positions, batch, c[:, 0], c[:, 1], s[:, 0], s[:, 1], table, k_weight=weights[1], q=x[:, :hq], q_weight=weights[0], **more)

    one, two, three = ((codes.cuda(), scales.cuda()) for _ in range(3))
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    call(*three, q_out=q_out)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call(*one, q_out=q_out)
    for i in range(4):
        x.copy_(normal(gen, x.shape, BF16, 2.0 ** i))
        lens.copy_(torch.arange(n, dtype=torch.int32) * 7 + i + 1)
        positions.copy_(lens - 1)
        torch.cuda.synchronize()
        graph.replay()
        want_q = call(*two)
        torch.cuda.synchronize()
        assert torch.equal(q_out, want_q)
        assert torch.equal(one[0].view(torch.uint8), two[0].view(torch.uint8)) and torch.equal(one[1].view(torch.uint8), two[1].view(torch.uint8))
        if i == 0:
            three = (codes.cuda(), scales.cuda())
        side.wait_stream(torch.cuda.current_stream())
        call(*three, stream=side)
        side.synchronize()
        assert torch.equal(three[0].view(torch.uint8), two[0].view(torch.uint8)) and torch.equal(three[1].view(torch.uint8), two[1].view(torch.uint8))
