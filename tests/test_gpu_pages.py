"""Copying and compacting pages on the GPU against plain implementations (tests/pages_reference.py)."""
import pytest
import torch

import pages_reference as pages

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsm():
    import paper_2511_16138_amd as lsm
    return lsm


def ints(v):
    return torch.tensor(v, dtype=torch.int32)


def random_bytes(gen, shape):
    return torch.randint(0, 256, shape, generator=gen, dtype=torch.uint8)


def buffers(gen, n, kinds):
    """Buffers of n pages (on the CPU): as they are used, and the memory around them."""
    made = []
    for kind in kinds:
        if kind == "blocks":          # all layers side by side
            made.append(random_bytes(gen, (n, 3, 2, 16, 2, 64)))
        elif kind == "layer":         # a layer's slice of blocks: pages with gaps between them
            made.append(random_bytes(gen, (n, 3, 16, 2, 64))[:, 1])
        elif kind == "long":          # more than one piece of a workgroup, no whole number of them
            made.append(random_bytes(gen, (n, 16384 * 3 + 48)))
        elif kind == "odd":           # no multiple of 16 bytes
            made.append(random_bytes(gen, (n, 37)))
        elif kind == "long odd":
            made.append(random_bytes(gen, (n, 40001)))
        elif kind == "unaligned":     # a multiple of 16 bytes at an address that is none
            made.append(random_bytes(gen, (n * 64 + 8,))[8:].view(n, 64))
        elif kind == "turned":        # a page's dimensions in another order
            made.append(random_bytes(gen, (n, 4, 8, 16)).permute(0, 3, 1, 2))
        elif kind == "half":
            made.append(random_bytes(gen, (n, 16, 4, 32)).view(torch.float16))
        elif kind == "one byte":
            made.append(random_bytes(gen, (n,)))
        elif kind == "empty":
            made.append(random_bytes(gen, (n, 0, 5)))
    return made


def on_gpu(made):
    """The same with the same strides, and the memory that they lie in."""
    out = []
    for t in made:
        base = t._base if t._base is not None else t
        flat = torch.empty(base.untyped_storage().nbytes(), dtype=torch.uint8, device="cuda")
        flat.copy_(torch.empty(0, dtype=torch.uint8).set_(base.untyped_storage()))
        size = t.element_size()
        out.append((torch.empty(0, dtype=t.dtype, device="cuda").set_(flat.untyped_storage(), t.storage_offset(), t.shape, t.stride()), flat, size))
    return out


KINDS = [["blocks"], ["layer", "odd"], ["long", "unaligned", "empty", "one byte"], ["turned", "half", "long odd"], ["empty"], ["layer"] * 70 + ["odd"]]


def same_bytes(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)) if a.numel() else a.shape == b.shape


@pytest.mark.parametrize("kinds", KINDS, ids=lambda k: "-".join(k[:3]) + str(len(k)))
@pytest.mark.parametrize("n, copies", [(1, 1), (7, 3), (60, 29)])
def test_copy_pages(lsm, kinds, n, copies):
    gen = torch.Generator().manual_seed(n + len(kinds))
    made = buffers(gen, n, kinds)
    held = on_gpu(made)
    order = torch.randperm(n, generator=gen).tolist()
    targets = order[:copies]
    rest = order[copies:] or order
    sources = [rest[i % len(rest)] for i in range(copies)]      # some of them several times
    pairs = list(zip(sources, targets))
    bad = [(-1, order[-1]), (order[-1], n), (2 ** 31 - 1, 0), (order[-1], -2 ** 31), (order[-1], order[-1])]
    mixed = bad[:2] + pairs + bad[2:]
    flat_before = [f.clone() for _, f, _ in held]
    lsm.lsm_copy_pages([t for t, _, _ in held], ints([s for s, _ in mixed]).cuda(), ints([t for _, t in mixed]).cuda())
    for (t, flat, _), before, around in zip(held, made, flat_before):
        want = before.clone()
        for s, d in pairs:
            want[d] = before[s]
        assert same_bytes(t.cpu(), want)
        # and nothing around them
        torch.empty(0, dtype=t.dtype, device="cuda").set_(around.untyped_storage(), t.storage_offset(), t.shape, t.stride()).copy_(want)
        assert torch.equal(flat, around)


def test_copy_pages_of_one_tensor_and_of_none(lsm):
    gen = torch.Generator().manual_seed(1)
    x = random_bytes(gen, (9, 64)).cuda()
    want = x.clone()
    version = x._version
    want[3] = want[8]
    lsm.lsm_copy_pages(x, ints([8]).cuda(), ints([3]).cuda())
    assert torch.equal(x, want) and x._version > version
    lsm.lsm_copy_pages([], ints([8]).cuda(), ints([3]).cuda())
    lsm.lsm_copy_pages(x, ints([]).cuda(), ints([]).cuda())
    assert torch.equal(x, want)


def test_copy_of_many_pages_and_offsets_past_32_bits(lsm):
    n, bytes_ = 70000, 1 << 16          # 4.6 GB
    x = torch.empty((n, bytes_), dtype=torch.uint8, device="cuda")
    gen = torch.Generator().manual_seed(2)
    order = torch.randperm(n, generator=gen).to(torch.int32)
    sources, targets = order[:30000].cuda(), order[30000:60000].cuda()
    x[sources.long()] = (sources.long() % 251).to(torch.uint8)[:, None]
    x[targets.long()] = 255
    lsm.lsm_copy_pages(x, sources, targets)
    assert bool((x[targets.long()] == (sources.long() % 251).to(torch.uint8)[:, None]).all())
    assert bool((x[sources.long()] == (sources.long() % 251).to(torch.uint8)[:, None]).all())


def check_compact(lsm, n, page_tokens, tables, lens, kinds, gen, **more):
    made = buffers(gen, n, kinds)
    held = on_gpu(made)
    dev = [t.cuda() for t in tables]
    got, moved, n_live = lsm.lsm_compact_pages([t for t, _, _ in held], dev, [x.cuda() for x in lens], page_tokens, **more)
    want, want_moved, want_live = pages.compact(n, page_tokens, [t.tolist() for t in tables], [x.tolist() for x in lens])
    assert n_live.tolist() == [want_live] and moved.tolist() == want_moved
    for t, old, g, w in zip(tables, dev, got, want):
        assert g.dtype == torch.int32 and g.shape == t.shape and g.tolist() == w
        assert torch.equal(old.cpu(), t)
    for (t, _, _), before in zip(held, made):
        expect = before.clone()
        for p, q in enumerate(want_moved):
            if q >= 0:
                expect[q] = before[p]
        assert same_bytes(t.cpu(), expect)
    return want_live


@pytest.mark.parametrize("n", [1, 2, 31, 33, 64, 700, 5000])
@pytest.mark.parametrize("share", [0.0, 0.1, 0.5, 0.95, 1.0])
def test_compact_pages(lsm, n, share):
    gen = torch.Generator().manual_seed(n)
    live = torch.randperm(n, generator=gen)[:int(n * share)]
    page, width = 16, 40
    # rows of any length, one prefix that several rows share, garbage behind the lengths, holes
    rows, at = [], 0
    while at < live.shape[0]:
        c = int(torch.randint(1, width, (1,), generator=gen))
        rows.append(live[at:at + c].tolist())
        at += c
    rows.append([])
    if len(rows) > 2:
        rows.append(rows[0][:5])
        rows.append([-1] + rows[1][:3] + [n, 2 ** 31 - 1] + rows[1][:1])
    lens = ints([max(0, len(r) * page - int(torch.randint(0, page, (1,), generator=gen))) for r in rows])
    lens[len([r for r in rows if r]) and rows.index([])] = -3
    table = torch.randint(0, n, (len(rows), width + 3), generator=gen, dtype=torch.int32)
    for i, r in enumerate(rows):
        table[i, :len(r)] = ints(r)
    check_compact(lsm, n, page, [table], [lens], ["layer", "odd"], gen)


def test_compact_pages_of_several_tables_and_many_buffers(lsm):
    gen = torch.Generator().manual_seed(3)
    n, page = 300, 32
    tables = [torch.randint(-5, n + 5, (r, w), generator=gen, dtype=torch.int32) for r, w in ((4, 6), (0, 5), (3, 0), (1, 1), (20, 3))]
    lens = [torch.randint(-10, w * page + 40, (r,), generator=gen, dtype=torch.int32) for r, w in ((4, 6), (0, 5), (3, 0), (1, 1), (20, 3))]
    check_compact(lsm, n, page, tables, lens, ["layer"] * 66 + ["odd"], gen)
    check_compact(lsm, n, page, tables, lens, ["long", "empty"], gen)
    # the plan alone
    got, moved, n_live = lsm.lsm_compact_pages([], [t.cuda() for t in tables], [x.cuda() for x in lens], page, n_pages=n)
    want = pages.compact(n, page, [t.tolist() for t in tables], [x.tolist() for x in lens])
    assert [g.tolist() for g in got] == want[0] and moved.tolist() == want[1] and n_live.tolist() == [want[2]]
    # one table, not in a list; no pages at all
    (alone,), _, _ = lsm.lsm_compact_pages([], tables[0].cuda(), lens[0].cuda(), page, n_pages=n)
    assert alone.tolist() == pages.compact(n, page, [tables[0].tolist()], [lens[0].tolist()])[0][0]
    (alone,), moved, n_live = lsm.lsm_compact_pages([], tables[0].cuda(), lens[0].cuda(), page, n_pages=0)
    assert torch.equal(alone.cpu(), tables[0]) and moved.shape == (0,) and n_live.tolist() == [0]


def test_compact_a_million_pages(lsm):
    """More words of live bits than the planning workgroup has threads."""
    gen = torch.Generator().manual_seed(4)
    n, page = 1_200_007, 16
    live = torch.randperm(n, generator=gen)[:500_000].to(torch.int32)
    table = live.view(500, 1000)
    x = torch.arange(n, dtype=torch.int32, device="cuda")[:, None].repeat(1, 4)
    (new,), moved, n_live = lsm.lsm_compact_pages(x, table.cuda(), torch.full((500,), 16000, dtype=torch.int32).cuda(), page)
    assert n_live.tolist() == [500_000]
    is_live = torch.zeros(n, dtype=torch.bool)
    is_live[live.long()] = True
    number = torch.arange(n)
    want = torch.where(is_live, number, torch.full_like(number, -1))
    movers, holes = torch.nonzero(is_live & (number >= 500_000)).flatten(), torch.nonzero(~is_live[:500_000]).flatten()
    want[movers] = holes
    assert torch.equal(moved.cpu().long(), want) and torch.equal(new.cpu().long(), want[table.long()])
    assert torch.equal(x[new.long().flatten(), 0].cpu(), table.flatten())


def test_compaction_in_a_graph_and_on_another_stream(lsm):
    gen = torch.Generator().manual_seed(5)
    n, page = 500, 16
    x, out = torch.zeros(n, 160, dtype=torch.uint8, device="cuda"), None
    table, lens = torch.zeros(10, 30, dtype=torch.int32, device="cuda"), torch.zeros(10, dtype=torch.int32, device="cuda")
    lsm.lsm_compact_pages(x, table, lens, page)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = lsm.lsm_compact_pages(x, table, lens, page)
        lsm.lsm_copy_pages(x, table[0, :5], table[1, :5])
    side = torch.cuda.Stream()
    for i in range(4):
        order = torch.randperm(n, generator=gen)[:300].view(10, 30).to(torch.int32)
        data = random_bytes(gen, (n, 160))
        table.copy_(order), lens.copy_(torch.randint(0, 481, (10,), generator=gen, dtype=torch.int32)), x.copy_(data)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        y = data.cuda()
        side.wait_stream(torch.cuda.current_stream())
        again = lsm.lsm_compact_pages(y, table, lens, page, stream=side)
        lsm.lsm_copy_pages(y, table[0, :5], table[1, :5], stream=side)
        side.synchronize()
        want = pages.compact(n, page, [order.tolist()], [lens.tolist()])
        for got in (out, again):
            assert got[0][0].tolist() == want[0][0] and got[1].tolist() == want[1] and got[2].tolist() == [want[2]]
        expect = data.clone()
        for p, q in enumerate(want[1]):
            if q >= 0:
                expect[q] = data[p]
        before = expect.clone()
        for s, d in zip(order[0, :5].tolist(), order[1, :5].tolist()):
            expect[d] = before[s]
        assert torch.equal(x.cpu(), expect) and torch.equal(y.cpu(), expect)
