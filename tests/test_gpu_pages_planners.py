"""Compaction by either planner (one launch for up to 2^15 entries and 2^19 pages, several for more) on tables with holes, shared pages and anything behind the
lengths; tables rewritten in place; the longer way in a graph."""
import ctypes as C

import pytest
import torch

import pages_reference as pages
from test_gpu_pages import check_compact, ints, random_bytes
from test_pages_host import Part, Table

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsm():
    import paper_2511_16138_amd as lsm
    return lsm


def tables_of(gen, n, page, shapes, live):
    """Tables that hold about `live` of n pages: some in one row, some in many, holes of either sign, lengths from below 0 to beyond the table."""
    some = torch.randperm(n, generator=gen)[:live].to(torch.int32)
    tables, lens = [], []
    for rows, width in shapes:
        t = some[torch.randint(0, live, (rows, width), generator=gen)]
        t[:, :width // 4] = some[torch.arange(width // 4) % live]               # a prefix of all rows
        hole = torch.rand((rows, width), generator=gen) < 0.02
        t = torch.where(hole, torch.randint(-2 ** 31, 2 ** 31, (rows, width), generator=gen, dtype=torch.int64).to(torch.int32), t)
        t[:, 0] = torch.where(torch.rand(rows, generator=gen) < 0.1, torch.full((), n, dtype=torch.int32), t[:, 0])
        length = torch.randint(-20, (width + 2) * page, (rows,), generator=gen, dtype=torch.int32)
        behind = torch.arange(width)[None] * page >= length[:, None]
        t = torch.where(behind, torch.randint(0, n, (rows, width), generator=gen, dtype=torch.int32), t)  # pages that nobody holds
        tables.append(t.contiguous()), lens.append(length)
    return tables, lens


LONG = [(300, 100), (1, 700), (0, 9), (400, 17)]


@pytest.mark.parametrize("n", [40, 700, 5000, 40007])
@pytest.mark.parametrize("share", [0.3, 0.9])
def test_long_tables(lsm, n, share):
    gen = torch.Generator().manual_seed(n)
    tables, lens = tables_of(gen, n, 16, LONG, max(4, int(n * share)))
    assert sum(t.numel() for t in tables) > 1 << 15
    assert check_compact(lsm, n, 16, tables, lens, ["layer", "odd"] if n < 10000 else ["odd"], gen) > 3


@pytest.mark.parametrize("width", [255, 256, 257])
def test_entries_about_the_border_between_planners(lsm, width):
    gen = torch.Generator().manual_seed(width)
    tables, lens = tables_of(gen, 3000, 16, [(64, width), (64, 256)], 2000)
    check_compact(lsm, 3000, 16, tables, lens, ["odd"], gen)


@pytest.mark.parametrize("n", [(1 << 19) - 1, 1 << 19, (1 << 19) + 1])
def test_pages_about_the_border_between_planners(lsm, n):
    gen = torch.Generator().manual_seed(n & 3)
    tables, lens = tables_of(gen, n, 32, [(20, 300)], 6000)
    tables[0][0, :2], lens[0][0] = ints([n - 1, 0]), 64
    check_compact(lsm, n, 32, tables, lens, ["one byte"], gen)


@pytest.mark.parametrize("shapes", [[(9, 40), (3, 5)], LONG])
def test_tables_rewritten_in_place(lsm, shapes):
    """By the C ABI: the package always makes new ones."""
    gen = torch.Generator().manual_seed(len(shapes))
    n, page = 900, 16
    tables, lens = tables_of(gen, n, page, shapes, 500)
    dev, dev_lens = [t.cuda() for t in tables], [x.cuda() for x in lens]
    before = random_bytes(gen, (n, 80))
    x, moved, n_live = before.cuda(), torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
    library = C.CDLL(lsm.library_path())
    library.lsm_compact_pages_workspace_bytes.restype = C.c_size_t
    size = library.lsm_compact_pages_workspace_bytes(C.c_uint64(n))
    space = torch.empty(size, dtype=torch.uint8, device="cuda")
    parts = (Part * 1)(Part(x.data_ptr(), 80, 80))
    held = (Table * len(dev))(*(Table(t.data_ptr(), s.data_ptr(), t.data_ptr(), t.shape[0], t.shape[1]) for t, s in zip(dev, dev_lens)))
    torch.cuda.synchronize()
    rc = library.lsm_compact_pages(parts, C.c_uint64(1), C.c_uint64(n), C.c_uint64(page), held, C.c_uint64(len(dev)), C.c_void_p(moved.data_ptr()), C.c_void_p(n_live.data_ptr()),
                                   C.c_void_p(space.data_ptr()), C.c_size_t(size), C.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert rc == 0
    torch.cuda.synchronize()
    want, want_moved, want_live = pages.compact(n, page, [t.tolist() for t in tables], [s.tolist() for s in lens])
    assert [t.tolist() for t in dev] == want and moved.tolist() == want_moved and n_live.tolist() == [want_live]
    expect = before.clone()
    for p, q in enumerate(want_moved):
        if q >= 0:
            expect[q] = before[p]
    assert torch.equal(x.cpu(), expect)


def test_long_tables_in_a_graph(lsm):
    """Recorded once, replayed on new tables, lengths and pages in the same memory; eager work and synchronizations in between."""
    gen = torch.Generator().manual_seed(6)
    n, page, shape = 3000, 16, (150, 230)
    assert shape[0] * shape[1] > 1 << 15
    x, table, lens = torch.zeros(n, 48, dtype=torch.uint8, device="cuda"), torch.zeros(shape, dtype=torch.int32, device="cuda"), torch.zeros(shape[0], dtype=torch.int32, device="cuda")
    lsm.lsm_compact_pages(x, table, lens, page)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = lsm.lsm_compact_pages(x, table, lens, page)
    for i in range(4):
        (t,), (length,) = tables_of(gen, n, page, [shape], 300 + 700 * i)
        data = random_bytes(gen, (n, 48))
        table.copy_(t), lens.copy_(length), x.copy_(data)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        y = data.cuda()
        again = lsm.lsm_compact_pages(y, t.cuda(), length.cuda(), page)
        want, want_moved, want_live = pages.compact(n, page, [t.tolist()], [length.tolist()])
        for got in (out, again):
            assert got[0][0].tolist() == want[0] and got[1].tolist() == want_moved and got[2].tolist() == [want_live]
        assert torch.equal(x, y)
