"""CPU-only checks of the calls of include/lsm_pages.h: they are exported, refuse bad arguments before anything is launched, size their workspaces, and the plain
implementations that the GPU tests compare with agree with torch and with cases worked by hand.  No kernel is launched here."""
import ctypes as C
import math
import os
import re

import pytest
import torch

import cache_reference as ref
import pages_reference as pages
from test_cache_host import AT, BAD, NULL, WORKSPACE, Attention, Heads, Pages, Rotation, attention, rotation

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Scales(C.Structure):
    _fields_ = [("data", C.c_void_p), ("page_stride", C.c_int64), ("block_stride", C.c_int64), ("head_stride", C.c_int64)]


class NewTokens(C.Structure):
    _fields_ = [("q_offsets", C.c_void_p), ("own_tables", C.c_void_p), ("own_lens", C.c_void_p), ("n_requests", C.c_uint64), ("own_width", C.c_uint64),
                ("n_pages", C.c_uint64), ("page_tokens", C.c_uint64)]


class Window(C.Structure):
    _fields_ = [("base", Attention), ("k_scales", Scales), ("v_scales", Scales), ("window", C.c_uint64), ("sinks", C.c_uint64)]


class Part(C.Structure):
    _fields_ = [("data", C.c_void_p), ("page_stride", C.c_int64), ("page_bytes", C.c_uint64)]


class Table(C.Structure):
    _fields_ = [("pages", C.c_void_p), ("lens", C.c_void_p), ("new_pages", C.c_void_p), ("rows", C.c_uint64), ("width", C.c_uint64)]


@pytest.fixture(scope="module")
def lib():
    import paper_2511_16138_amd.binding as B
    if not os.path.exists(B.library_path()):
        import __graft_entry__
        __graft_entry__.build()
    L = C.CDLL(B.library_path())
    L.lsm_window_attention_workspace_bytes.restype = C.c_size_t
    L.lsm_prefix_attention_workspace_bytes.restype = C.c_size_t
    L.lsm_compact_pages_workspace_bytes.restype = C.c_size_t
    return L


def test_every_declared_call_is_exported_by_library_and_package(lib):
    import paper_2511_16138_amd as lsm
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "lsm_pages.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(lsm_[a-z_0-9]+)\s*\(", text))
    assert {"lsm_kv_append8", "lsm_window_attention", "lsm_window_attention_workspace_bytes", "lsm_copy_pages", "lsm_compact_pages", "lsm_compact_pages_workspace_bytes"} == names
    for name in names:
        assert hasattr(lib, name), name
    for name in ("lsm_kv_append8", "lsm_copy_pages", "lsm_compact_pages"):
        assert callable(getattr(lsm, name)) and name in lsm.__all__


# ---------------------------------------------------------------------------------------------------------------------
# refusals of the library
# ---------------------------------------------------------------------------------------------------------------------
def append8(lib, how=None, k=Heads(AT, 1024, 128, 8), v=Heads(AT, 1024, 128, 8), k_pages=Pages(AT, 16 * 1024, 1024, 128), v_pages=Pages(AT, 16 * 1024, 1024, 128), k_scales=Scales(AT, 8, 8, 1),
            v_scales=Scales(AT, 8, 8, 1), k_weight=None, to=None, q=None, q_out=None, **change):
    new = dict(q_offsets=AT, own_tables=AT, own_lens=AT, n_requests=3, own_width=4, n_pages=50, page_tokens=16)
    new.update(change)
    to = NewTokens(*(new[n] for n, _ in NewTokens._fields_)) if to is None else to
    p = lambda x: None if x is None else C.byref(x)  # noqa: E731
    return lib.lsm_kv_append8(p(how or rotation()), p(k), C.c_void_p(k_weight), p(v), p(to) if to else None, p(k_pages), p(k_scales), p(v_pages), p(v_scales), p(q), None, p(q_out), None)


@pytest.mark.parametrize("change, rc", [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(k_pages=None), NULL), (dict(v_pages=None), NULL), (dict(k_scales=None), NULL), (dict(v_scales=None), NULL), (dict(to=False), NULL),
    (dict(k=Heads(None, 1024, 128, 8)), NULL), (dict(v=Heads(None, 1024, 128, 8)), NULL), (dict(k_pages=Pages(None, 16 * 1024, 1024, 128)), NULL), (dict(v_scales=Scales(None, 8, 8, 1)), NULL),
    (dict(k=Heads(AT, 1024, 128, 4)), BAD), (dict(k=Heads(AT + 1, 1024, 128, 8)), BAD), (dict(k=Heads(AT, 0, 128, 1 << 17), v=Heads(AT, 0, 128, 1 << 17)), BAD), (dict(k_weight=AT + 1), BAD),
    (dict(q_offsets=None), NULL), (dict(own_tables=None), NULL), (dict(own_lens=None), NULL), (dict(q_offsets=AT + 2), BAD), (dict(own_lens=AT + 1), BAD), (dict(own_tables=AT + 3), BAD),
    (dict(page_tokens=0), BAD), (dict(page_tokens=24), BAD), (dict(page_tokens=8), BAD), (dict(page_tokens=1 << 30), BAD), (dict(own_width=1 << 26), BAD), (dict(own_width=1 << 60), BAD),
    (dict(n_requests=1 << 24), BAD), (dict(n_pages=1 << 31), BAD), (dict(how=rotation(n_tokens=1 << 24)), BAD), (dict(how=rotation(head_dim=12)), BAD), (dict(how=rotation(positions=None)), NULL),
    (dict(how=rotation(dtype=5)), BAD), (dict(q=Heads(AT, 1024, 128, 8)), NULL), (dict(q=Heads(AT, 1024, 128, 8), q_out=Heads(AT, 1024, 128, 4)), BAD)])
def test_append8_refusals(lib, change, rc):
    assert append8(lib, **change) == rc


def test_append8_of_nothing_is_no_error(lib):
    none = dict(k=Heads(None, 1024, 128, 8), v=Heads(None, 1024, 128, 8), k_pages=Pages(None, 0, 0, 0), v_pages=Pages(None, 0, 0, 0), k_scales=Scales(None, 0, 0, 0), v_scales=Scales(None, 0, 0, 0))
    assert append8(lib, how=rotation(n_tokens=0, positions=None), **none) == 0
    assert append8(lib, n_requests=0, q_offsets=None, own_tables=None, own_lens=None, **none) == 0
    assert append8(lib, n_pages=0, own_tables=None, **none) == 0


def window(base=None, k_scales=Scales(AT, 8, 8, 1), v_scales=Scales(AT, 8, 8, 1), w=0, sinks=0, **change):
    return Window(base or attention(**change), k_scales, v_scales, w, sinks)


NO_SCALES = Scales(None, 0, 0, 0)


@pytest.mark.parametrize("change, rc", [
    (dict(k_scales=NO_SCALES), NULL), (dict(v_scales=NO_SCALES), NULL), (dict(sinks=4), BAD), (dict(w=1 << 30), BAD), (dict(w=5, sinks=1 << 30), BAD), (dict(w=1 << 63), BAD), (dict(w=9, own_width=1 << 25, prefix_width=1 << 25), BAD),
    (dict(dtype=2), BAD), (dict(head_dim=96), BAD), (dict(page_tokens=8), BAD), (dict(scale=0.0), BAD), (dict(w=7, scale=math.nan), BAD), (dict(q_offsets=None), NULL),
    (dict(own_lens=None), NULL), (dict(k_pages=Pages(None, 1 << 15, 1024, 128)), NULL),
    (dict(k_pages=Pages(AT, 1 << 15, 1024 + 8, 128)), BAD), (dict(v_pages=Pages(AT + 8, 1 << 15, 1024, 128)), BAD),      # 8 bytes are no row's alignment in 8 bits
    (dict(k_pages=Pages(AT, 1 << 31, 1024, 128)), BAD), (dict(v_pages=Pages(AT, -(1 << 15), 1024, 128)), BAD), (dict(n_tokens=1 << 24), BAD)])
def test_window_attention_refusals(lib, change, rc):
    a = window(**change)
    assert lib.lsm_window_attention(C.byref(a), C.c_void_p(AT), C.c_size_t(1 << 40), None) == rc
    assert lib.lsm_window_attention_workspace_bytes(C.byref(a)) == 0


def test_window_attention_workspace(lib):
    assert lib.lsm_window_attention(None, None, C.c_size_t(0), None) == NULL and lib.lsm_window_attention_workspace_bytes(None) == 0
    row = 128 * 4 + 8
    a = window()
    need = lib.lsm_window_attention_workspace_bytes(C.byref(a))
    assert need % (300 * 32 * row) == 0 and need >= 2 * 300 * 32 * row  # both stages have parts
    for ws, size in ((None, need), (AT, need - 1), (AT + 128, need)):
        assert lib.lsm_window_attention(C.byref(a), C.c_void_p(ws), C.c_size_t(size), None) == WORKSPACE
    # without scales and window it is the other call
    b = window(k_scales=NO_SCALES, v_scales=NO_SCALES)
    assert lib.lsm_window_attention_workspace_bytes(C.byref(b)) == lib.lsm_prefix_attention_workspace_bytes(C.byref(b.base))
    # a short window needs no parts, however long the tables are; a long one of few requests does
    assert lib.lsm_window_attention_workspace_bytes(C.byref(window(w=256, sinks=4))) == 0
    few = dict(n_tokens=1, n_requests=1, n_groups=1, own_width=1 << 20, kv_heads=1)
    assert 0 < lib.lsm_window_attention_workspace_bytes(C.byref(window(w=1 << 20, **few))) <= 64 * 32 * row
    empty = window(n_tokens=0, n_requests=0, n_groups=0)
    assert lib.lsm_window_attention_workspace_bytes(C.byref(empty)) == 0 and lib.lsm_window_attention(C.byref(empty), None, C.c_size_t(0), None) == 0


def parts_of(*parts):
    return (Part * max(1, len(parts)))(*parts), C.c_uint64(len(parts))


GOOD = Part(AT, 4096, 4096)


@pytest.mark.parametrize("parts, n_pages, sources, targets, n, rc", [
    ([GOOD], 1 << 30, AT, AT, 4, BAD), ([GOOD] * 1025, 9, AT, AT, 4, BAD), ([Part(AT, 1 << 40, 1 << 36)], 9, AT, AT, 4, BAD), ([Part(None, 64, 64)], 9, AT, AT, 4, NULL),
    ([GOOD], 9, None, AT, 4, NULL), ([GOOD], 9, AT, None, 4, NULL), ([GOOD], 9, AT + 2, AT, 4, BAD), ([GOOD], 9, AT, AT + 1, 4, BAD), ([GOOD], 9, AT, AT, 1 << 31, BAD),
    ([], 9, None, None, 4, 0), ([GOOD], 9, None, None, 0, 0), ([GOOD], 0, None, None, 4, 0)])
def test_copy_pages_refusals(lib, parts, n_pages, sources, targets, n, rc):
    p, count = parts_of(*parts)
    assert lib.lsm_copy_pages(p, count, C.c_uint64(n_pages), C.c_void_p(sources), C.c_void_p(targets), C.c_uint64(n), None) == rc


def test_copy_pages_without_a_list(lib):
    assert lib.lsm_copy_pages(None, C.c_uint64(1), C.c_uint64(9), C.c_void_p(AT), C.c_void_p(AT), C.c_uint64(4), None) == NULL


def compact(lib, parts=(GOOD,), n_pages=100, page_tokens=16, tables=(Table(AT, AT, AT, 3, 4),), moved=AT, n_live=AT, workspace=AT, size=None, n_tables=None):
    p, count = parts_of(*parts)
    t = (Table * max(1, len(tables)))(*tables) if tables is not None else None
    return lib.lsm_compact_pages(p, count, C.c_uint64(n_pages), C.c_uint64(page_tokens), t, C.c_uint64(len(tables or ()) if n_tables is None else n_tables), C.c_void_p(moved), C.c_void_p(n_live),
                                 C.c_void_p(workspace), C.c_size_t(lib.lsm_compact_pages_workspace_bytes(C.c_uint64(n_pages)) if size is None else size), None)


@pytest.mark.parametrize("change, rc", [
    (dict(n_pages=1 << 30), BAD), (dict(page_tokens=0), BAD), (dict(page_tokens=1 << 31), BAD), (dict(parts=[Part(None, 64, 64)]), NULL), (dict(tables=None, n_tables=1), NULL),
    (dict(tables=[Table(AT, AT, AT, 1, 1)] * 17), BAD), (dict(tables=[Table(AT, AT, AT, 1 << 16, 1 << 16)]), BAD), (dict(tables=[Table(AT, AT, AT, 1 << 63, 2)]), BAD),
    (dict(tables=[Table(None, AT, AT, 3, 4)]), NULL), (dict(tables=[Table(AT, None, AT, 3, 4)]), NULL), (dict(tables=[Table(AT, AT, None, 3, 4)]), NULL), (dict(tables=[Table(AT + 2, AT, AT, 3, 4)]), BAD),
    (dict(tables=[Table(AT, AT, AT + 1, 3, 4)]), BAD), (dict(moved=None), NULL), (dict(n_live=None), NULL), (dict(moved=AT + 2), BAD), (dict(n_live=AT + 1), BAD),
    (dict(workspace=None), WORKSPACE), (dict(workspace=AT + 64), WORKSPACE), (dict(size=100), WORKSPACE)])
def test_compact_pages_refusals(lib, change, rc):
    assert compact(lib, **change) == rc


def test_compact_pages_workspace(lib):
    last = 0
    for n in (0, 1, 31, 1000, 1 << 20, (1 << 30) - 1):
        size = lib.lsm_compact_pages_workspace_bytes(C.c_uint64(n))
        assert size >= last and n // 8 + 4 * n <= size + 8 <= n // 8 + 4 * n + 2048
        last = size
    assert lib.lsm_compact_pages_workspace_bytes(C.c_uint64(1 << 30)) == 0


# ---------------------------------------------------------------------------------------------------------------------
# refusals of the package
# ---------------------------------------------------------------------------------------------------------------------
def calls(**change):
    import paper_2511_16138_amd as lsm
    t = dict(q=torch.zeros(2, 4, 64, dtype=torch.bfloat16), k=torch.zeros(2, 2, 64, dtype=torch.bfloat16), v=torch.zeros(2, 2, 64, dtype=torch.bfloat16), w=torch.ones(64),
             pages=torch.zeros(3, 16, 2, 64).to(pages.E4M3), scales=torch.ones(3, 1, 2).to(pages.E8M0), positions=torch.zeros(2, dtype=torch.int32), table=torch.zeros(8, 64), out=None,
             rows=torch.zeros(3, 7))
    t.update(change)
    ints = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    batch = lsm.PrefixBatch(ints([0, 2]), ints([[0]]), ints([16]), ints([0, 1, 2]), ints([[1], [2]]), ints([1, 1]))
    return {
        "append8": lambda: lsm.lsm_kv_append8(t["k"], t["v"], t["positions"], batch, t["pages"], t["pages"], t["scales"], t["scales"], t["table"], k_weight=t["w"], q=t["q"], q_out=t["out"]),
        "attend8": lambda: lsm.lsm_prefix_attention(t["q"], t["pages"], t["pages"], batch, k_scales=t["scales"], v_scales=t["scales"], out=t["out"]),
        "window": lambda: lsm.lsm_prefix_attention(t["q"], t["pages"], t["pages"], batch, window=5, out=t["out"]),
        "copy": lambda: lsm.lsm_copy_pages([t["rows"]], ints([0]), ints([1])),
        "compact": lambda: lsm.lsm_compact_pages([t["rows"]], [ints([[0]])], [ints([1])], 16),
    }


@pytest.mark.parametrize("name, what", [("append8", "k"), ("attend8", "q"), ("window", "q"), ("copy", "sources"), ("compact", "a table")])
def test_host_tensors_raise_value_error(name, what):
    with pytest.raises(ValueError, match=f"^{what} must be a GPU tensor"):
        calls()[name]()


@pytest.mark.parametrize("name, change", [("append8", dict(k=5)), ("append8", dict(pages=None)), ("attend8", dict(q=5)), ("attend8", dict(pages=5)), ("window", dict(q="x"))])
def test_what_is_no_tensor_raises_value_error(name, change):
    with pytest.raises(ValueError, match="must be a tensor"):
        calls(**change)[name]()


def test_lists_of_tensors_are_looked_at():
    import paper_2511_16138_amd as lsm
    ints = torch.zeros(1, dtype=torch.int32)
    for bad in (5, "pages", {"a": ints}):
        with pytest.raises(ValueError, match="must be a tensor, or a list or tuple of tensors"):
            lsm.lsm_copy_pages(bad, ints, ints)
    with pytest.raises(ValueError, match="must be a tensor"):
        lsm.lsm_copy_pages([ints], None, ints)
    for tables, lens in (([], []), ([ints[None]], []), ([ints[None]] * 17, [ints] * 17)):
        with pytest.raises(ValueError, match="1 to 16 tables"):
            lsm.lsm_compact_pages([], tables, lens, 16, n_pages=4)


@pytest.mark.parametrize("name, which", [("append8", "k"), ("append8", "v"), ("append8", "w"), ("append8", "q"), ("append8", "table"), ("append8", "out"), ("attend8", "q"), ("attend8", "out"),
                                         ("window", "q"), ("window", "out")])
@pytest.mark.parametrize("kind", ["gradients", "tangent"])
def test_inputs_with_gradients_or_tangents_are_refused(name, which, kind):
    from torch.autograd import forward_ad
    shapes = dict(q=(2, 4, 64), k=(2, 2, 64), v=(2, 2, 64), w=(64,), table=(8, 64), out=(2, 4, 64))
    with forward_ad.dual_level():
        x = torch.zeros(shapes[which], dtype=torch.float32 if which in ("w", "table") else torch.bfloat16)
        x = x.requires_grad_() if kind == "gradients" else forward_ad.make_dual(x, torch.ones_like(x))
        with pytest.raises(ValueError, match=kind):
            calls(**{which: x})[name]()


# ---------------------------------------------------------------------------------------------------------------------
# the plain implementations
# ---------------------------------------------------------------------------------------------------------------------
def test_reference_codes_agree_with_torch():
    grid = torch.arange(127, dtype=torch.uint8).view(pages.E4M3).float()
    assert torch.equal(pages.codes_of(grid.double()).float(), grid)
    ties = (grid[1:] + grid[:-1]) / 2
    x = torch.cat([ties, torch.nextafter(ties, torch.zeros(())), torch.nextafter(ties, torch.full((), 1e9)), torch.logspace(-12, 2.65, 5000)])
    x = torch.cat([x, -x])
    assert torch.equal(pages.codes_of(x.double()).float(), x.to(pages.E4M3).float())


def test_reference_scales():
    for top, e in ((448.0, 0), (448.0001, 1), (447.0, 0), (224.0, -1), (1.0, -8), (0.875, -9), (0.8750001, -8), (0.0, -100), (1e-35, -100), (61440.0, 8), (1.875 * 2.0 ** 127, 120)):
        assert pages.scale_for(top) == e, top
    codes, e = torch.tensor([[[[1.5, -448.0]]]]).to(pages.E4M3).expand(1, 16, 1, 2), torch.tensor([[[130]]], dtype=torch.uint8).view(pages.E8M0)
    assert pages.decode(codes, e)[0, 3, 0].tolist() == [12.0, -3584.0]


def test_reference_window_agrees_with_a_dense_mask():
    """Prefix and own pages, every window: softmax of a masked matrix."""
    gen = torch.Generator().manual_seed(1)
    n, heads, kv, d, page, prefix = 37, 4, 2, 64, 16, 32
    q, k, v = (torch.randn(n, h, d, generator=gen) for h in (heads, kv, kv))
    held = torch.zeros(2, 3, page, kv, d)
    held[0].view(-1, kv, d)[:n], held[1].view(-1, kv, d)[:n] = k, v
    parts = ([0, 1], torch.tensor([[0, 1]]), [prefix], [0, n - prefix], torch.tensor([[2]]), [n - prefix])
    i = torch.arange(n)
    for window, sinks in ((0, 0), (1, 0), (3, 2), (20, 5), (4, 36), (100, 0)):
        out, lse, _, _ = pages.attention(q[prefix:], held[0], held[1], *parts, window=window, sinks=sinks)
        sees = i[None] <= i[prefix:, None]
        if window:
            sees &= (i[None] < sinks) | (i[None] > i[prefix:, None] - window)
        s = torch.einsum("qhd,khd->hqk", q[prefix:].double(), k.double().repeat_interleave(2, 1)) / d ** 0.5
        s = s.masked_fill(~sees, -math.inf)
        assert torch.allclose(out, torch.einsum("hqk,khd->qhd", torch.softmax(s, -1), v.double().repeat_interleave(2, 1)), atol=1e-12)
        assert torch.allclose(lse, torch.logsumexp(s, -1).T, atol=1e-12)
    plain = ref.attention(q[prefix:], held[0], held[1], *parts)
    ours = pages.attention(q[prefix:], held[0], held[1], *parts)
    assert all(torch.allclose(a, b, rtol=1e-6, atol=1e-12) for a, b in zip(plain, ours))


def test_reference_compaction_worked_by_hand():
    # ten pages; 7, 2, 9 and 4 are held: four live ones, so 2 stays, 4, 7 and 9 go to 0, 1 and 3
    tables, moved, n = pages.compact(10, 16, [[[7, 2, 5], [9, -1, 4], [3, 3, 3]]], [[32, 33, 0]])
    assert n == 4 and moved == [-1, -1, 2, -1, 0, -1, -1, 1, -1, 3] and tables == [[[1, 2, 5], [3, -1, 0], [3, 3, 3]]]
    assert pages.compact(3, 16, [], []) == ([], [-1, -1, -1], 0)
