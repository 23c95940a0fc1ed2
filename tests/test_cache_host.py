"""CPU-only checks of the paged-cache calls: they are exported, refuse bad arguments before anything is launched, size their workspaces, and the plain
implementation that the GPU tests compare with agrees with torch.  No kernel is launched here."""
import ctypes as C
import math
import os
import re

import pytest
import torch

import cache_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, BAD, WORKSPACE = -1, -2, -4


class Heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64), ("heads", C.c_uint64)]


class Pages(C.Structure):
    _fields_ = [("data", C.c_void_p), ("page_stride", C.c_int64), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class Rotation(C.Structure):
    _fields_ = [("positions", C.c_void_p), ("table", C.c_void_p), ("n_positions", C.c_uint64), ("n_tokens", C.c_uint64), ("rot_dim", C.c_uint32),
                ("head_dim", C.c_uint32), ("dtype", C.c_uint32), ("weight_dtype", C.c_uint32), ("interleaved", C.c_uint32), ("eps", C.c_float)]


class Attention(C.Structure):
    _fields_ = [("q", Heads), ("out", Heads), ("lse", C.c_void_p), ("k_pages", Pages), ("v_pages", Pages), ("group_offsets", C.c_void_p),
                ("prefix_tables", C.c_void_p), ("prefix_lens", C.c_void_p), ("q_offsets", C.c_void_p), ("own_tables", C.c_void_p), ("own_lens", C.c_void_p),
                ("n_tokens", C.c_uint64), ("n_requests", C.c_uint64), ("n_groups", C.c_uint64), ("prefix_width", C.c_uint64), ("own_width", C.c_uint64),
                ("n_pages", C.c_uint64), ("page_tokens", C.c_uint64), ("kv_heads", C.c_uint64), ("head_dim", C.c_uint32), ("dtype", C.c_uint32),
                ("scale", C.c_float), ("reserved", C.c_uint32)]


@pytest.fixture(scope="module")
def lib():
    import paper_2511_16138_amd.binding as B
    if not os.path.exists(B.library_path()):
        import __graft_entry__
        __graft_entry__.build()
    L = C.CDLL(B.library_path())
    L.lsm_prefix_attention_workspace_bytes.restype = C.c_size_t
    L.lsm_rope_table.argtypes = [C.c_void_p, C.c_uint64, C.c_uint32, C.c_double, C.c_void_p]
    return L


def test_every_declared_call_is_exported_by_library_and_package(lib):
    import paper_2511_16138_amd as lsm
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "lsm_cache.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(lsm_[a-z_]+)\s*\(", text))
    assert {"lsm_rope_table", "lsm_rotate_heads", "lsm_kv_append", "lsm_prefix_attention", "lsm_prefix_attention_workspace_bytes"} == names
    for name in names:
        assert hasattr(lib, name), name
    for name in names - {"lsm_prefix_attention_workspace_bytes"}:
        assert callable(getattr(lsm, name)) and name in lsm.__all__
    assert "PrefixBatch" in lsm.__all__


AT = 1 << 20  # an address that nothing may touch


def rotation(**change):
    how = dict(positions=AT, table=AT, n_positions=100, n_tokens=4, rot_dim=64, head_dim=128, dtype=0, weight_dtype=0, interleaved=0, eps=1e-6)
    how.update(change)
    return Rotation(*(how[n] for n, _ in Rotation._fields_))


def test_rope_table_refusals(lib):
    for args, rc in (((None, 8, 64, 1e4), NULL), ((AT, 8, 63, 1e4), BAD), ((AT, 8, 0, 1e4), BAD), ((AT, 8, 258, 1e4), BAD), ((AT, 8, 64, 0.0), BAD),
                     ((AT, 8, 64, math.nan), BAD), ((AT, 1 << 31, 64, 1e4), BAD), ((AT + 2, 8, 64, 1e4), BAD)):
        assert lib.lsm_rope_table(*args, None) == rc, args
    assert lib.lsm_rope_table(None, 0, 64, 1e4, None) == 0


@pytest.mark.parametrize("change, rc", [
    (dict(head_dim=0), BAD), (dict(head_dim=12), BAD), (dict(head_dim=264), BAD), (dict(rot_dim=63), BAD), (dict(rot_dim=0), BAD), (dict(rot_dim=130), BAD),
    (dict(dtype=3), BAD), (dict(weight_dtype=1), BAD), (dict(interleaved=2), BAD), (dict(eps=-1.0), BAD), (dict(eps=math.nan), BAD), (dict(n_positions=0), BAD),
    (dict(n_tokens=1 << 31), BAD), (dict(positions=None), NULL), (dict(positions=AT + 1), BAD), (dict(table=AT + 2), BAD)])
def test_rotation_refusals(lib, change, rc):
    q, p = Heads(AT, 1024, 128, 8), Pages(AT, 16 * 1024, 1024, 128)
    how = rotation(**change)
    assert lib.lsm_rotate_heads(C.byref(how), C.byref(q), None, C.byref(q), None, None, None, None) == rc
    assert lib.lsm_kv_append(C.byref(how), C.byref(q), None, C.byref(q), C.c_void_p(AT), C.byref(p), C.byref(p), C.c_uint64(4), C.c_uint64(16), None, None, None, None) == rc


def test_heads_and_pages_refusals(lib):
    how, good, p = rotation(), Heads(AT, 1024, 128, 8), Pages(AT, 16 * 1024, 1024, 128)

    def rotate(q, out, weight=None):
        return lib.lsm_rotate_heads(C.byref(how), C.byref(q), C.c_void_p(weight), None if out is None else C.byref(out), None, None, None, None)

    def append(k=good, v=good, slots=AT, kp=p, vp=p, pages=4, page=16):
        ref_or_none = lambda x: None if x is None else C.byref(x)  # noqa: E731
        return lib.lsm_kv_append(C.byref(how), ref_or_none(k), None, ref_or_none(v), C.c_void_p(slots), ref_or_none(kp), ref_or_none(vp), C.c_uint64(pages), C.c_uint64(page), None,
                                 None, None, None)

    assert lib.lsm_rotate_heads(None, C.byref(good), None, C.byref(good), None, None, None, None) == NULL
    assert rotate(good, None) == NULL
    assert rotate(Heads(None, 1024, 128, 8), good) == NULL and rotate(good, Heads(None, 1024, 128, 8)) == NULL
    assert rotate(good, Heads(AT, 1024, 128, 4)) == BAD                    # another number of heads
    assert rotate(Heads(AT + 1, 1024, 128, 8), good) == BAD                # not even an element's alignment
    assert rotate(good, good, AT + 1) == BAD
    assert rotate(Heads(AT, 0, 128, 1 << 17), Heads(AT, 0, 128, 1 << 17)) == BAD
    assert append(k=None) == NULL and append(v=None) == NULL and append(kp=None) == NULL and append(vp=None) == NULL and append(slots=None) == NULL
    assert append(v=Heads(AT, 1024, 128, 4)) == BAD
    assert append(slots=AT + 4) == BAD
    assert append(page=0) == BAD and append(pages=1 << 31) == BAD and append(page=1 << 31) == BAD
    assert append(kp=Pages(None, 16 * 1024, 1024, 128)) == NULL
    # nothing to do is no error
    how = rotation(n_tokens=0, positions=None)
    assert rotate(Heads(None, 1024, 128, 8), Heads(None, 1024, 128, 8)) == 0 and append(slots=None) == 0


def attention(**change):
    a = dict(q=Heads(AT, 4096, 128, 32), out=Heads(AT, 4096, 128, 32), lse=None, k_pages=Pages(AT, 1 << 15, 1024, 128), v_pages=Pages(AT, 1 << 15, 1024, 128),
             group_offsets=AT, prefix_tables=AT, prefix_lens=AT, q_offsets=AT, own_tables=AT, own_lens=AT, n_tokens=300, n_requests=300, n_groups=3, prefix_width=4096,
             own_width=40, n_pages=5000, page_tokens=16, kv_heads=8, head_dim=128, dtype=0, scale=0.1, reserved=0)
    a.update(change)
    return Attention(*(a[n] for n, _ in Attention._fields_))


@pytest.mark.parametrize("change, rc", [
    (dict(dtype=2), BAD), (dict(dtype=7), BAD), (dict(head_dim=96), BAD), (dict(head_dim=512), BAD), (dict(page_tokens=8), BAD), (dict(page_tokens=24), BAD),
    (dict(page_tokens=512), BAD), (dict(kv_heads=0), BAD), (dict(kv_heads=5), BAD), (dict(q=Heads(AT, 4096, 128, 0)), BAD), (dict(out=Heads(AT, 4096, 128, 16)), BAD),
    (dict(scale=0.0), BAD), (dict(scale=-1.0), BAD), (dict(scale=math.inf), BAD), (dict(scale=math.nan), BAD), (dict(reserved=1), BAD), (dict(n_requests=0), BAD),
    (dict(n_tokens=1 << 24), BAD), (dict(n_tokens=1 << 23, q=Heads(AT, 4096, 128, 512), out=Heads(AT, 4096, 128, 512)), BAD), (dict(n_pages=1 << 31), BAD),
    (dict(own_width=1 << 27), BAD), (dict(prefix_width=1 << 27), BAD), (dict(q=Heads(None, 4096, 128, 32)), NULL), (dict(out=Heads(None, 4096, 128, 32)), NULL),
    (dict(q_offsets=None), NULL), (dict(own_lens=None), NULL), (dict(own_tables=None), NULL), (dict(prefix_tables=None), NULL), (dict(prefix_lens=None), NULL),
    (dict(group_offsets=None), NULL), (dict(k_pages=Pages(None, 1 << 15, 1024, 128)), NULL), (dict(v_pages=Pages(None, 1 << 15, 1024, 128)), NULL),
    (dict(q=Heads(AT + 2, 4096, 128, 32)), BAD), (dict(q=Heads(AT, 4097, 128, 32)), BAD), (dict(out=Heads(AT, 4096, 132, 32)), BAD),
    (dict(k_pages=Pages(AT, 1 << 15, 1028, 128)), BAD), (dict(v_pages=Pages(AT + 8, 1 << 15, 1024, 128)), BAD), (dict(v_pages=Pages(AT, -(1 << 15), 1024, 128)), BAD),
    (dict(k_pages=Pages(AT, 1 << 31, 1024, 128)), BAD), (dict(k_pages=Pages(AT, 1 << 15, 1 << 22, 128)), BAD), (dict(lse=AT + 2), BAD), (dict(own_lens=AT + 1), BAD)])
def test_attention_refusals(lib, change, rc):
    a = attention(**change)
    assert lib.lsm_prefix_attention(C.byref(a), C.c_void_p(AT), C.c_size_t(1 << 40), None) == rc
    assert lib.lsm_prefix_attention_workspace_bytes(C.byref(a)) == 0


def test_attention_workspace(lib):
    a = attention()
    need = lib.lsm_prefix_attention_workspace_bytes(C.byref(a))
    # at least one part of the prefix and one of the own pages: 128 floats, a maximum and a sum for every row
    assert need % (300 * 32 * (128 * 4 + 8)) == 0 and need >= 2 * 300 * 32 * (128 * 4 + 8)
    for ws, size in ((None, need), (AT, need - 1), (AT + 128, need)):
        assert lib.lsm_prefix_attention(C.byref(a), C.c_void_p(ws), C.c_size_t(size), None) == WORKSPACE
    assert lib.lsm_prefix_attention(None, None, C.c_size_t(0), None) == NULL and lib.lsm_prefix_attention_workspace_bytes(None) == 0
    empty = attention(n_tokens=0, n_requests=0, n_groups=0)
    assert lib.lsm_prefix_attention_workspace_bytes(C.byref(empty)) == 0 and lib.lsm_prefix_attention(C.byref(empty), None, C.c_size_t(0), None) == 0
    # a short batch is one pass without parts; never more than 128 parts
    short = attention(n_tokens=2, n_requests=2, n_groups=1, prefix_width=8)
    assert lib.lsm_prefix_attention_workspace_bytes(C.byref(short)) == 0
    long = attention(n_tokens=1, n_requests=1, n_groups=1, own_width=1 << 20, kv_heads=1)
    assert 0 < lib.lsm_prefix_attention_workspace_bytes(C.byref(long)) <= 128 * 32 * (128 * 4 + 8)


def test_host_tensors_are_refused():
    import paper_2511_16138_amd as lsm
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    pages = torch.zeros(3, 16, 4, 64, dtype=torch.bfloat16)
    ints = torch.zeros(2, dtype=torch.int32)
    if torch.cuda.is_available():
        pytest.skip("tested where there is no GPU")
    for call in (lambda: lsm.lsm_rotate_heads(q, None, ints, None), lambda: lsm.lsm_kv_append(q, q, ints, ints.long(), pages, pages, None),
                 lambda: lsm.lsm_prefix_attention(q, pages, pages, lsm.PrefixBatch(ints, ints[None], ints, ints, ints[None], ints))):
        with pytest.raises((ValueError, RuntimeError)):
            call()
    with pytest.raises(ValueError):
        lsm.lsm_rope_table(8, 0)


def test_reference_attention_agrees_with_torch():
    """Pages in order, no prefix, one request: causal attention as torch has it."""
    gen = torch.Generator().manual_seed(1)
    n, heads, kv, d, page = 37, 6, 2, 64, 16
    q, k, v = (torch.randn(n, h, d, generator=gen) for h in (heads, kv, kv))
    pages = torch.zeros(2, 3, page, kv, d)
    pages[0].view(-1, kv, d)[:n], pages[1].view(-1, kv, d)[:n] = k, v
    out, lse, _, _ = ref.attention(q, pages[0], pages[1], [0, 1], torch.zeros(1, 0), [0], [0, n], torch.arange(3)[None], [n])
    want = torch.nn.functional.scaled_dot_product_attention(q.double().transpose(0, 1), k.double().repeat_interleave(3, 1).transpose(0, 1),
                                                            v.double().repeat_interleave(3, 1).transpose(0, 1), is_causal=True).transpose(0, 1)
    assert torch.allclose(out, want, atol=1e-12) and bool(torch.isfinite(lse).all())
    # the same tokens with the first 16 as a shared prefix
    again, lse2, _, _ = ref.attention(q[16:], pages[0], pages[1], [0, 1], torch.zeros(1, 1), [16], [0, n - 16], torch.tensor([[1, 2]]), [n - 16])
    assert torch.allclose(again, want[16:], atol=1e-12) and torch.allclose(lse2, lse[16:], atol=1e-12)


def test_reference_rotation_is_a_rotation():
    gen = torch.Generator().manual_seed(2)
    x = torch.randn(5, 3, 16, generator=gen)
    angle = torch.arange(9.0)[:, None] * 10000.0 ** (-torch.arange(4.0) / 4)
    table = torch.cat([angle.cos(), angle.sin()], 1)
    p = torch.tensor([0, 1, 2, 7, 8], dtype=torch.int32)
    for interleaved in (False, True):
        y, _ = ref.rotate(x, None, table, p, interleaved=interleaved)
        assert torch.allclose(y[0], x[0].double()) and torch.allclose(y.norm(dim=-1), x.double().norm(dim=-1), rtol=1e-6) and torch.equal(y[..., 8:], x[..., 8:].double())
        # scores depend on differences of positions alone
        z = torch.randn(1, 1, 16, generator=gen).double()
        a, b = (ref.rotate(z, None, table, torch.tensor([i], dtype=torch.int32), interleaved=interleaved)[0] for i in (1, 3))
        c, e = (ref.rotate(z, None, table, torch.tensor([i], dtype=torch.int32), interleaved=interleaved)[0] for i in (5, 7))
        assert abs(float((a * b).sum() - (c * e).sum())) < 1e-6
