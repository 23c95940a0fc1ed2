"""lsm_prefix_attention where a row's keys are dealt to several workgroups: the joins, and the two stages of one launch (a group's prefix, then each
request's own pages).  Which way a batch goes is read off the kernels that a recorded call holds."""
import ctypes
import math
import re

import pytest
import torch

import cache_reference as ref
from test_gpu_cache import BF16, FP16, make_batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsm():
    import paper_2511_16138_amd as lsm
    return lsm


class KernelNode(ctypes.Structure):
    _fields_ = [("block", ctypes.c_uint32 * 3), ("extra", ctypes.c_void_p), ("func", ctypes.c_void_p), ("grid", ctypes.c_uint32 * 3),
                ("params", ctypes.c_void_p), ("shared", ctypes.c_uint32)]


def kernels(call):
    """The names of the kernels that a call launches, from a graph that records it (and is not run)."""
    hip = ctypes.CDLL(next(line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line))
    hip.hipKernelNameRefByPtr.restype = ctypes.c_char_p
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    handle, n = ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t(0)
    assert hip.hipGraphGetNodes(handle, None, ctypes.byref(n)) == 0
    nodes = (ctypes.c_void_p * n.value)()
    assert hip.hipGraphGetNodes(handle, nodes, ctypes.byref(n)) == 0
    names = []
    for node in nodes:
        kind, params = ctypes.c_int(-1), KernelNode()
        assert hip.hipGraphNodeGetType(ctypes.c_void_p(node), ctypes.byref(kind)) == 0 and kind.value == 0  # a kernel
        assert hip.hipGraphKernelNodeGetParams(ctypes.c_void_p(node), ctypes.byref(params)) == 0
        names.append(hip.hipKernelNameRefByPtr(ctypes.c_void_p(params.func), None).decode())
    return names


WAYS = {"both stages": 0, "narrow alone": 1, "wide alone": 2}  # the third argument of attention_kernel


def attend(lsm, q, blocks, parts, way, joined=True):
    """(out, lse) of a batch that has to go a certain way."""
    held, batch, q = blocks.cuda(), lsm.PrefixBatch(*(p.cuda() for p in parts)), q.cuda()
    call = lambda: lsm.lsm_prefix_attention(q, held[:, 0], held[:, 1], batch, with_lse=True)  # noqa: E731
    out, lse = call()
    names = kernels(call)
    d, kind = q.shape[2], 0 if q.dtype == BF16 else 1
    assert re.search(rf"attention_kernelILi{kind}ELi{d}ELi{WAYS[way]}E", names[0]), names
    assert len(names) == (2 if joined else 1) and (not joined or f"join_kernelILi{kind}ELi{d}E" in names[1]), names
    again, _ = call()
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))
    return out, lse


# One key in the last quarter of a row's keys outweighs all others by more than 2^160; what is not finite is among the values of an early key.
# name, way, joined, groups, prefix, own lengths, new tokens, query heads, KV heads, head, spare columns, the request and the key (prefix or own) of the
# value, the strong key (prefix or own)
GAPS = [
    ("one range", "narrow alone", False, [1], [0], [600], [1], 4, 1, 64, 0, ("own", 40), ("own", 590)),
    ("ranges of one request", "narrow alone", True, [1], [0], [4096], [1], 4, 1, 64, 0, ("own", 300), ("own", 4000)),
    ("ranges of one request, the strong one first", "narrow alone", True, [1], [0], [4096], [1], 4, 2, 128, 0, ("own", 3000), ("own", 5)),
    ("ranges of wide tiles", "wide alone", True, [1], [0], [2048], [80], 8, 1, 64, 0, ("own", 200), ("own", 1900)),
    ("a value of the prefix", "both stages", True, [3], [300], [40, 50, 60], [1, 1, 1], 4, 1, 128, 300, ("prefix", 20), ("own", 39)),
    ("a value of the own pages", "both stages", True, [3], [300], [40, 50, 60], [1, 1, 1], 4, 1, 128, 300, ("own", 20), ("prefix", 290)),
]


@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("case", GAPS, ids=[c[0] for c in GAPS])
def test_what_is_not_finite_is_not_lost_in_a_join(lsm, case, value):
    """A seen value that is infinite or NaN decides its column of the row, however small its key's weight is and however keys are dealt out."""
    name, way, joined, groups, prefix, own, q_lens, hq, hkv, d, spare, (segment, at), (strong_segment, strong_at) = case
    gen = torch.Generator().manual_seed(21)
    page = 256 if spare else 16
    q, blocks, parts = make_batch(gen, groups, prefix, q_lens, own, hq, hkv, d, page, BF16, spare=spare)
    q[:] = 1.0
    blocks[:, 0] *= 0.05

    def place(segment, i):
        return int(parts[1 if segment == "prefix" else 4][0, i // page]), i % page

    p, row = place(strong_segment, strong_at)
    blocks[p, 0, row] = 16.0  # score 16 d / sqrt(d) against about 0.05: 128 and more apart, 184 as an exponent of two
    p, row = place(segment, at)
    blocks[p, 1, row, :, 9] = value
    out, lse = attend(lsm, q, blocks, parts, way, joined)
    want, want_lse, bound, lse_bound = ref.attention(q, blocks[:, 0], blocks[:, 1], *parts)
    first = out[:q_lens[0]].cpu()
    assert not bool(torch.isfinite(first[..., 9]).any()), "a value that is not finite is lost"
    keep = [c for c in range(d) if c != 9]
    ref.assert_within(out[..., keep], want[..., keep], bound[..., keep], "the other columns")
    ref.assert_within(lse, want_lse, lse_bound, "lse")


# Both stages in one launch, with tiles of either kind in each: a stage's tiles are wide where its owners (groups, requests) have more than 48 rows
# on average, a row being a query head of a KV head's share.  (There are fewer groups than requests, so the first stage is never the narrower one.)  Spare columns make the tables long, which is what the choice of two stages goes by.
STAGES = [
    # groups, prefix, q_lens, own_lens, hq, hkv, d, page, dtype, spare
    ("narrow, narrow", [3, 2, 4], [100, 65, 300], [1] * 9, [1, 17, 40, 64, 65, 3, 130, 2, 33], 8, 2, 128, 64, BF16, 400),
    ("narrow, narrow, fp16", [3, 2, 4], [100, 65, 300], [1] * 9, [1, 17, 40, 64, 65, 3, 130, 2, 33], 8, 2, 64, 64, FP16, 800),
    ("narrow, narrow, 8 KV heads", [4, 1, 3], [70, 16, 129], [1] * 8, [5, 1, 90, 16, 300, 31, 33, 2], 32, 8, 128, 64, BF16, 200),
    ("narrow, narrow, heads of 256", [3, 3], [90, 200], [1] * 6, [40, 1, 33, 70, 2, 16], 8, 2, 256, 64, FP16, 300),
    ("narrow, narrow, few new tokens", [3, 2], [31, 197], [3, 1, 2, 2, 3], [3, 50, 80, 2, 65], 8, 2, 128, 64, FP16, 800),
    ("narrow, narrow, no prefix in some", [3, 2, 2], [0, 65, 0], [1] * 7, [1, 17, 40, 64, 65, 3, 130], 8, 2, 128, 64, BF16, 500),
    ("wide, narrow", [20, 9], [700, 130], [1] * 29, [1 + 5 * i % 70 for i in range(29)], 16, 2, 128, 64, BF16, 200),
    ("wide, narrow, fp16", [9, 20], [130, 400], [1] * 29, [1 + 5 * i % 70 for i in range(29)], 16, 2, 64, 64, FP16, 400),
    ("wide, narrow, 8 KV heads", [15], [400], [1] * 15, [1 + 5 * i % 70 for i in range(15)], 32, 8, 64, 64, BF16, 200),
    ("wide, narrow, heads of 256", [12, 8], [300, 90], [1] * 20, [1 + 7 * i % 50 for i in range(20)], 16, 2, 256, 64, BF16, 200),
    ("wide, narrow, few new tokens", [10, 6], [300, 33], [1 + i % 4 for i in range(16)], [4 + 9 * i % 60 for i in range(16)], 16, 2, 128, 64, FP16, 300),
    ("wide, wide", [3, 2], [300, 77], [20, 33, 1, 40, 17], [60, 33, 90, 40, 64], 8, 2, 128, 64, BF16, 800),
    ("wide, wide, fp16", [2, 2], [130, 500], [30, 14, 25, 60], [30, 100, 25, 61], 8, 2, 64, 64, FP16, 1600),
    ("wide, wide, heads of 256", [4], [150], [20, 3, 40, 30], [20, 50, 70, 33], 8, 2, 256, 64, FP16, 300),
    ("wide, wide, 8 KV heads", [3], [200], [20, 33, 12], [60, 33, 12], 32, 8, 64, 64, BF16, 600),
    ("empty groups and requests without tokens", [0, 3, 0, 2, 2, 0], [64, 100, 0, 33, 200, 1], [1, 0, 2, 1, 1, 0, 1], [9, 30, 2, 1, 100, 0, 64], 8, 2, 128, 64, BF16, 500),
    ("nothing of its own", [3, 2], [200, 70], [1, 1, 1, 2, 1], [0, 1, 0, 1, 0], 8, 2, 128, 64, BF16, 800),
    ("every head its own", [10, 5], [65, 100], [1] * 15, [1 + 3 * i for i in range(15)], 4, 4, 64, 64, BF16, 600),
    ("a share of seven", [6, 5], [150, 50], [1] * 11, [1 + 13 * i for i in range(11)], 28, 4, 128, 64, FP16, 200),
    ("more than 64 groups", [2] * 70, [10 + i for i in range(70)], [1] * 140, [1 + i % 20 for i in range(140)], 4, 1, 64, 16, BF16, 160),
]


def kinds(groups, q_lens, hq, hkv):
    """Which stages have wide tiles, by the rule."""
    rows = sum(q_lens) * (hq // hkv)
    return ["wide" if rows // len(owners) > 48 else "narrow" for owners in (groups, q_lens)]


@pytest.mark.parametrize("case", STAGES, ids=[c[0] for c in STAGES])
def test_two_stages(lsm, case):
    name, groups, prefix, q_lens, own, hq, hkv, d, page, dtype, spare = case
    if name.startswith(("wide", "narrow")):
        assert kinds(groups, q_lens, hq, hkv) == name.split(", ")[:2]
    gen = torch.Generator().manual_seed(len(name) * 100 + d)
    q, blocks, parts = make_batch(gen, groups, prefix, q_lens, own, hq, hkv, d, page, dtype, spare=spare)
    out, lse = attend(lsm, q, blocks, parts, "both stages")
    want, want_lse, bound, lse_bound = ref.attention(q, blocks[:, 0], blocks[:, 1], *parts)
    ref.assert_within(out, want, bound, "out")
    ref.assert_within(lse, want_lse, lse_bound, "lse")


@pytest.mark.parametrize("garbage", [math.nan, math.inf])
@pytest.mark.parametrize("i", [0, 1, 6, 9, 11, 15])
def test_two_stages_never_use_what_no_length_reaches(lsm, i, garbage):
    name, groups, prefix, q_lens, own, hq, hkv, d, page, dtype, spare = STAGES[i]
    gen = torch.Generator().manual_seed(23 + i)
    q, blocks, parts = make_batch(gen, groups, prefix, q_lens, own, hq, hkv, d, page, dtype, spare=spare, garbage=garbage)
    out, lse = attend(lsm, q, blocks, parts, "both stages")
    want, want_lse, bound, lse_bound = ref.attention(q, blocks[:, 0], blocks[:, 1], *parts)
    ref.assert_within(out, want, bound, "out")
    ref.assert_within(lse, want_lse, lse_bound, "lse")


@pytest.mark.parametrize("i", [0, 2, 6, 9, 11, 13])
def test_two_stages_with_holes(lsm, i):
    name, groups, prefix, q_lens, own, hq, hkv, d, page, dtype, spare = STAGES[i]
    gen = torch.Generator().manual_seed(24 + i)
    q, blocks, parts = make_batch(gen, groups, prefix, q_lens, own, hq, hkv, d, page, dtype, spare=spare, holes=2)
    out, lse = attend(lsm, q, blocks, parts, "both stages")
    want, want_lse, bound, lse_bound = ref.attention(q, blocks[:, 0], blocks[:, 1], *parts)
    ref.assert_within(out, want, bound, "out")
    ref.assert_within(lse, want_lse, lse_bound, "lse")


@pytest.mark.parametrize("i", [4, 10, 11, 13])
def test_two_stages_keep_what_is_not_finite_from_tokens_before_it(lsm, i):
    """NaN in the value of a request's last token: it reaches that token alone."""
    name, groups, prefix, q_lens, own, hq, hkv, d, page, dtype, spare = STAGES[i]
    gen = torch.Generator().manual_seed(25 + i)
    q, blocks, parts = make_batch(gen, groups, prefix, q_lens, own, hq, hkv, d, page, dtype, spare=spare)
    for r, length in enumerate(own):
        blocks[int(parts[4][r, (length - 1) // page]), 1, (length - 1) % page, r % hkv, (5 * r) % d] = math.nan
    out, lse = attend(lsm, q, blocks, parts, "both stages")
    want, want_lse, bound, lse_bound = ref.attention(q, blocks[:, 0], blocks[:, 1], *parts)
    ref.assert_within(out, want, bound, "out")
    ref.assert_within(lse, want_lse, lse_bound, "lse")
    finite = torch.isfinite(out.cpu()).all(-1).all(-1)
    ends = [sum(q_lens[:r + 1]) - 1 for r in range(len(q_lens))]
    assert (~finite).nonzero().flatten().tolist() == ends


@pytest.mark.parametrize("way, groups, q_lens, hq, hkv, joined", [
    ("narrow alone", [1] * 130, [1] * 130, 4, 1, False), ("narrow alone", [1, 0, 2] * 50, [1 + i % 3 for i in range(150)], 8, 2, False),
    ("wide alone", [1] * 70, [20 + i % 9 for i in range(70)], 4, 1, False), ("narrow alone", [0] * 64 + [2] + [0] * 70 + [1], [1, 2, 1], 4, 1, False)])
def test_one_pass_over_more_than_64_groups(lsm, way, groups, q_lens, hq, hkv, joined):
    """Every request finds its group, however many there are and however many of them are empty."""
    gen = torch.Generator().manual_seed(31)
    n = len(q_lens)
    prefix = [(7 * i) % 90 for i in range(len(groups))]
    q, blocks, parts = make_batch(gen, groups, prefix, q_lens, [m + i % 30 for i, m in enumerate(q_lens)], hq, hkv, 64, 16, BF16)
    assert int(parts[0][-1]) == n
    out, lse = attend(lsm, q, blocks, parts, way, joined)
    want, want_lse, bound, lse_bound = ref.attention(q, blocks[:, 0], blocks[:, 1], *parts)
    ref.assert_within(out, want, bound, "out")
    ref.assert_within(lse, want_lse, lse_bound, "lse")
