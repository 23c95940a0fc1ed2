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
