"""CPU-only checks of the paged-cache calls at the ends of their ranges: what cannot be computed or launched is refused before anything is."""
import ctypes as C
import math

import pytest

import test_cache_host
from test_cache_host import AT, BAD, attention

lib = test_cache_host.lib


def attend(lib, a):
    need = lib.lsm_prefix_attention_workspace_bytes(C.byref(a))
    return need, lib.lsm_prefix_attention(C.byref(a), C.c_void_p(AT), C.c_size_t(1 << 62), None)


@pytest.mark.parametrize("scale", [3.0e38, 2.4e38, 2.36e38])
def test_a_scale_that_is_infinite_for_exponents_of_two_is_refused(lib, scale):
    """The kernels multiply scores by scale log2(e): beyond 3.4e38 / 1.4427 that is infinite, and a score of 0 becomes NaN."""
    assert attend(lib, attention(scale=scale)) == (0, BAD)


def test_an_infinite_base_of_angles_is_refused(lib):
    """Its logarithm times 0, the exponent of the first pair, is no number."""
    assert lib.lsm_rope_table(AT, 8, 64, math.inf, None) == BAD


@pytest.mark.parametrize("change", [
    # HIP takes launches of fewer than 2^32 threads, 256 a workgroup here
    dict(n_tokens=3 << 20, n_requests=3 << 20, n_groups=0, own_width=1),                                      # 3M decodes, 8 KV heads: 25M workgroups
    dict(n_tokens=3 << 20, n_requests=3 << 20, n_groups=1, own_width=1, prefix_width=1 << 20),                # behind a prefix
    dict(n_tokens=1 << 22, n_requests=1 << 20, n_groups=1, own_width=4, prefix_width=1 << 12, kv_heads=1, q=test_cache_host.Heads(AT, 8192, 128, 64),
         out=test_cache_host.Heads(AT, 8192, 128, 64)),                                                       # 5M workgroups, but 32M join their parts
])
def test_batches_of_more_workgroups_than_a_launch_takes_are_refused(lib, change):
    assert attend(lib, attention(**change)) == (0, BAD)


def test_the_largest_batches_have_a_workspace(lib):
    """A million decodes of 8 KV heads behind a prefix: 10M workgroups, and 4M that join their parts."""
    a = attention(n_tokens=(1 << 20), n_requests=(1 << 20), n_groups=1, own_width=1, prefix_width=1 << 20)
    assert lib.lsm_prefix_attention_workspace_bytes(C.byref(a)) > 0
