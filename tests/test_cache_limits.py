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
