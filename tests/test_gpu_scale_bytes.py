"""The first and the last byte that a scale may be, in attention over pages of 8 bits."""
import pytest
import torch

import cache_reference as ref
import pages_reference as pages
from test_gpu_cache import make_batch
from test_gpu_window import BF16, FP16, to_8_bits, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsm():
    import paper_2511_16138_amd as lsm
    return lsm


def compare(lsm, q, codes, parts, scales, held, scale=None, **more):
    """held: what the pages hold.  In fp16 the weights of the softmax that are below 2^-14 of the largest are rounded to multiples of 2^-24, each off by 2^-25 at most, and
    their sum is 1 at least: a result is off by 2^-25 of the values' magnitudes more than the reference's bound, which counts 2^-11 of each weight."""
    want, want_lse, bound, lse_bound = pages.attention(q, held[:, 0], held[:, 1], *parts, scale=scale, **more)
    if q.dtype == FP16:
        most = int((parts[2].max() + parts[5].max()))  # keys of a row
        bound = bound + most * 2.0 ** -25 * float(held[:, 1].double().abs().nan_to_num(0.0).max())
    dev, s = codes.cuda(), scales.cuda()
    out, lse = lsm.lsm_prefix_attention(q.cuda(), dev[:, 0], dev[:, 1], lsm.PrefixBatch(*(p.cuda() for p in parts)), scale=scale, with_lse=True, k_scales=s[:, 0], v_scales=s[:, 1], **more)
    ref.assert_within(out, want, bound, "out")
    ref.assert_within(lse, want_lse, lse_bound, "lse")
    return out


@pytest.mark.parametrize("window", [0, 40])
@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("q_lens, hq", [([1, 2], 4), ([40, 30], 8)])  # narrow tiles, wide ones
def test_byte_255_on_the_keys_side(lsm, q_lens, hq, dtype, window):
    """A block's keys are NaN for one head: rows that see one of them have no result, others are as they were."""
    gen = torch.Generator().manual_seed(hq)
    q, blocks, parts = make_batch(gen, [1, 1], [64, 32], q_lens, [64, 70], hq, 2, 64, 16, dtype)
    codes, scales = to_8_bits(gen, blocks)
    sinks = dict(window=window, sinks=5) if window else {}
    before = compare(lsm, q, codes, parts, scales, values(codes, scales, dtype), **sinks)
    scales.view(torch.uint8)[int(parts[1][0, 1]), 0, 0, 1] = 255   # tokens 16 to 31 of the first request's prefix, the second head's keys
    held = values(codes, scales, dtype)
    assert torch.isnan(held[int(parts[1][0, 1]), 0, :, 1]).all() and int(torch.isnan(held).sum()) == 16 * 64
    after = compare(lsm, q, codes, parts, scales, held, **sinks)
    n, share = q_lens[0], hq // 2
    assert bool(torch.isnan(after[:n, share:]).all()) == (window == 0)
    assert torch.equal(before[n:].view(torch.int16), after[n:].view(torch.int16)) and torch.equal(before[:, :share].view(torch.int16), after[:, :share].view(torch.int16))


@pytest.mark.parametrize("byte", [0, 1, 2])
@pytest.mark.parametrize("q_lens, hq", [([1, 2], 4), ([40, 30], 8)])
def test_the_smallest_scales(lsm, byte, q_lens, hq):
    """Bytes 0, 1, 2: exponents -127, -126, -125, not 0.  Codes of 64 and more are ordinary numbers of bfloat16 then, and too small for float16."""
    gen = torch.Generator().manual_seed(hq + byte)
    q, blocks, parts = make_batch(gen, [1, 1], [64, 32], q_lens, [64, 70], hq, 2, 64, 16, BF16)
    codes, scales = to_8_bits(gen, blocks)
    codes.view(torch.uint8)[:] = codes.view(torch.uint8) & 0x80 | torch.randint(0x68, 0x7F, codes.shape, generator=gen, dtype=torch.uint8)  # 64 to 448
    scales.view(torch.uint8)[:, 1] = byte
    held = values(codes, scales, BF16)
    assert float(held[:, 1].float().abs().min()) >= 64 * 2.0 ** (byte - 127) and float(held[:, 1].float().abs().max()) <= 448 * 2.0 ** (byte - 127)
    out = compare(lsm, q, codes, parts, scales, held, scale=1e-4)  # all weights alike
    assert float(out.abs().max()) > 2.0 ** (byte - 127 + 4)
    compare(lsm, q.to(FP16), codes, parts, scales, values(codes, scales, FP16), scale=1e-4)
    scales.view(torch.uint8)[:, 0] = byte  # keys: every score is 0, next to
    compare(lsm, q, codes, parts, scales, values(codes, scales, BF16))
