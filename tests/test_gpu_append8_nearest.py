"""Codes of normed and rotated keys are the nearest ones to the formula's values (tests/nearest_codes.py): four million of each way through the kernels, of
which computation in 32 bits gets several wrong (tests/test_nearest_codes.py), and values next to a border."""
import pytest
import torch

import nearest_codes as nearest
import pages_reference as pages

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def lsm():
    import paper_2511_16138_amd as lsm
    return lsm


def ints(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


def append(lsm, x, weight, table, positions, eps, interleaved, aligned=True):
    """Appends x [n, heads, d] as keys and values of one request to pages of 16, in order: codes and scales of the keys."""
    n, heads, d = x.shape
    shift = 0 if aligned else 1
    dev = torch.zeros((n, heads, d + 8), dtype=x.dtype, device="cuda")[..., shift:shift + d]
    dev.copy_(x)
    codes = torch.zeros((n // 16, 16, heads, d), dtype=torch.uint8, device="cuda").view(pages.E4M3)
    scales = torch.zeros((n // 16, 1, heads), dtype=torch.uint8, device="cuda").view(pages.E8M0)
    v_codes, v_scales = codes.clone(), scales.clone()
    batch = lsm.PrefixBatch(ints([0, 1]), ints([[]]).reshape(1, 0), ints([0]), ints([0, n]), torch.arange(n // 16, dtype=torch.int32).view(1, -1).cuda(), ints([n]))
    lsm.lsm_kv_append8(dev, dev, positions.cuda(), batch, codes, v_codes, scales, v_scales, table.cuda(), k_weight=None if weight is None else weight.cuda(), eps=eps, interleaved=interleaved)
    return codes.cpu(), scales.cpu()[:, 0]


WAYS = [
    # dtype, weight's, d, rot, interleaved, aligned
    (BF16, BF16, 128, 128, False, True),
    (BF16, BF16, 128, 128, True, True),
    (FP16, FP16, 128, 64, False, True),
    (FP16, FP16, 64, 64, True, True),
    (BF16, BF16, 256, 128, False, True),
    (BF16, BF16, 128, 128, False, False),    # rows at any address
    (FP16, FP16, 80, 40, False, True),       # half of the rotated part is no whole number of lanes
    (BF16, FP32, 128, 128, True, False),
    (BF16, FP32, 128, 128, False, True),     # weights of 32 bits
    (FP16, FP32, 128, 128, True, True),
    (FP32, FP32, 128, 128, False, True),
    (FP32, FP32, 64, 32, True, True),
    (BF16, None, 128, 128, False, True),
    (FP16, None, 128, 128, True, True),
    (FP32, None, 256, 256, False, True),
]


@pytest.mark.parametrize("way", WAYS, ids=lambda w: "-".join(str(v).replace("torch.", "") for v in w))
def test_codes_are_the_nearest(lsm, way):
    dtype, weight_dtype, d, rot, interleaved, aligned = way
    gen = torch.Generator().manual_seed(d * 1000 + rot + interleaved)
    heads = 4
    n = (1 << 22) // (heads * d) // 16 * 16
    x = torch.randn((n, heads, d), generator=gen).to(dtype)
    weight = None if weight_dtype is None else (1 + 0.2 * torch.randn(d, generator=gen)).to(weight_dtype)
    table, positions = lsm.lsm_rope_table(4096, rot).cpu(), torch.randint(0, 4096, (n,), generator=gen, dtype=torch.int32)
    codes, scales = append(lsm, x, weight, table, positions, 1e-6, interleaved, aligned)
    y, bound = nearest.keys(x, weight, table, positions, 1e-6, interleaved)
    wrong_scales, wrong_codes, either = nearest.compare(codes, scales, y, bound, dtype)
    assert (wrong_scales, wrong_codes) == (0, 0) and either <= 1


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
@pytest.mark.parametrize("aligned", [True, False])
def test_values_next_to_a_border_are_rounded_once(lsm, dtype, aligned):
    x, table = nearest.next_to_borders()
    assert torch.equal(x.to(dtype).double(), x)
    positions = torch.arange(64, dtype=torch.int32) // 32
    codes, scales = append(lsm, x.to(dtype), None, table, positions, 0.0, False, aligned)
    y, bound = nearest.keys(x, None, table, positions, 0.0)
    assert nearest.compare(codes, scales, y, bound, dtype) == (0, 0, 0)
