"""Norm of keys of any magnitude in the append to 8 bits: products of elements and weights beyond the range of 32 bits are ordinary values once they are divided by
the root of the mean square."""
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


def inputs(gen, kind, n, heads, d, dtype):
    """(keys, weight, eps)"""
    x, w = torch.randn((n, heads, d), generator=gen, dtype=torch.float64), 1 + 0.5 * torch.randn(d, generator=gen, dtype=torch.float64)
    if kind == "largest":   # up to the type's largest number, by weights around 4
        x, w, eps = x * 2.0 ** 125, w * 4, 1e-6
    elif kind == "two":     # one magnitude, one weight: 2 and -2
        x, w, eps = torch.where(x < 0, -1.0, 1.0).double() * 2.0 ** 127, torch.full_like(w, 2.0), 1e-6
    elif kind == "smallest":  # subnormal elements, or next to them, and products below what the type has
        x, w, eps = x * 2.0 ** -126, w * 2.0 ** -15, 0.0
    else:                   # large products and small ones in a row
        size = torch.randint(-60, 61, (d,), generator=gen).double()
        x, w, eps = x * torch.exp2(size + 60), w * torch.exp2(size), 0.0
    most = float(torch.finfo(dtype).max)
    x = x.clamp(-most, most).to(dtype)
    x[..., 0] = torch.where(x[..., 0] == 0, torch.full_like(x[..., 0], float(torch.finfo(dtype).tiny)), x[..., 0])  # no row of zeros, which has no norm without eps
    return x, w.to(dtype), eps


@pytest.mark.parametrize("way", ["pairs apart", "neighbours", "rows at any address", "weights of 32 bits", "weights of 32 bits, neighbours", "no rotation", "elements of 32 bits"])
@pytest.mark.parametrize("kind", ["largest", "two", "smallest", "every size"])
def test_norm_of_any_magnitude(lsm, kind, way):
    gen = torch.Generator().manual_seed(len(kind) * 100 + len(way))
    n, heads, d, dtype = 64, 2, 128, FP32 if "elements" in way else BF16
    x, w, eps = inputs(gen, kind, n, heads, d, BF16)
    x, w = x.to(dtype), w.to(FP32 if "32" in way else dtype)
    table = None if way == "no rotation" else lsm.lsm_rope_table(200, d)
    positions = torch.randint(0, 200, (n,), generator=gen, dtype=torch.int32)
    shift = 1 if way == "rows at any address" else 0
    dev = torch.zeros((n, heads, d + 8), dtype=dtype, device="cuda")[..., shift:shift + d]
    dev.copy_(x)
    codes = torch.zeros((n // 16, 16, heads, d), dtype=torch.uint8, device="cuda").view(pages.E4M3)
    scales = torch.zeros((n // 16, 1, heads), dtype=torch.uint8, device="cuda").view(pages.E8M0)
    v_codes, v_scales = codes.clone(), scales.clone()
    batch = lsm.PrefixBatch(ints([0, 1]), ints([[]]).reshape(1, 0), ints([0]), ints([0, n]), torch.arange(n // 16, dtype=torch.int32).view(1, -1).cuda(), ints([n]))
    lsm.lsm_kv_append8(dev, dev, positions.cuda(), batch, codes, v_codes, scales, v_scales, table, k_weight=w.cuda(), eps=eps, interleaved="neighbours" in way)
    y, bound = nearest.keys(x, w, None if table is None else table.cpu(), positions, eps, "neighbours" in way)
    assert bool(torch.isfinite(y).all())
    assert int(torch.isnan(codes.cpu().float()).sum()) == 0, "finite keys became NaN"
    assert nearest.compare(codes.cpu(), scales.cpu()[:, 0], y, bound, dtype)[:2] == (0, 0)
