"""Append to pages of 8 bits by more requests than a wave looks at at a time, and than it finds one of in two and in three looks."""
import pytest
import torch

import pages_reference as pages
from nearest_codes import scales_for

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lsm():
    import paper_2511_16138_amd as lsm
    return lsm


@pytest.mark.parametrize("n", [64, 65, 4096, 4097, 262144, 300001])
@pytest.mark.parametrize("most", [1, 3])
def test_many_requests(lsm, n, most):
    """Requests of no token to a few, each in a block of its own that may hold older ones; values as they are, so that codes are known exactly."""
    gen = torch.Generator().manual_seed(n + most)
    d, dtype = 8, torch.bfloat16
    q_lens = torch.randint(0, most + 1, (n,), generator=gen)
    q_lens[torch.randint(0, n, (8,), generator=gen)] = 16
    own_lens = (q_lens + torch.randint(0, 17, (n,), generator=gen)).clamp(max=16)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), q_lens.cumsum(0)])
    x = (torch.randn((int(offsets[-1]), 2, d), generator=gen) * 4).to(dtype)
    page_of = torch.randperm(n, generator=gen)
    codes = (torch.randint(0, 127, (n, 16, 2, d), generator=gen, dtype=torch.uint8) | torch.randint(0, 2, (n, 16, 2, d), generator=gen, dtype=torch.uint8) << 7).view(pages.E4M3)
    scales = torch.randint(114, 124, (n, 1, 2), generator=gen, dtype=torch.uint8).view(pages.E8M0)  # (keys and values side by side: the second head is the values')
    c, s, dev = codes.cuda(), scales.cuda(), x.cuda()
    ints = lambda t: t.to(torch.int32).cuda()  # noqa: E731
    batch = lsm.PrefixBatch(ints(torch.tensor([0, n])), ints(torch.zeros(1, 0)), ints(torch.zeros(1)), ints(offsets), ints(page_of[:, None]), ints(own_lens))
    lsm.lsm_kv_append8(dev[:, :1], dev[:, 1:], None, batch, c[:, :, :1], c[:, :, 1:], s[:, :, :1], s[:, :, 1:], None)

    row = torch.arange(16)[None]
    new = (row >= (own_lens - q_lens)[:, None]) & (row < own_lens[:, None])            # [n, 16], by request
    token = (offsets[:-1, None] + row - (own_lens - q_lens)[:, None]).clamp(0, max(0, x.shape[0] - 1))
    values = torch.where(new[..., None, None], x[token].double(), torch.zeros((), dtype=torch.float64))
    old, old_e = codes[page_of].float().double(), pages.exponents(scales[page_of])[:, 0]
    e = scales_for(values.abs().amax((1, 3)))
    goes_on = ((own_lens > q_lens) & (q_lens > 0))[:, None]
    e = torch.where(goes_on, torch.maximum(e, old_e), e)
    want_e = torch.where((q_lens > 0)[:, None], e, old_e)
    shift = pages.two_to(old_e - e)[:, None, :, None]
    kept = torch.where((goes_on & (e != old_e))[:, None, :, None] & (row < (own_lens - q_lens)[:, None])[..., None, None], pages.codes_of(old * shift), old)
    want = torch.where(new[..., None, None], pages.codes_of((values * pages.two_to(-e)[:, None, :, None]).clamp(-448, 448)), kept)
    got, got_e = c.cpu()[page_of].float().double(), pages.exponents(s.cpu()[page_of])[:, 0]
    assert torch.equal(got_e, want_e)
    assert torch.equal(got, want)
