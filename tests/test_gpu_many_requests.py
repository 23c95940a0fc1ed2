"""Attention of more requests and groups than a wave looks at at a time, and than it finds one of in two and in three looks, against 64 bits."""
import math

import pytest
import torch

import cache_reference as ref

pytestmark = pytest.mark.gpu

PAGE, D = 16, 64


@pytest.fixture(scope="module")
def lsm():
    import paper_2511_16138_amd as lsm
    return lsm


def attention(q, k, v, sees, scale):
    """(out, bound) of tokens [n, heads, d] over keys and values [n, keys, d] of which a token sees some, [n, keys]; bounds as in cache_reference.attention."""
    out, bound = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    for first in range(0, q.shape[0], 20000):
        part = slice(first, first + 20000)
        x, kh, vh, see = q[part].double(), k[part].double(), v[part].double(), sees[part, None]
        s = torch.where(see, (x[:, :, None] * kh[:, None]).sum(-1) * scale, torch.full((), -math.inf, dtype=torch.float64))
        w = torch.softmax(s, 2).nan_to_num(0.0)
        out[part] = (w[..., None] * vh[:, None]).sum(2)
        size = (w[..., None] * vh[:, None].abs()).sum(2)
        reach = torch.where(see, (x.abs()[:, :, None] * kh.abs()[:, None]).sum(-1), torch.zeros((), dtype=torch.float64)).amax(2)
        off = 2 * ((D + 8) * ref.U32 * reach * scale + 8 * ref.U32 * torch.where(see, s.abs(), torch.zeros((), dtype=torch.float64)).amax(2)) + 2.0 ** -21
        bound[part] = ref.u(q.dtype) * out[part].abs() + size * (ref.u(q.dtype) + 2 * off + 4 * (k.shape[1] + 64) * ref.U32)[..., None]
    return out, bound + torch.finfo(q.dtype).smallest_normal * torch.finfo(q.dtype).eps


@pytest.mark.parametrize("kind", ["16 bits", "8 bits", "window"])
@pytest.mark.parametrize("n, groups, prefix", [
    (65, 1, 0), (4097, 1, 0), (300001, 1, 0),   # requests alone
    (5000, 5000, 20), (4097, 4200, 5),          # a prefix each, and groups without a request
    (40000, 70, 30), (40000, 5000, 30),         # in two stages
])
def test_many_requests(lsm, n, groups, prefix, kind):
    """Requests of no new token, or one to three; prefixes of any length up to `prefix`."""
    gen = torch.Generator().manual_seed(n + groups)
    dtype, heads, own_width, width = torch.bfloat16, 2, 1, -(-prefix // PAGE)
    q_lens = torch.randint(0, 4, (n,), generator=gen)
    own_lens = (q_lens + torch.randint(0, 17, (n,), generator=gen)).clamp(max=PAGE)
    starts = torch.cat([torch.zeros(1, dtype=torch.int64), torch.sort(torch.randint(0, n + 1, (groups - 1,), generator=gen))[0], torch.full((1,), n)])
    group = torch.bucketize(torch.arange(n), starts[1:-1], right=True)
    prefix_lens = torch.randint(0, prefix + 1, (groups,), generator=gen)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), q_lens.cumsum(0)])
    n_pages = 1009
    own_tables, prefix_tables = torch.randint(0, n_pages, (n, own_width), generator=gen), torch.randint(0, n_pages, (groups, width), generator=gen)
    q = torch.randn((int(offsets[-1]), heads, D), generator=gen).to(dtype)
    pages, more = torch.randn((n_pages, 2, PAGE, 1, D), generator=gen), {}
    if kind == "8 bits":
        held = pages.to(torch.float8_e4m3fn).cuda()
        pages = held.cpu().float().to(dtype)
        ones = torch.full((n_pages, 1, 1), 127, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
        more = dict(k_scales=ones, v_scales=ones)
    else:
        pages = pages.to(dtype)
        held = pages.cuda()
    window = 7 if kind == "window" else 1 << 20
    if kind == "window":
        more = dict(window=window, sinks=2)
    ints = lambda t: t.to(torch.int32).cuda()  # noqa: E731
    batch = lsm.PrefixBatch(ints(starts), ints(prefix_tables), ints(prefix_lens), ints(offsets), ints(own_tables), ints(own_lens))
    out = lsm.lsm_prefix_attention(q.cuda(), held[:, 0], held[:, 1], batch, **more).cpu().double()

    request = torch.repeat_interleave(torch.arange(n), q_lens)
    head = prefix_lens[group[request]]
    place = head + own_lens[request] - q_lens[request] + torch.arange(q.shape[0]) - offsets[request]
    i, j = torch.arange(width * PAGE)[None], torch.arange(PAGE)[None]
    at = torch.cat([torch.where(i < head[:, None], i, 1 << 29), torch.where(j < own_lens[request][:, None], head[:, None] + j, 1 << 29)], 1)
    sees = (at <= place[:, None]) & ((at > place[:, None] - window) | (at < 2))
    flat = pages.reshape(n_pages, 2, PAGE, D)
    keys, values = (torch.cat([flat[prefix_tables[group[request]], x].reshape(q.shape[0], width * PAGE, D), flat[own_tables[request], x].reshape(q.shape[0], PAGE, D)], 1) for x in (0, 1))
    want, bound = attention(q, keys, values, sees, D ** -0.5)
    ref.assert_within(out, want, bound, "out")
