"""Refusals of the calls of include/lsm_pages.h on GPU tensors, errors of the library, and version counters."""
import pytest
import torch

import pages_reference as pages

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32
E4M3, E8M0 = pages.E4M3, pages.E8M0


@pytest.fixture(scope="module")
def lsm():
    import paper_2511_16138_amd as lsm
    return lsm


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def zeros(*shape, dtype=BF16):
    return torch.zeros(shape, device="cuda").to(dtype)


def scale_bytes(*shape):
    return torch.full(shape, 127, dtype=torch.uint8, device="cuda").view(E8M0)


def tensors(**change):
    t = dict(q=zeros(2, 4, 64), k=zeros(2, 2, 64), v=zeros(2, 2, 64), k_pages=zeros(3, 32, 2, 64, dtype=E4M3), v_pages=zeros(3, 32, 2, 64, dtype=E4M3), k_scales=scale_bytes(3, 2, 2),
             v_scales=scale_bytes(3, 2, 2), positions=ints([0, 0]), table=zeros(8, 64, dtype=FP32), w=None, out=None, q_offsets=ints([0, 1, 2]), own_tables=ints([[1], [2]]), own_lens=ints([1, 1]),
             window=0, sinks=0, lse=False)
    assert set(change) <= set(t)
    t.update(change)
    return t


def batch(lsm, t):
    return lsm.PrefixBatch(ints([0, 2]), ints([[0]]), ints([16]), t["q_offsets"], t["own_tables"], t["own_lens"])


def append(lsm, **change):
    t = tensors(**change)
    return lsm.lsm_kv_append8(t["k"], t["v"], t["positions"], batch(lsm, t), t["k_pages"], t["v_pages"], t["k_scales"], t["v_scales"], t["table"], k_weight=t["w"], q=t["q"], q_out=t["out"])


def attend(lsm, **change):
    t = tensors(**change)
    return lsm.lsm_prefix_attention(t["q"], t["k_pages"], t["v_pages"], batch(lsm, t), k_scales=t["k_scales"], v_scales=t["v_scales"], window=t["window"], sinks=t["sinks"], out=t["out"])


def test_what_they_take(lsm):
    assert append(lsm).shape == (2, 4, 64)
    assert attend(lsm).shape == (2, 4, 64) and attend(lsm, window=3, sinks=1).shape == (2, 4, 64)
    held = dict(k_pages=zeros(3, 32, 2, 64), v_pages=zeros(3, 32, 2, 64), k_scales=None, v_scales=None)
    assert attend(lsm, window=3, **held).shape == (2, 4, 64)


@pytest.mark.parametrize("change, match", [
    (lambda: dict(k=zeros(2, 2, 64, dtype=torch.float64)), "heads must be"), (lambda: dict(v=zeros(2, 2, 64, dtype=FP16)), "v must be"), (lambda: dict(v=zeros(2, 1, 64)), "v have as many heads"),
    (lambda: dict(k=zeros(2, 2, 128)[..., ::2]), "contiguous"), (lambda: dict(q=zeros(3, 4, 64)), "q must be"), (lambda: dict(out=zeros(2, 4, 64, dtype=FP16)), "q_out must be"),
    (lambda: dict(k_pages=zeros(3, 32, 2, 64)), "k_pages must be Float8_e4m3fn"), (lambda: dict(v_pages=zeros(3, 32, 2, 64, dtype=torch.float8_e5m2)), "v_pages must be Float8_e4m3fn"),
    (lambda: dict(v_pages=zeros(4, 32, 2, 64, dtype=E4M3)), "v_pages must be"), (lambda: dict(k_pages=zeros(3, 32, 1, 64, dtype=E4M3)), "must be"),
    (lambda: dict(k_pages=zeros(3, 24, 2, 64, dtype=E4M3), v_pages=zeros(3, 24, 2, 64, dtype=E4M3)), "k_scales must be"),
    (lambda: dict(k_scales=zeros(3, 2, 2, dtype=FP32)), "k_scales must be Float8_e8m0fnu"), (lambda: dict(v_scales=scale_bytes(3, 1, 2)), "v_scales must be"), (lambda: dict(k_scales=None), "must be a tensor"),
    (lambda: dict(q_offsets=ints([0, 2])), "q_offsets must be"), (lambda: dict(own_lens=ints([1, 1]).long()), "own_lens must be"), (lambda: dict(own_tables=ints([1, 2])), "own_tables must be"),
    (lambda: dict(own_tables=ints([[1, 2], [2, 0]])[:, ::2]), "contiguous"), (lambda: dict(positions=None), "needs positions"), (lambda: dict(positions=ints([0])), "positions must be"),
    (lambda: dict(w=zeros(64, dtype=FP16)), "weight"), (lambda: dict(k=zeros(2, 2, 64).cpu()), "GPU tensor"), (lambda: dict(k_scales=scale_bytes(3, 2, 2).cpu()), "GPU tensor")])
def test_append8_refuses(lsm, change, match):
    with pytest.raises(ValueError, match=match):
        append(lsm, **change())


@pytest.mark.parametrize("change, match", [
    (lambda: dict(k_scales=None), "need k_scales and v_scales"), (lambda: dict(v_scales=None), "need k_scales and v_scales"), (lambda: dict(k_scales=None, v_scales=None, window=4), "need k_scales and v_scales"),
    (lambda: dict(k_pages=zeros(3, 32, 2, 64)), "k_pages must be Float8_e4m3fn"), (lambda: dict(v_pages=zeros(3, 32, 2, 64)), "v_pages must be Float8_e4m3fn"),
    (lambda: dict(q=zeros(2, 4, 64, dtype=FP32)), "q must be"), (lambda: dict(sinks=4), "sinks need a window"), (lambda: dict(window=-1), "negative"), (lambda: dict(window=2, sinks=-3), "negative"),
    (lambda: dict(k_scales=scale_bytes(3, 2, 1)), "k_scales must be"), (lambda: dict(v_scales=zeros(3, 2, 2, dtype=E4M3)), "Float8_e8m0fnu"), (lambda: dict(out=zeros(2, 4, 32)), "out must be"),
    (lambda: dict(v_scales=scale_bytes(3, 2, 2).cpu()), "GPU tensor")])
def test_attention_refuses(lsm, change, match):
    with pytest.raises(ValueError, match=match):
        attend(lsm, **change())


def test_a_window_that_is_no_number(lsm):
    for bad in (1.5, "4", None):
        with pytest.raises((ValueError, TypeError)):
            attend(lsm, window=bad)


def test_errors_of_the_library(lsm):
    with pytest.raises(lsm.LsmError, match="lsm_window_attention"):
        attend(lsm, window=1 << 30)
    with pytest.raises(lsm.LsmError, match="lsm_window_attention"):  # rows at odd places
        flat = zeros(3 * 32 * 2 * 64 + 8, dtype=E4M3)[8:].view(3, 32, 2, 64)
        attend(lsm, k_pages=flat)
    with pytest.raises(lsm.LsmError, match="lsm_kv_append8"):        # heads of 12
        t = dict(q=zeros(2, 4, 12), k=zeros(2, 2, 12), v=zeros(2, 2, 12), k_pages=zeros(3, 32, 2, 12, dtype=E4M3), v_pages=zeros(3, 32, 2, 12, dtype=E4M3), table=None)
        append(lsm, **t)
    with pytest.raises(lsm.LsmError, match="lsm_compact_pages"):
        lsm.lsm_compact_pages([], [ints([[0]])], [ints([1])], 0, n_pages=4)
    with pytest.raises(lsm.LsmError, match="lsm_copy_pages"):
        lsm.lsm_copy_pages([zeros(4, 64)] * 1025, ints([0]), ints([1]))


@pytest.mark.parametrize("call, match", [
    (lambda lsm: lsm.lsm_copy_pages(zeros(4, 64), ints([0]).long(), ints([1])), "sources must be"), (lambda lsm: lsm.lsm_copy_pages(zeros(4, 64), ints([0]), ints([1, 2])), "targets must be"),
    (lambda lsm: lsm.lsm_copy_pages(zeros(4, 64), ints([[0]]), ints([1])), "sources must be"), (lambda lsm: lsm.lsm_copy_pages(zeros(4, 64), ints([0, 1, 2])[::2], ints([1, 3])), "contiguous"),
    (lambda lsm: lsm.lsm_copy_pages([zeros(4, 64), zeros(5, 64)], ints([0]), ints([1])), "as many pages"), (lambda lsm: lsm.lsm_copy_pages(zeros(4, 64).cpu(), ints([0]), ints([1])), "GPU tensor"),
    (lambda lsm: lsm.lsm_copy_pages(zeros(4, 8, 64)[:, ::2], ints([0]), ints([1])), "one stretch"), (lambda lsm: lsm.lsm_copy_pages(zeros(4, 64)[:, ::2], ints([0]), ints([1])), "one stretch"),
    (lambda lsm: lsm.lsm_copy_pages(zeros(4, 1).expand(4, 64), ints([0]), ints([1])), "one stretch"), (lambda lsm: lsm.lsm_copy_pages(zeros(1, 64).expand(4, 64), ints([0]), ints([1])), "overlap"),
    (lambda lsm: lsm.lsm_copy_pages(zeros(256).as_strided((4, 64), (32, 1)), ints([0]), ints([1])), "overlap"), (lambda lsm: lsm.lsm_copy_pages(zeros(1)[0], ints([0]), ints([1])), "must be"),
    (lambda lsm: lsm.lsm_copy_pages(zeros(4, 64).requires_grad_(), ints([0]), ints([1])), "gradients"),
    (lambda lsm: lsm.lsm_compact_pages(zeros(4, 64).requires_grad_(), ints([[0]]), ints([1]), 16), "gradients"),
    (lambda lsm: lsm.lsm_compact_pages([], ints([[0]]), ints([1]), 16), "n_pages must be given"), (lambda lsm: lsm.lsm_compact_pages(zeros(4, 64), ints([[0]]), ints([1]), 16, n_pages=5), "n_pages is not"),
    (lambda lsm: lsm.lsm_compact_pages([], ints([[0]]), ints([1]), 16, n_pages=1 << 30), "2.30"), (lambda lsm: lsm.lsm_compact_pages([], ints([[0]]), ints([1]), 16, n_pages=-1), "negative"),
    (lambda lsm: lsm.lsm_compact_pages([], ints([0]), ints([1]), 16, n_pages=4), "rows, width"), (lambda lsm: lsm.lsm_compact_pages([], ints([[0]]), ints([1, 2]), 16, n_pages=4), "lens of a table"),
    (lambda lsm: lsm.lsm_compact_pages([], ints([[0]]).long(), ints([1]), 16, n_pages=4), "a table must be"), (lambda lsm: lsm.lsm_compact_pages([], ints([[0]]), ints([1]), -16, n_pages=4), "negative")])
def test_moves_refuse(lsm, call, match):
    with pytest.raises(ValueError, match=match):
        call(lsm)


def test_written_tensors_bump_their_versions(lsm):
    t = tensors(out=zeros(2, 4, 64))
    watched = ["k_pages", "v_pages", "k_scales", "v_scales", "out"]
    before = {n: t[n]._version for n in watched}
    append(lsm, **t)
    assert all(t[n]._version > before[n] for n in watched)
    before = {n: t[n]._version for n in watched}
    attend(lsm, **t)
    assert t["out"]._version > before["out"] and all(t[n]._version == before[n] for n in watched[:4])
    x = zeros(4, 64)
    version = x._version
    lsm.lsm_compact_pages(x, ints([[3]]), ints([1]), 16)
    assert x._version > version
    with torch.inference_mode():
        y = zeros(4, 64)
        lsm.lsm_copy_pages(y, ints([0]), ints([1]))  # counts no writes
    # a saved tensor that is overwritten is noticed
    w = torch.ones(4, 64, device="cuda", requires_grad=True)
    z = (w * x).sum()
    lsm.lsm_copy_pages(x, ints([0]), ints([1]))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.backward()


def test_the_workspace_of_windows(lsm):
    """A caller's own workspace: large enough, or refused."""
    gen = torch.Generator().manual_seed(1)
    q, pool = torch.randn(1, 8, 64, generator=gen).to(BF16).cuda(), torch.randn(200, 2, 16, 1, 64, generator=gen).to(BF16).cuda()
    b = lsm.PrefixBatch(ints([0, 1]), ints([]).reshape(1, 0), ints([0]), ints([0, 1]), torch.arange(200, dtype=torch.int32, device="cuda")[None], ints([3100]))
    want = lsm.lsm_prefix_attention(q, pool[:, 0], pool[:, 1], b, window=2500, sinks=3)
    space = torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(lsm.lsm_prefix_attention(q, pool[:, 0], pool[:, 1], b, window=2500, sinks=3, workspace=space), want)
    with pytest.raises(lsm.LsmError):
        lsm.lsm_prefix_attention(q, pool[:, 0], pool[:, 1], b, window=2500, sinks=3, workspace=space[:1024])
