"""CPU-only checks of what the package's paged-cache calls refuse before the library is called."""
import pytest
import torch


@pytest.mark.parametrize("device", ["cpu", "meta", torch.device("cpu"), "cuda:1", torch.device("cuda", 7)])
def test_rope_table_is_made_on_the_current_gpu_alone(monkeypatch, device):
    """Host memory, or another GPU's, must not reach a kernel on the current one's stream."""
    import paper_2511_16138_amd as lsm
    from paper_2511_16138_amd import cache

    class Library:
        @staticmethod
        def lsm_rope_table(*args):
            raise AssertionError("the library was called")

    monkeypatch.setattr(cache, "_load", lambda: Library)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch, "empty", lambda *a, **k: pytest.fail("memory was taken"))
    with pytest.raises(ValueError, match="device"):
        lsm.lsm_rope_table(8, 64, device=device)


def calls(**change):
    """The three calls on tensors of matching shapes, some of them exchanged."""
    import paper_2511_16138_amd as lsm
    t = dict(q=torch.zeros(2, 4, 64, dtype=torch.bfloat16), k=torch.zeros(2, 2, 64, dtype=torch.bfloat16), v=torch.zeros(2, 2, 64, dtype=torch.bfloat16),
             pages=torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16), w=torch.ones(64), positions=torch.zeros(2, dtype=torch.int32), slots=torch.zeros(2, dtype=torch.int64),
             table=torch.zeros(8, 64), out=None)
    t.update(change)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=getattr(t["v"], "device", "cpu"))  # noqa: E731
    batch = lsm.PrefixBatch(ints([0, 2]), ints([[0]]), ints([16]), ints([0, 1, 2]), ints([[1], [2]]), ints([1, 1]))
    return {
        "rotate": lambda: lsm.lsm_rotate_heads(t["q"], t["k"], t["positions"], t["table"], q_weight=t["w"], q_out=t["out"]),
        "append": lambda: lsm.lsm_kv_append(t["k"], t["v"], t["positions"], t["slots"], t["pages"], t["pages"], t["table"], k_weight=t["w"], q=t["q"], q_out=t["out"]),
        "attend": lambda: lsm.lsm_prefix_attention(t["q"], t["pages"], t["pages"], batch, out=t["out"]),
    }


@pytest.mark.parametrize("name, what", [("rotate", "q"), ("append", "k"), ("attend", "q")])
def test_host_tensors_raise_value_error_with_or_without_a_gpu(name, what):
    with pytest.raises(ValueError, match=f"^{what} must be a GPU tensor"):
        calls()[name]()


@pytest.mark.parametrize("name", ["rotate", "append", "attend"])
def test_what_is_no_tensor_raises_value_error_with_or_without_a_gpu(name):
    with pytest.raises(ValueError, match="must be a tensor"):
        calls(**({"pages": 5} if name == "attend" else {"k": 5, "q": 5}))[name]()


@pytest.mark.parametrize("name, which", [("rotate", "q"), ("rotate", "k"), ("rotate", "w"), ("rotate", "table"), ("rotate", "out"), ("append", "k"), ("append", "v"),
                                         ("append", "q"), ("append", "w"), ("append", "pages"), ("append", "out"), ("attend", "q"), ("attend", "pages"), ("attend", "out")])
@pytest.mark.parametrize("kind", ["gradients", "tangent"])
def test_inputs_with_gradients_or_tangents_are_refused(name, which, kind):
    """There is no backward pass and no forward mode: outputs would be without a word about it constants of either."""
    from torch.autograd import forward_ad

    def run(want):
        shapes = dict(q=(2, 4, 64), k=(2, 2, 64), v=(2, 2, 64), pages=(3, 16, 2, 64), w=(64,), table=(8, 64), out=(2, 4, 64))
        x = torch.zeros(shapes[which], dtype=torch.float32 if which in ("w", "table") else torch.bfloat16)
        x = x.requires_grad_() if kind == "gradients" else forward_ad.make_dual(x, torch.ones_like(x))
        # on the CPU: whatever has no gradients or tangents is refused for being no GPU tensor
        with pytest.raises(ValueError) as e:
            calls(**{which: x})[name]()
        assert (kind in str(e.value)) == want, str(e.value)

    if kind == "gradients":
        run(True)
        with torch.no_grad():
            run(False)
    else:
        with forward_ad.dual_level():
            run(True)
            with forward_ad._set_fwd_grad_enabled(False):
                run(False)
