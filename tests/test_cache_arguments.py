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
