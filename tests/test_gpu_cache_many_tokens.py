"""lsm_rotate_heads and lsm_kv_append of more tokens than one launch has threads for: HIP takes fewer than 2^32 of them, 64 a token."""
import pytest
import torch

import cache_reference as ref

pytestmark = pytest.mark.gpu

TOKENS = (1 << 26) + 37  # one head of 8 elements each: 1 GiB


def test_rotation_of_more_tokens_than_a_launch_has_threads_for():
    import paper_2511_16138_amd as lsm
    x = torch.empty((TOKENS, 1, 8), dtype=torch.bfloat16, device="cuda").normal_()
    table = lsm.lsm_rope_table(1000, 8)
    positions = (torch.arange(TOKENS, device="cuda") * 7 % 1000).to(torch.int32)
    print("rotate", TOKENS, flush=True)
    out, _ = lsm.lsm_rotate_heads(x, None, positions, table)
    for part in (slice(0, 300), slice((1 << 25) - 150, (1 << 25) + 150), slice(TOKENS - 300, TOKENS)):
        ref.assert_within(out[part], *ref.rotate(x[part].cpu(), None, table.cpu(), positions[part].cpu()), "rotated")
    # every token: a rotation keeps lengths
    for first in range(0, TOKENS, 1 << 23):
        a, b = (t[first:first + (1 << 23)].float().norm(dim=-1) for t in (x, out))
        assert bool(((a - b).abs() <= 0.01 * a + 1e-3).all())
    del out
    print("append", TOKENS, flush=True)
    pages = torch.zeros((2, (TOKENS + 15) // 16, 16, 1, 8), dtype=torch.bfloat16, device="cuda")
    slots = torch.arange(TOKENS, device="cuda").flip(0)
    lsm.lsm_kv_append(x, x, None, slots, pages[0], pages[1], None)
    for side in pages:
        assert torch.equal(side.view(-1, 1, 8)[:TOKENS].flip(0), x)
