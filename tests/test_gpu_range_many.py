"""lsm_range_scan of more ranges than one launch has workgroups for: HIP takes fewer than 2^32 threads, 512 a range."""
import pytest
import torch

from gpu_util import build_tree, dev

pytestmark = pytest.mark.gpu

RANGES = (1 << 23) + 77


def test_range_scan_of_more_ranges_than_a_launch_takes():
    import paper_2511_16138_amd as g
    from workloads import lsm
    run = lsm.config1(device=dev()).runs[0][:4001].contiguous()
    tree = build_tree(g, [run])
    lo, hi = run[:-1, :4].contiguous(), run[1:, :4].contiguous()
    entries, counts = g.lsm_range_scan(tree, lo, hi, 1)           # 4,000 ranges of one entry (or one tombstone) each
    assert int(counts.max()) == 1
    at = torch.arange(RANGES, device=dev()) % 4000
    many = torch.full((RANGES, 1, 8), -1, dtype=torch.int64, device=dev())
    print("range scan", RANGES, flush=True)
    _, found = g.lsm_range_scan(tree, lo[at], hi[at], 1, entries=many)
    torch.cuda.synchronize()
    assert torch.equal(found, counts[at])
    live = counts == 1
    for first in range(0, RANGES, 1 << 21):
        part = slice(first, first + (1 << 21))
        keep = live[at[part]]
        assert torch.equal(many[part][keep], entries[at[part]][keep]) and bool((many[part][~keep] == -1).all())
