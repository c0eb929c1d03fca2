"""What the cache's calls keep of device memory."""
import torch
import pytest

from test_gpu_cache import DEV, ints, steel

pytestmark = pytest.mark.gpu


def test_results_do_not_hold_the_workspace():
    """A result kept by its user keeps its own bytes, not the call's workspace (12 bytes a page)."""
    s, P = steel(), 70000
    t, l, r = ints([[0, -1], [1, -1]]), ints([5, 64]), ints([1, 1] + [0] * (P - 2))
    kept = [*s.pages_grow(t, l, r, ints([1, 1]))]
    pool = torch.zeros((P, 1, 16), dtype=torch.uint8, device=DEV)
    kept.append(s.pages_compact(pool, t, l, r))
    torch.cuda.synchronize()
    assert all(x.untyped_storage().nbytes() <= 64 for x in kept)


def test_a_wide_table_costs_no_workspace_without_a_mask():
    """A table for 2^20 tokens, 64 sequences of 8 heads: the 67 MB of lists of live pages are
    taken with a page mask only; both give the same."""
    s, B, M = steel(), 64, 16384
    pool = torch.full((3, 8, 68 * 64), 0x77, dtype=torch.uint8, device=DEV)
    t, l = torch.zeros((B, M), dtype=torch.int32, device=DEV), ints([100] * B)
    t[:, 1] = 2
    q = torch.ones((B, 8, 1, 64), dtype=torch.bfloat16, device=DEV)
    mask = torch.ones((B, 8, M), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    used, outs = [], []
    for m in (None, mask):
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        outs.append(s.attn_cache(q, pool, t, l, block_mask=m))
        used.append(torch.cuda.max_memory_allocated() - before)
    torch.cuda.synchronize()
    assert used[0] < 1 << 24 < 8 * B * 8 * M <= used[1]
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
