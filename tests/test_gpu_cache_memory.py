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
