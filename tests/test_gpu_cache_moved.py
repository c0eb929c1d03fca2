"""Where a compaction puts the pages that its table does not hold."""
import numpy as np
import pytest
import torch

import oracle.kv_cache as kv
from test_gpu_cache import DEV, gpu, ints, random_rows, steel

pytestmark = pytest.mark.gpu


# up to 65,536 pages are ranked by one workgroup, more by several
@pytest.mark.parametrize("B,M,P", [(1, 2, 3), (5, 9, 70), (30, 30, 1000), (40, 200, 9000), (3, 2, 4096),
                                   (200, 300, 65536), (200, 300, 70003)])
def test_compaction_tells_where_pages_went(B, M, P):
    """Every live page, held by this table, by another or by none, is found where `to` says, and
    a second table follows by it."""
    rng = np.random.default_rng(P)
    table, lens, refs = random_rows(rng, B, M, P)
    other = np.where(rng.random(P) < 0.3)[0].astype(np.int32)  # pages that others hold
    refs[other] += 1
    pool = rng.integers(0, 256, (1, P, 1, 16), dtype=np.uint8)
    pd, t, r = gpu(pool), ints(table), ints(refs)
    to = torch.full((P,), 77, dtype=torch.int32, device=DEV)
    live = int(steel().pages_compact(pd, t, ints(lens), r, to=to))
    got, moved = to.cpu().numpy(), pd.cpu().numpy()
    assert live == (refs > 0).sum() and (got[refs == 0] == -1).all()
    at = got[refs > 0]
    assert np.array_equal(np.sort(at), np.arange(live))
    assert np.array_equal(moved[0, at], pool[0, refs > 0])
    assert np.array_equal(r.cpu().numpy()[at], refs[refs > 0])
    stay = np.flatnonzero(refs[:live] > 0)
    assert np.array_equal(got[stay], stay)
    for b in range(B):
        held = kv.held(table, lens, b)
        assert np.array_equal(t.cpu().numpy()[b, :len(held)], got[held])
    if len(other):  # a second table, as a user rewrites it
        second = to[ints(other).long()]
        assert torch.equal(pd[0][second.long()], gpu(pool[0][other]))


def test_to_is_checked():
    s = steel()
    pool, t, l, r = torch.zeros((4, 1, 16), dtype=torch.uint8, device=DEV), ints([[0]]), ints([3]), ints([1] * 4)
    with pytest.raises(s.SteelError, match="alias"):
        s.pages_compact(pool, t, l, r, to=r)
    with pytest.raises(ValueError, match="to must be"):
        s.pages_compact(pool, t, l, r, to=ints([0] * 3))
