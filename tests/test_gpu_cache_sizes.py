"""Calls on the paged cache at the sizes where an index passes 31 bits or a rule changes."""
import numpy as np
import pytest
import torch

from test_gpu_cache import DEV, ints, say, steel

pytestmark = pytest.mark.gpu


def test_rows_of_an_empty_sequence_beyond_31_bits():
    """2^21 key/value heads of 32 rows of 128 channels, a sequence without a token and a table that
    is split over workgroups: 2^31 groups of 4 channels to fill with zeros."""
    H, G, D = 1 << 21, 32, 128
    say(f"[cache] {H} heads, {torch.cuda.mem_get_info()[0] >> 30} GiB free")
    pool = torch.zeros((1, H, 68 * D), dtype=torch.uint8, device=DEV)
    q = torch.ones((1, 1, 1, D), dtype=torch.bfloat16, device=DEV).expand(1, H * G, 1, D)
    out = torch.ones((1, H * G, 1, D), dtype=torch.bfloat16, device=DEV)
    lse = torch.ones((1, H * G, 1), dtype=torch.float32, device=DEV)
    steel().attn_cache(q, pool, ints(np.zeros((1, 25))), ints([0]), out_dtype=torch.bfloat16, out=out, lse=lse)
    torch.cuda.synchronize()
    assert not any(bool(x.any()) for x in out.view(64, -1)) and bool(torch.isneginf(lse).all())
