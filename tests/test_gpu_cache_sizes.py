"""Calls on the paged cache at the sizes where an index passes 31 bits or a rule changes."""
import numpy as np
import pytest
import torch

from test_gpu_cache import DEV, bf16, check_attention, ints, random_pool, say, steel

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


@pytest.mark.parametrize("B,H,D,S,lo", [
    (447, 1, 64, 1, 1700), (448, 1, 128, 1, 1700), (64, 7, 64, 2, 1400), (512, 1, 64, 1, 1700),
    (513, 1, 64, 1, 1700), (703, 1, 64, 1, 1700), (704, 1, 64, 1, 1700), (769, 1, 64, 1, 1700),
    (192, 1, 64, 1, 1400), (193, 1, 64, 1, 1700), (448, 1, 64, 20, 1700), (128, 1, 64, 20, 1400),
    (129, 1, 64, 20, 1700)])
def test_lists_around_the_rules_of_the_deal(B, H, D, S, lo):
    """Lists of nearly one length (or not) on both sides of where each has a workgroup of its own, and
    of where few are filled up: a quarter of the 768 workgroups (512 with more than 16 rows)."""
    rng = np.random.default_rng(B * H + S)
    lens = rng.integers(lo, 1801, B)
    pool = random_pool(rng, 120, H, D, 122, 129)
    table = rng.integers(0, 120, (B, 29)).astype(np.int32)
    check_attention(f"{B * H} lists", pool, table, lens, bf16(rng, (B, H, S, D)), D ** -0.5)
