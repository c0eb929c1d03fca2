"""Scores of attention over the paged cache whose products differ much in size: the sums have to
be fp32.

A score of D products is off by at most (D + 2) 2^-24 times the sum of their magnitudes A (D
additions and two roundings of 2^-24 each), and lse of one key, which is the scaled score, by
2^-20 (1 + |lse|) more for the logarithm and its base."""
import numpy as np
import pytest
import torch

import oracle.kv_cache as kv
from test_gpu_cache import bf16, gpu, ints, random_pool, say, steel

pytestmark = pytest.mark.gpu


def check_one_key(name, pool, q, scale):
    """Sequences of one token, one page each: lse against the exact score."""
    B, Hq, S, D = q.shape
    new = ints(np.ones(B))
    _, lse = steel().attn_cache(gpu(q), gpu(pool), ints(np.arange(B)[:, None]), ints(np.ones(B)),
                                new=new, scale=scale)
    got = lse.double().cpu().numpy()[:, :, 0]
    k = np.stack([kv.unpack(pool, b, 0, 0)[0] for b in range(B)])
    x = q.double().numpy()[:, :, 0]
    want, A = (np.einsum("bd,bhd->bh", f(k), f(x)) * scale for f in (np.asarray, np.abs))
    tol = (D + 2) * 2.0 ** -24 * A + 2.0 ** -20 * (1 + np.abs(want))
    say(f"[cache] scores {name}: q {tuple(q.shape)}, share of the bound {(np.abs(got - want) / tol).max():.2f}")
    assert (np.abs(got - want) <= tol).all(), name


# rows of a key/value head: 8 and 32 in one tile or two, more in tiles of 128
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S", [1, 4, 40])
def test_small_products_beside_a_large_one(D, S):
    """One channel of the query 2^8, 2^11 or 2^14 times larger than the others, at every place."""
    rng = np.random.default_rng(D + S)
    B, G = 2 * D, 8
    pool = random_pool(rng, B, 1, D, 127, 128)
    for e in (8, 11, 14):
        q = bf16(rng, (B, G, S, D))
        q[torch.arange(B), :, :, torch.arange(B) % D] *= 2.0 ** e
        check_one_key(f"2^{e}", pool, q, D ** -0.5)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S", [1, 4, 40])
def test_large_products_that_cancel(D, S):
    """Two channels of opposite products, and what the small ones leave."""
    rng = np.random.default_rng(D + S + 1)
    B, G = 2 * D, 8
    pool = random_pool(rng, B, 1, D, 127, 128)
    pool[..., :32 * D] = 0x22  # key codes 1
    a, b = np.arange(B) % D, (np.arange(B) * 7 + 1) % D
    for e in (4, 10):
        q = bf16(rng, (B, G, S, D))
        q[torch.arange(B), :, :, torch.tensor(a)] = 2.0 ** e
        q[torch.arange(B)[torch.tensor(a != b)], :, :, torch.tensor(b[a != b])] = -2.0 ** e
        check_one_key(f"2^{e} - 2^{e}", pool, q, 1.0)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S", [1, 4, 40])
def test_scores_of_every_mixture_of_scales(D, S):
    """Key scales from 2^-7 to 2^3 and normal queries, as a model might have them."""
    rng = np.random.default_rng(D + S + 2)
    check_one_key("mixed", random_pool(rng, 512, 1, D), bf16(rng, (512, 8, S, D)), D ** -0.5)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("S", [1, 4, 40])
def test_a_query_of_infinities_is_nan_whatever_the_keys(D, S):
    """Also where every score would be -inf, and a row must not pass for one without a key."""
    B = 4
    pool = np.zeros((B, 1, 68 * D), np.uint8)
    pool[..., 64 * D:] = 127
    pool[0, :, :32 * D], pool[1, :, :32 * D], pool[2, :, :32 * D] = 0x22, 0xAA, 0x00  # 1, -1, 0
    q = torch.ones((B, 8, S, D), dtype=torch.bfloat16)
    q[:, 0, 0, D - 1], q[:, 1, 0, 0], q[:, 2, 0, D // 2] = float("inf"), -float("inf"), float("nan")
    s = steel()
    out, lse = s.attn_cache(gpu(q), gpu(pool), ints(np.arange(B)[:, None]), ints([S] * B))
    bad = torch.zeros((B, 8, S), dtype=torch.bool, device=out.device)
    bad[:, :3, 0] = True
    assert torch.equal(torch.isnan(out).all(-1), bad) and torch.equal(torch.isnan(lse), bad)
