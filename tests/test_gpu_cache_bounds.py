"""Attention over the paged cache where values of very different sizes stand side by side: every
row against its own bound.

With p the weights of a row, A = max_j sum_d |q_d k_jd| scale over the keys it sees, n their
number and V the largest |v| of a 32-channel group among them, and with u = 2^-8 for the
rounding of a weight to bf16,

  |out - exact| <= (u + 2 (D + 2) 2^-24 A + 2^-18) sum_j p_j |v_j| + n (V 2^-126 + 2^-123)

sum by sum as in test_gpu_cache.py.  The last term: a weight below 2^-126 is not a normal fp32
number and counts for anything up to that, and so does a product of a weight and a scale,
which meets codes of up to 6 < 2^3.  It belongs to the row and the channel group: what stands in other
sequences, groups or behind the row's last key does not widen it."""
import numpy as np
import pytest
import torch

import oracle.kv_cache as kv
from test_gpu_cache import bf16, gpu, ints, random_pool, random_table, say, steel

pytestmark = pytest.mark.gpu


def by_row(q, pool, table, lens, scale):
    """Exact rows, sum p |v|, n V and A of every row (causal), from keys and values that the model
    reads out of the pool."""
    B, Hq, S, D = q.shape
    H = pool.shape[1]
    out, spread, top = (np.zeros((B, Hq, S, D)) for _ in range(3))
    big, lse, count = np.zeros((B, Hq, S)), np.full((B, Hq, S), -np.inf), np.zeros((B, Hq, S))
    for b in range(B):
        n = int(lens[b])
        pages = table[b, :-(-n // 64)]
        for g in range(H):
            k, v = (np.concatenate([kv.unpack(pool, p, g, w) for p in pages])[:n] for w in (0, 1))
            for h in range(g * Hq // H, (g + 1) * Hq // H):
                for i in range(S):
                    m = n - S + i + 1
                    if m <= 0:
                        continue
                    s = k[:m] @ q[b, h, i] * scale
                    w = np.exp(s - s.max())
                    lse[b, h, i] = s.max() + np.log(w.sum())
                    w /= w.sum()
                    out[b, h, i], spread[b, h, i] = w @ v[:m], w @ np.abs(v[:m])
                    group = np.abs(v[:m]).max(0).reshape(-1, 32).max(1)
                    top[b, h, i], count[b, h, i] = np.repeat(group, 32), m
                    big[b, h, i] = (np.abs(k[:m]) @ np.abs(q[b, h, i])).max() * scale
    return out, spread, top, big, lse, count


def check(name, pool, table, lens, q, scale):
    """Returns the part of the bound that does not shrink with the row, relative to sum p |v|."""
    out, lse = steel().attn_cache(gpu(q), gpu(pool), ints(table), ints(lens), scale=scale)
    got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
    D = q.shape[3]
    want, spread, top, big, wl, n = by_row(q.double().numpy(), pool, table, lens, scale)
    e = (D + 2) * 2.0 ** -24 * big[..., None]
    slack = n[..., None] * (top * 2.0 ** -126 + 2.0 ** -123)
    tol = (2.0 ** -8 + 2 * e + 2.0 ** -18) * spread + slack
    off = np.abs(got - want)
    say(f"[cache] {name}: q {tuple(q.shape)} lens {list(lens)}, share of the bound "
        f"{(off / np.maximum(tol, 1e-300)).max():.2f}")
    assert (off <= tol).all(), name
    seen = n > 0
    assert (np.abs(gl - wl)[seen] <= (e[..., 0] + 2.0 ** -20 * (1 + np.abs(wl)))[seen]).all()
    return slack, spread


SHAPES = [(64, 1, [700, 130, 3]), (128, 1, [700, 130, 3]), (128, 4, [700, 130, 4]), (64, 7, [333, 70, 7]),
          (128, 40, [300, 130, 40]), (64, 40, [300, 130, 40]), (128, 1, [3000, 130, 900]),
          (64, 5, [2500, 100, 64])]


@pytest.mark.parametrize("D,S,lens", SHAPES)
def test_one_size_for_each_sequence(D, S, lens):
    """Values around 2^-87, 1 and 2^123, a sequence each: the small ones keep their precision."""
    rng = np.random.default_rng(D + S)
    P = sum(-(-n // 64) for n in lens) + 2
    pool, table = random_pool(rng, P, 2, D), random_table(rng, lens, P)
    for b, e in enumerate((40, 127, 250)):
        pool[table[b][table[b] >= 0], :, 66 * D:] = e
    slack, spread = check("a size each", pool, table, lens, bf16(rng, (3, 8, S, D)), D ** -0.5)
    # the bound can fail: a row's fixed part is nothing beside a typical channel of it
    assert (slack.max(-1) <= 2.0 ** -10 * 2.0 ** -8 * np.median(spread, -1)).all()


@pytest.mark.parametrize("D,S,lens", SHAPES)
def test_one_size_for_each_group_of_channels(D, S, lens):
    """Groups of 32 channels around 2^-60, 2^60, 2^-5, 2^20 in the same tokens."""
    rng = np.random.default_rng(D + S + 1)
    P = sum(-(-n // 64) for n in lens) + 2
    pool, table = random_pool(rng, P, 2, D), random_table(rng, lens, P)
    groups = np.array([67, 187, 122, 147], np.uint8)[:D // 32]
    pool[..., 66 * D:] = np.tile(groups, 64)
    slack, spread = check("a size a group", pool, table, lens, bf16(rng, (3, 8, S, D)), D ** -0.5)
    typical = np.repeat(np.median(spread.reshape(*spread.shape[:-1], -1, 32), -1), 32, -1)
    assert (slack <= 2.0 ** -10 * 2.0 ** -8 * typical).all()


@pytest.mark.parametrize("D,S,lens", SHAPES)
@pytest.mark.parametrize("scale", [None, 2.0])
def test_sizes_mixed_token_by_token(D, S, lens, scale):
    """Scales from 2^-90 to 2^63 (exponents add up inside 16 bits) and to 2^120, side by side; with a
    scale of 2 most weights are 0, next to values of any size."""
    rng = np.random.default_rng(D + S + 2)
    P = sum(-(-n // 64) for n in lens) + 2
    pool, table = random_pool(rng, P, 2, D), random_table(rng, lens, P)
    for lo, hi in ((37, 191), (100, 192), (37, 248), (120, 128)):
        pool[..., 66 * D:] = rng.integers(lo, hi, (P, 2, 2 * D))
        check(f"scales {lo} .. {hi}", pool, table, lens, bf16(rng, (3, 8, S, D)), scale or D ** -0.5)


@pytest.mark.parametrize("D,S", [(64, 1), (128, 1), (128, 3), (64, 40)])
def test_small_values_behind_weightless_large_ones(D, S):
    """Keys of one sign make the last token's weight all but 1 and every other 0 in fp32; the others'
    values are 2^70 times larger and must not show."""
    rng = np.random.default_rng(D * S)
    lens = [64 * 5 + S]
    pool, table = random_pool(rng, 8, 1, D), random_table(rng, lens, 8)
    pool[..., :32 * D] = 0xAA  # keys -1 ..
    pool[..., 64 * D:66 * D] = 127
    for i in range(S):  # .. and +1 for the tokens that the queries stand at, later ones larger
        page, tok = table[0, (lens[0] - S + i) // 64], (lens[0] - S + i) % 64
        pool[page, 0, tok * (D // 2):(tok + 1) * (D // 2)] = 0x22
        pool[page, 0, 64 * D:66 * D].reshape(64, D // 32)[tok] = 127 + i // 8
    pool[..., 66 * D:] = 127 + 50
    for i in range(S):
        page, tok = table[0, (lens[0] - S + i) // 64], (lens[0] - S + i) % 64
        pool[page, 0, 66 * D:].reshape(64, D // 32)[tok] = 127 - 20
    q = torch.ones((1, 4, S, D), dtype=torch.bfloat16)
    slack, spread = check("weightless", pool, table, lens, q, 4.0)
    assert (slack <= 2.0 ** -20 * np.median(spread, -1)[..., None]).all()
