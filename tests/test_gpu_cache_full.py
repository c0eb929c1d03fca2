"""Decoding steps on a pool that is too full: nothing is written, and the search goes on
once pages are free."""
import numpy as np
import pytest
import torch

import oracle.kv_cache as kv
from test_gpu_cache import DEV, bf16, gpu, ints, random_pool, steel

pytestmark = pytest.mark.gpu


def grown(B, P, spare, seed):
    """B sequences of 1 .. 200 tokens in a pool of P pages of which `spare` are free; rows 0 and 1
    share their pages."""
    rng = np.random.default_rng(seed)
    lens = rng.integers(1, 200, B).astype(np.int32)
    lens[0] = lens[1] = 100  # the shared last page is written into
    M = 8
    ids, table = list(rng.permutation(P)[spare:]), np.full((B, M), -1, np.int32)
    refs = np.zeros(P, np.int32)
    refs[ids] = 1  # held elsewhere, but for those that a row takes
    for b in range(B):
        n = -(-int(lens[b]) // 64)
        table[b, :n] = table[0, :n] if b == 1 else [ids.pop() for _ in range(n)]
    refs[table[1, :2]] += 1
    return rng, table, lens, refs


# 1024 rows and 65,536 pages are the most of the growth by one thread a row
@pytest.mark.parametrize("B,P", [(3, 30), (40, 400), (1024, 5000), (1025, 5000), (5, 65600)])
def test_took_is_new_or_nothing(B, P):
    s = steel()
    for spare in (0, B // 2, 8 * B):
        rng, table, lens, refs = grown(B, P + 8 * B, spare, B + spare)
        for new in (rng.integers(-2, 90, B), np.ones(B, int), np.zeros(B, int), np.full(B, 8 * 64)):
            new = new.astype(np.int32)
            t, l, r, took = ints(table), ints(lens), ints(refs), ints(np.full(B, 77))
            src, dst, left = s.pages_grow(t, l, r, ints(new), took=took)
            wt, wl, wr, ws, wd, wleft = kv.grow(table, lens, refs, new)
            want = np.maximum(new, 0) if wleft >= 0 else 0 * new
            assert int(left) == wleft and np.array_equal(took.cpu().numpy(), want)
            for got, exact in ((t, wt), (l, wl), (r, wr), (src, ws), (dst, wd)):
                assert np.array_equal(got.cpu().numpy(), exact)


@pytest.mark.parametrize("captured", [False, True])
def test_a_step_on_a_full_pool_writes_nothing(captured):
    """Grow, copy, append and attend: with no page free every byte stays, the rows are 0; after
    another holder let go of pages the same step (or graph) goes on."""
    s, H, D, B, P = steel(), 2, 64, 4, 12
    rng, table, lens, refs = grown(B, P, 0, 3)
    pool = random_pool(rng, P, H, D, 122, 129)
    st = [gpu(pool), ints(table), ints(lens), ints(refs)]
    k, v, q = gpu(bf16(rng, (B, H, 1, D))), gpu(bf16(rng, (B, H, 1, D))), gpu(bf16(rng, (B, 4, 1, D)))
    new, took = ints(np.ones(B)), ints(np.zeros(B))

    def step():
        src, dst, left = s.pages_grow(*st[1:], new, took=took)
        s.pages_copy(st[0], src, dst)
        s.cache_append(k, v, *st[:3], new=took)
        return left, *s.attn_cache(q, *st[:3], new=took)

    if captured:
        step()  # a first call outside: it fits no page and changes nothing
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = step()

        def run():
            graph.replay()
            return outs
    else:
        run = step
    for _ in range(3):
        left, out, lse = run()
        torch.cuda.synchronize()
        assert int(left) < 0 and not took.any()
        assert not out.any() and torch.isneginf(lse).all()
        for got, was in zip(st, (pool, table, lens, refs)):
            assert np.array_equal(got.cpu().numpy(), was)
    held = set(table[table >= 0].tolist())
    refs[[p for p in range(P) if p not in held]] = 0
    st[3].copy_(ints(refs))
    left, out, lse = run()
    torch.cuda.synchronize()
    ones = np.ones(B, np.int32)
    table, lens, refs, ws, wd, wleft = kv.grow(table, lens, refs, ones)
    assert int(left) == wleft >= 0 and took.tolist() == [1] * B
    for a, b in zip(ws, wd):
        if a >= 0:
            pool[b] = pool[a]
    kv.append(k.cpu().double().numpy(), v.cpu().double().numpy(), pool, table, lens, ones)
    for got, want in zip(st, (pool, table, lens, refs)):
        assert np.array_equal(got.cpu().numpy(), want)
    wo, wl = kv.attention(q.cpu().double().numpy(), pool, table, lens, D ** -0.5, new=ones)
    # weights in bf16: 2^-8 of sum p |v| <= 6 * 2 (scales up to 2^1), 1% for the fp32 terms
    assert np.abs(out.cpu().double().numpy() - wo).max() <= 2.0 ** -8 * 1.01 * 12
    assert np.abs(lse.cpu().double().numpy() - wl).max() <= 1e-4


def test_took_is_checked():
    s = steel()
    t, l, r, n = ints([[0, -1]]), ints([3]), ints([1, 0]), ints([1])
    with pytest.raises(s.SteelError, match="alias"):
        s.pages_grow(t, l, r, n, took=n)
    with pytest.raises(ValueError, match="took"):
        s.pages_grow(t, l, r, n, took=torch.zeros(2, dtype=torch.int32, device=DEV))
    with pytest.raises(ValueError, match="took"):
        s.pages_grow(t, l, r, n, took=torch.zeros(1, dtype=torch.int64, device=DEV))
    assert l.tolist() == [3]
