"""The model of the page growth where pages are missing."""
import numpy as np

import oracle.kv_cache as kv


def test_growth_counts_the_pages_that_are_missing():
    """As many as were missing: with so many more pages the same call fits, and with one fewer it
    does not."""
    # two rows write into page 0 that both hold: one copies, the other keeps it
    table, lens, refs = np.array([[0, -1], [0, -1]]), np.array([5, 5]), np.array([2])
    assert kv.grow(table, lens, refs, [1, 1])[5] == -1
    rng = np.random.default_rng(0)
    for _ in range(200):
        B, M, P = int(rng.integers(1, 7)), 6, 30
        lens = rng.integers(0, 3 * 64, B)
        lens[rng.random(B) < 0.5] = lens[0]
        table, ids = np.full((B, M), -1), list(rng.permutation(P))
        for b in range(B):
            n = -(-int(lens[b]) // 64)
            table[b, :n] = table[0, :n] if b and lens[b] == lens[0] else [ids.pop() for _ in range(n)]
        refs = np.ones(P, np.int32)  # none is free
        for p in range(P):
            refs[p] = max(1, (table == p).sum())
        new = rng.integers(0, 150, B)
        t, l, r, src, dst, left = kv.grow(table, lens, refs, new)
        assert left <= 0
        if left < 0:
            assert (t == table).all() and (l == lens).all() and (r == refs).all()
            assert (src == -1).all() and (dst == -1).all()
            assert kv.grow(table, lens, np.append(refs, [0] * -(left + 1)), new)[5] == -1
        assert kv.grow(table, lens, np.append(refs, [0] * -left), new)[5] == 0
