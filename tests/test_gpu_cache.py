"""The paged 4-bit cache on the GPU against its float64 model.

Bytes, tables and counts have to be equal.  Attention: with u = 2^-8 the rounding of
a number to bf16, every weight is rounded once (u), the sums are fp32 and a score of
D products is off by at most (D + 2) 2^-24 times the sum of their magnitudes A, which
moves its weight by that much (twice: numerator and denominator), so

  |out - exact| <= (u + 2 (D + 2) 2^-24 A + 2^-18) sum_j p_j |v_j|  (+ u |out| in bf16)
  |lse - exact| <= (D + 2) 2^-24 A + 2^-20 (1 + |lse|)

with 2^-18 and 2^-20 for the sums' own roundings and the exponential's (a few units of 2^-24 a
step over the pages and segments of a row).  A weight below 2^-126 of the largest is
not a normal fp32 number and may count as 0: each of a row's n keys then changes out by
up to 2^-126 max |v|, so n max |v| 2^-126 is added to the first bound (1e-34 where exact
outputs are smaller still, as with scores hundreds apart).
"""
import sys
import zlib

import numpy as np
import pytest
import torch

import oracle.kv_cache as kv

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")


def steel():
    import paper_2607_09385_amd as s
    s.load()
    return s


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def gpu(x, dtype=None):
    t = x if isinstance(x, torch.Tensor) else torch.from_numpy(np.ascontiguousarray(x))
    return t.to(DEV) if dtype is None else t.to(DEV, dtype)


def ints(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def random_pool(rng, P, H, D, lo=120, hi=131):
    """Random codes, scales 2^(lo - 127) .. 2^(hi - 128)."""
    pool = rng.integers(0, 256, (P, H, 68 * D), dtype=np.uint8)
    pool[..., 64 * D:] = rng.integers(lo, hi, (P, H, 4 * D))
    return pool


def random_table(rng, lens, P, extra=1):
    M = max(-(-max(n, 0) // 64) for n in lens) + extra
    ids = rng.permutation(P)
    table, at = np.full((len(lens), M), -1, np.int32), 0
    for b, n in enumerate(lens):
        k = -(-max(n, 0) // 64)
        table[b, :k] = ids[at:at + k]
        at += k
    return table


def bf16(rng, shape):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(torch.bfloat16)


# ---- append and load ----

APPENDS = [
    # name, Hkv, D, S, lens, new
    ("one_token", 2, 128, 1, [1, 64, 65, 200], None),
    ("one_token_d64", 3, 64, 1, [130], None),
    ("ragged", 1, 64, 70, [70, 133, 5, 64, 300], [70, 69, 5, 0, 33]),
    ("ragged_d128", 5, 128, 33, [40, 33, 90], [1, 33, 32]),
    ("clamped", 2, 64, 8, [20, 30, 8, 4], [100, -3, 8, 8]),  # more than S, negative, all, before 0
]


@pytest.mark.parametrize("case", APPENDS, ids=[c[0] for c in APPENDS])
@pytest.mark.parametrize("order", ["bhsd", "bshd", "shared_head"])
def test_append_and_load(case, order):
    name, H, D, S, lens, new = case
    rng = np.random.default_rng(zlib.crc32(name.encode()))
    B = len(lens)
    P = sum(-(-n // 64) for n in lens) + 2
    pool, table = rng.integers(0, 256, (P, H, 68 * D), dtype=np.uint8), random_table(rng, lens, P)
    if name == "ragged":
        table[1, 1], table[4, 4] = -7, P + 5  # pages that do not exist: dropped
    k, v = bf16(rng, (B, H, S, D)), bf16(rng, (B, H, S, D)) * 100
    if order == "shared_head":
        k, v = k[:, :1].expand(B, H, S, D), v[:, :1].expand(B, H, S, D)
    kd, vd = gpu(k), gpu(v)
    if order == "bshd":
        kd, vd = (t.transpose(1, 2).contiguous().transpose(1, 2) for t in (kd, vd))
    elif order == "shared_head":
        kd, vd = (t[:, :1].contiguous().expand(B, H, S, D) for t in (kd, vd))
    say(f"[cache] append {name} {order}")
    s, pd, td, ld = steel(), gpu(pool), ints(table), ints(lens)
    s.cache_append(kd, vd, pd, td, ld, new=None if new is None else ints(new))
    lk, lv = s.cache_load(pd, td, ld, S + 3, start=ints([n - S for n in lens]))
    torch.cuda.synchronize()
    want = pool.copy()
    kv.append(k.double().numpy(), v.double().numpy(), want, table, lens, new)
    assert np.array_equal(pd.cpu().numpy(), want)
    wk, wv = kv.load(want, table, lens, S + 3, [n - S for n in lens])
    # the pool began as random bytes: what its largest scales hold is beyond bf16
    for got, exact in ((lk, wk), (lv, wv)):
        fits = np.abs(exact) < 3e38
        assert np.array_equal(got.cpu().double().numpy()[fits], exact[fits])
        assert np.isnan(got.cpu().double().numpy()[np.isnan(exact)]).all()


def test_append_of_every_kind_of_number():
    """Every bf16 number as the largest of its 32 channels and as a smaller one."""
    bits = np.arange(65536, dtype=np.uint32).astype(np.uint16).view(np.int16)
    x = torch.from_numpy(bits.copy()).view(torch.bfloat16).view(1, 1, 512, 128)
    y = x.clone()
    y[..., ::32] = torch.tensor(2.0 ** 20, dtype=torch.bfloat16)
    finite = torch.isfinite(x)
    x = torch.where(finite | (torch.arange(512).view(1, 1, 512, 1) % 7 == 0), x, torch.zeros_like(x))
    rng = np.random.default_rng(0)
    perm = torch.from_numpy(rng.permutation(65536))
    z = x.reshape(-1)[perm].view(1, 1, 512, 128)  # neighbours of other sizes
    s = steel()
    table, lens = ints([np.arange(8)]), ints([512])
    for k, v in ((x, y), (z, x)):
        pd = torch.zeros((8, 1, 68 * 128), dtype=torch.uint8, device=DEV)
        s.cache_append(gpu(k), gpu(v), pd, table, lens)
        torch.cuda.synchronize()
        want = np.zeros((8, 1, 68 * 128), np.uint8)
        kv.append(k.double().numpy(), v.double().numpy(), want, np.arange(8)[None], [512])
        assert np.array_equal(pd.cpu().numpy(), want)


def test_load_of_lengths_that_do_not_fit():
    """Lengths below 0 and beyond the table, starts before 0: rows of zeros."""
    rng = np.random.default_rng(3)
    pool = random_pool(rng, 4, 2, 64)
    table, lens, start = np.array([[0, 1], [2, 3], [1, 9]]), [-5, 1000, 128], [0, 100, -10]
    s = steel()
    k, v = s.cache_load(gpu(pool), ints(table), ints(lens), 140, start=ints(start))
    wk, wv = kv.load(pool, table, lens, 140, start)
    assert np.array_equal(k.cpu().double().numpy(), wk) and np.array_equal(v.cpu().double().numpy(), wv)


# ---- attention ----

def check_attention(name, pool, table, lens, q, scale, out_dtype=None, order="bhsd", **kw):
    s = steel()
    say(f"[cache] attention {name}: q {tuple(q.shape)} pool {pool.shape} lens {list(lens)[:8]} "
        f"{ {k: v for k, v in kw.items() if not isinstance(v, np.ndarray)} }")
    qd = gpu(q)
    if order == "bshd":
        qd = qd.transpose(1, 2).contiguous().transpose(1, 2)
    dkw = {k: (ints(v) if k == "new" and v is not None else gpu(v) if isinstance(v, np.ndarray) else v)
           for k, v in kw.items()}
    out, lse = s.attn_cache(qd, gpu(pool), ints(table), ints(lens), scale=scale, out_dtype=out_dtype, **dkw)
    torch.cuda.synchronize()
    qn = q.double().numpy()
    wo, wl = kv.attention(qn, pool, table, lens, scale, **kw)
    D = q.shape[3]
    mag = pool.copy()
    mag[..., :64 * D] &= 0x77
    spread, _ = kv.attention(qn, np.concatenate((pool[..., :32 * D], mag[..., 32 * D:64 * D],
                                                 pool[..., 64 * D:]), -1), table, lens, scale, **kw)
    # A: the largest sum of magnitudes of a score, from the largest key magnitude
    kmax = np.nanmax(np.where(pool[..., 64 * D:66 * D] == 255, np.nan,
                              6 * 2.0 ** (pool[..., 64 * D:66 * D].astype(float) - 127)))
    A = min(np.abs(qn).sum(-1).max() * kmax * scale, 1e6)
    u, e = 2.0 ** -8, (D + 2) * 2.0 ** -24 * A
    got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(wo)), f"{name}: NaN pattern"
    assert np.array_equal(np.isneginf(gl), np.isneginf(wl)), f"{name}: -inf pattern"
    tol = (u + 2 * e + 2.0 ** -18) * spread + (u * np.abs(wo) if out_dtype == torch.bfloat16 else 0)
    vmax = 6 * 2.0 ** (pool[..., 66 * D:].astype(float) - 127)
    tol = tol + max(lens) * vmax[pool[..., 66 * D:] != 255].max() * 2.0 ** -126
    fin = ~np.isnan(wo)
    worst = (np.abs(got - wo) - tol)[fin]
    say(f"  max_abs {np.abs(got - wo)[fin].max():.2e} of {np.abs(wo)[fin].max():.2e}, "
        f"share of the tolerance {(np.abs(got - wo)[fin] / np.maximum(tol[fin], 1e-30)).max():.2f}")
    assert worst.max() <= 0, name
    dead = np.isneginf(wl)
    assert (got[dead] == 0).all()
    ok = np.isfinite(wl)
    assert (np.abs(gl[ok] - wl[ok]) <= e + 2.0 ** -20 * (1 + np.abs(wl[ok]))).all(), f"{name}: lse"
    return out, lse


ATTN = [
    # name, Hq, Hkv, D, S_q, lens, options
    ("token", 8, 2, 128, 1, [200, 64, 65, 1, 63], {}),
    ("token_d64", 12, 12, 64, 1, [130, 512], {}),
    ("token_bf16", 8, 8, 128, 1, [300, 17], {"out_dtype": torch.bfloat16}),
    ("group_of_five", 20, 4, 128, 1, [100, 333], {}),
    ("group_of_32", 32, 1, 64, 1, [190], {}),
    ("draft", 8, 2, 128, 4, [4, 67, 130, 200], {}),
    ("draft_d64", 6, 6, 64, 7, [7, 70, 135], {"out_dtype": torch.bfloat16, "order": "bshd"}),
    ("wide_group_draft", 24, 2, 64, 3, [100, 65], {}),
    ("chunk", 8, 2, 128, 90, [90, 200, 333], {}),
    ("chunk_d64", 4, 4, 64, 130, [130, 131, 400], {"order": "bshd"}),
    ("chunk_group_of_seven", 7, 1, 128, 65, [65, 300], {"out_dtype": torch.bfloat16}),
    ("not_causal", 4, 2, 64, 5, [200, 5, 64], {"causal": False}),
    ("not_causal_chunk", 4, 2, 128, 70, [200, 70], {"causal": False}),
    ("window", 8, 2, 128, 1, [700, 64, 65, 1], {"window_blocks": 2, "sink_blocks": 1}),
    ("window_one", 4, 4, 64, 3, [700, 66], {"window_blocks": 1}),
    ("window_wide_sink", 4, 2, 64, 1, [300, 100], {"window_blocks": 1, "sink_blocks": 50}),
    ("window_chunk", 8, 2, 64, 200, [700, 200, 264], {"window_blocks": 2, "sink_blocks": 1}),
    ("window_not_causal", 4, 2, 64, 70, [400, 70], {"window_blocks": 2, "causal": False}),
    ("padded", 8, 2, 128, 6, [100, 200, 3, 50], {"new": [6, 1, 0, 9]}),
    ("padded_chunk", 4, 2, 64, 100, [100, 300, 7, 50], {"new": [100, 33, 7, 0]}),
    ("more_queries_than_tokens", 4, 2, 64, 8, [3, 0, 100, 8], {}),
    ("more_queries_than_tokens_not_causal", 4, 2, 64, 8, [3, 0, 100], {"causal": False}),
    ("empty_sequences", 8, 2, 128, 1, [0, 100, 0, 0], {}),
    ("length_below_zero", 4, 2, 64, 1, [-3, 70], {}),
]


@pytest.mark.parametrize("case", ATTN, ids=[c[0] for c in ATTN])
def test_attention(case):
    name, Hq, H, D, S, lens, kw = case
    rng = np.random.default_rng(zlib.crc32(name.encode()))
    P = sum(-(-max(n, 0) // 64) for n in lens) + 2
    pool, table = random_pool(rng, P, H, D), random_table(rng, lens, P)
    q = bf16(rng, (len(lens), Hq, S, D))
    check_attention(name, pool, table, np.array(lens), q, D ** -0.5, **kw)


@pytest.mark.parametrize("S,D,keep", [(1, 128, 0.4), (1, 64, 0.0), (4, 128, 0.3), (90, 64, 0.5), (90, 128, 0.0)])
def test_attention_with_a_page_mask(S, D, keep):
    """Masked pages, down to none that is live for a head: rows of zeros."""
    rng = np.random.default_rng(int(S + D + 10 * keep))
    lens, H = np.array([700, S, 130]), 2
    P = sum(-(-n // 64) for n in lens) + 2
    pool, table = random_pool(rng, P, H, D), random_table(rng, lens, P)
    mask = (rng.random((3, H, table.shape[1])) < keep).astype(np.uint8) * 3
    mask[0, 1] = 0
    for kw in ({}, {"window_blocks": 3, "sink_blocks": 2}, {"causal": False}):
        check_attention("mask", pool, table, lens, bf16(rng, (3, 8, S, D)), D ** -0.5, block_mask=mask, **kw)


@pytest.mark.parametrize("S,D", [(1, 64), (5, 128), (80, 64), (80, 128)])
def test_pages_that_do_not_exist(S, D):
    rng = np.random.default_rng(S)
    lens, H = np.array([300, 200, 2000]), 2
    pool = random_pool(rng, 9, H, D)
    table = np.array([[0, -1, 2, 9, 4], [-1, -1, -1, -5, 7], [8, 1 << 30, 3, 5, 6]])
    check_attention("no page", pool, table, lens, bf16(rng, (3, 4, S, D)), D ** -0.5)


@pytest.mark.parametrize("S,D", [(1, 64), (1, 128), (3, 128), (70, 64), (70, 128)])
def test_bytes_behind_the_length_and_nan(S, D):
    """Whatever stands behind a sequence's tokens changes nothing; a stored NaN makes
    exactly the rows that see it NaN."""
    rng = np.random.default_rng(S + D)
    lens, H = np.array([100, 190, 65]), 2
    pool, table = random_pool(rng, 9, H, D), random_table(rng, [100, 190, 65], 9)
    q = bf16(rng, (3, 4, S, D))
    base = check_attention("clean", pool, table, lens, q, D ** -0.5)
    dirty = pool.copy()
    for b, n in enumerate(lens):
        page = table[b, (n - 1) // 64]
        for w in (0, 1):
            at = 64 * D + 2 * D * w
            dirty[page, :, at:at + 2 * D].reshape(H, 64, D // 32)[:, (n - 1) % 64 + 1:] = \
                rng.choice([0, 1, 253, 254, 255], (H, 63 - (n - 1) % 64, 1))
    unused = np.setdiff1d(np.arange(9), table[table >= 0])
    dirty[unused] = 255
    s = steel()
    out, lse = s.attn_cache(gpu(q), gpu(dirty), ints(table), ints(lens), scale=D ** -0.5)
    assert torch.equal(out, base[0]) and torch.equal(lse, base[1])
    for w, tok in ((0, 97), (1, 98), (1, 99), (1, 5)):
        bad = pool.copy()
        at = 64 * D + 2 * D * w
        bad[table[0, tok // 64], 1, at:at + 2 * D].reshape(64, D // 32)[tok % 64] = 255
        bad[table[0, tok // 64], 1, 32 * D * w:32 * D * (w + 1)].reshape(64, D // 2)[tok % 64] = 0
        want, _ = kv.attention(q.double().numpy(), bad, table, lens, D ** -0.5)
        got, _ = s.attn_cache(gpu(q), gpu(bad), ints(table), ints(lens), scale=D ** -0.5)
        got = got.cpu().double().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(want))
        assert np.array_equal(got[:, :2], base[0].cpu().double().numpy()[:, :2])


@pytest.mark.parametrize("D,Hq,H,S", [(64, 16, 1, 1), (128, 17, 1, 1), (64, 32, 1, 1), (128, 33, 1, 1),
                                      (128, 16, 1, 4), (64, 48, 1, 1), (128, 127, 1, 1), (64, 43, 1, 3)])
def test_rows_around_the_tiles(D, Hq, H, S):
    """16, 17, 32, 33, 64, 127 and 129 rows of one key/value head."""
    rng = np.random.default_rng(Hq)
    lens = np.array([1500, 200])
    pool, table = random_pool(rng, 30, H, D), random_table(rng, lens, 30)
    check_attention("tiles", pool, table, lens, bf16(rng, (2, Hq, S, D)), D ** -0.5)


@pytest.mark.parametrize("D,S", [(64, 1), (128, 2), (64, 50), (128, 50)])
def test_queries_that_are_not_finite(D, S):
    """They make their own rows NaN; in padding they are not read."""
    rng = np.random.default_rng(D)
    lens, H = np.array([300, 70]), 2
    pool, table = random_pool(rng, 9, H, D), random_table(rng, lens, 9)
    q = bf16(rng, (2, 8, S, D))
    s = steel()
    args = (gpu(pool), ints(table), ints(lens))
    clean, cl = s.attn_cache(gpu(q), *args)
    bad = q.clone()
    bad[0, 3, 0, 7] = float("nan")
    bad[1, 6, S - 1, D - 1] = float("inf")
    bad[1, 1, 0, 33] = -float("inf")
    out, lse = s.attn_cache(gpu(bad), *args)
    rows = torch.zeros((2, 8, S), dtype=torch.bool, device=DEV)
    rows[0, 3, 0] = rows[1, 6, S - 1] = rows[1, 1, 0] = True
    assert torch.isnan(out[rows]).all() and torch.isnan(lse[rows]).all()
    assert torch.equal(out[~rows], clean[~rows]) and torch.equal(lse[~rows], cl[~rows])
    if S > 1:
        new = ints([1, S - 1])
        pad = q.clone()
        pad[0, :, 1:] = float("nan")
        pad[1, :, S - 1:] = float("inf")
        a = s.attn_cache(gpu(pad), *args, new=new)
        b = s.attn_cache(gpu(q), *args, new=new)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and not torch.isnan(a[0]).any()


@pytest.mark.parametrize("D,S", [(64, 1), (128, 1), (128, 40), (64, 40)])
def test_values_of_every_size(D, S):
    """Scales from 2^-90 to 2^120 next to each other, keys included where scores allow it, and
    future tokens of the largest scales."""
    rng = np.random.default_rng(D + S)
    lens = np.array([700, 130, S])
    P = 20
    pool, table = random_pool(rng, P, 2, D), random_table(rng, lens, P)
    pool[..., 66 * D:] = rng.integers(37, 248, (P, 2, 2 * D))
    q = bf16(rng, (3, 8, S, D))
    check_attention("large", pool, table, lens, q, D ** -0.5)
    # one size per sequence: the small ones keep their precision
    for b, e in enumerate((40, 127, 250)):
        pool[table[b][table[b] >= 0], :, 66 * D:] = e
    check_attention("one size each", pool, table, lens, q, D ** -0.5)
    pool[..., 66 * D:] = rng.integers(122, 129, (P, 2, 2 * D))
    base = check_attention("plain", pool, table, lens, q, D ** -0.5)
    plain = pool.copy()
    if S > 1:  # the last token's value is large: only the last query sees it
        page, tok = table[0, 10], 699 % 64
        pool[page, :, 66 * D:].reshape(2, 64, D // 32)[:, tok] = 252
        pool[page, :, 32 * D:64 * D].reshape(2, 64, D // 2)[:, tok] = 0x77
        s = steel()
        out, _ = s.attn_cache(gpu(q), gpu(pool), ints(table), ints(lens), scale=D ** -0.5)
        # The page's large value moves the maximum of its rows at once, and rows of one wave
        # move it together, so the others' weights may round elsewhere: both results are
        # within u = 2^-8 of sum p |v| (u / 10 covers the fp32 terms), 2 u of each other.
        mag = plain.copy()
        mag[..., 32 * D:64 * D] &= 0x77
        spread, _ = kv.attention(q.double().numpy(), mag, table, lens, D ** -0.5)
        off = np.abs(out.cpu().double().numpy() - base[0].cpu().double().numpy())
        assert (off[0, :, :S - 1] <= 2 * 1.1 * 2.0 ** -8 * spread[0, :, :S - 1]).all()


@pytest.mark.parametrize("S", [1, 60])
def test_lengths_beyond_the_table(S):
    """Keys end with the table, positions do not."""
    rng = np.random.default_rng(S)
    pool, table = random_pool(rng, 12, 2, 64), rng.permutation(12).reshape(3, 4).astype(np.int32)
    lens = np.array([256, 300, 2 ** 31 - 1])
    for kw in ({}, {"causal": False}, {"window_blocks": 2, "sink_blocks": 1}):
        check_attention("beyond", pool, table, lens, bf16(rng, (3, 4, S, 64)), 0.125, **kw)


@pytest.mark.parametrize("D,S", [(64, 1), (128, 1), (128, 40)])
def test_sharp_and_flat_scores(D, S):
    """Scores of hundreds (one key takes all), far below zero, and all equal."""
    rng = np.random.default_rng(D)
    lens = np.array([900, 333])
    pool, table = random_pool(rng, 24, 2, D), random_table(rng, lens, 24)
    q = bf16(rng, (2, 8, S, D))
    check_attention("sharp", pool, table, lens, q, 2.0)
    check_attention("flat", pool, table, lens, q * 0, 1.0)
    pool[..., :32 * D] = 0x22  # all key codes +1: scores the sign of sum(q)
    check_attention("one sign", pool, table, lens, -q.abs(), 3.0)


LONG = [
    ("one_long", 32, 8, 128, 1, [20000], {}),
    ("ragged", 8, 2, 128, 1, [5000, 1, 64, 9000, 300, 2, 4097] + [33 * i for i in range(20)], {}),
    ("ragged_d64", 24, 24, 64, 2, [3000, 2, 65, 1000], {}),
    ("batch_of_many", 4, 2, 64, 1, [1 + (37 * i) % 200 for i in range(700)], {}),
    ("groups_of_four_rows", 32, 4, 64, 5, [2000, 777], {}),
    ("window", 8, 2, 64, 4, [9000, 5000, 100], {"window_blocks": 20, "sink_blocks": 2}),
    ("chunk", 8, 2, 128, 300, [3001, 300], {}),
    ("chunk_window", 4, 4, 64, 500, [4000, 777], {"window_blocks": 4, "sink_blocks": 1}),
    ("chunk_few_rows", 4, 4, 128, 17, [6000], {}),
    ("chunk_padded", 8, 8, 64, 256, [3000, 2000, 500], {"new": [256, 1, 100]}),
]


@pytest.mark.parametrize("case", LONG, ids=[c[0] for c in LONG])
def test_long_and_many(case):
    name, Hq, H, D, S, lens, kw = case
    rng = np.random.default_rng(zlib.crc32(name.encode()))
    P = sum(-(-n // 64) for n in lens) + 5
    pool, table = random_pool(rng, P, H, D, 122, 129), random_table(rng, lens, P, extra=7)
    q = bf16(rng, (len(lens), Hq, S, D))
    check_attention(name, pool, table, np.array(lens), q, D ** -0.5, out_dtype=torch.bfloat16, **kw)


SHORT = [c for c in ATTN if c[4] * c[1] // c[2] <= 32]


@pytest.mark.parametrize("case", SHORT, ids=[c[0] for c in SHORT])
def test_short_sequences_in_a_wide_table(case):
    """As test_attention, with room for more pages than one workgroup takes."""
    name, Hq, H, D, S, lens, kw = case
    rng = np.random.default_rng(zlib.crc32(name.encode()) + 1)
    P = sum(-(-max(n, 0) // 64) for n in lens) + 2
    pool, table = random_pool(rng, P, H, D), random_table(rng, lens, P, extra=40)
    kw = {k: v for k, v in kw.items() if k not in ("window_blocks", "sink_blocks")}
    check_attention(name, pool, table, np.array(lens), bf16(rng, (len(lens), Hq, S, D)), D ** -0.5, **kw)


@pytest.mark.parametrize("name,B,Hq,H,D,S,lo,hi", [
    ("one length", 57, 8, 8, 64, 1, 1900, 1900), ("nearly", 64, 16, 8, 128, 1, 1700, 1900),
    ("not nearly", 64, 8, 8, 64, 1, 1200, 1900), ("drafts", 128, 8, 4, 64, 3, 1700, 1800),
    ("too many", 100, 8, 8, 64, 1, 1700, 1700), ("three a unit", 95, 16, 8, 64, 2, 1800, 1801)])
def test_many_sequences_of_nearly_one_length(name, B, Hq, H, D, S, lo, hi):
    rng = np.random.default_rng(B)
    lens = rng.integers(lo, hi + 1, B)
    pool = random_pool(rng, 200, H, D, 122, 129)
    table = rng.integers(0, 200, (B, 30)).astype(np.int32)
    check_attention(name, pool, table, lens, bf16(rng, (B, Hq, S, D)), D ** -0.5)


@pytest.mark.parametrize("S,D", [(1, 64), (1, 128), (4, 128)])
def test_values_of_every_size_in_long_sequences(S, D):
    """Their partial results joined: values of 2^-90 to 2^120 and weights far apart."""
    rng = np.random.default_rng(D + S)
    lens = np.array([4000, 130, 9000])
    P = 210
    pool, table = random_pool(rng, P, 2, D), random_table(rng, lens, P)
    pool[..., 66 * D:] = rng.integers(37, 248, (P, 2, 2 * D))
    q = bf16(rng, (3, 8, S, D))
    check_attention("large", pool, table, lens, q, D ** -0.5)
    pool[..., 66 * D:] = rng.integers(122, 129, (P, 2, 2 * D))
    check_attention("sharp", pool, table, lens, q, 2.0)


@pytest.mark.parametrize("S,D", [(1, 64), (1, 128), (4, 128)])
def test_nan_in_a_long_sequence(S, D):
    """A stored NaN, in whatever part of its list, makes exactly the rows that see it NaN."""
    rng = np.random.default_rng(S + D)
    lens = np.array([5000, 900])
    pool, table = random_pool(rng, 100, 2, D, 122, 129), random_table(rng, lens, 100)
    q = bf16(rng, (2, 8, S, D))
    s = steel()
    base, _ = s.attn_cache(gpu(q), gpu(pool), ints(table), ints(lens))
    for w, tok in ((0, 3000), (1, 0), (1, 2500), (1, 4997), (0, 4999)):
        bad = pool.copy()
        at = 64 * D + 2 * D * w
        bad[table[0, tok // 64], 1, at:at + 2 * D].reshape(64, D // 32)[tok % 64] = 255
        bad[table[0, tok // 64], 1, 32 * D * w:32 * D * (w + 1)].reshape(64, D // 2)[tok % 64] = 0
        got, lse = s.attn_cache(gpu(q), gpu(bad), ints(table), ints(lens))
        sees = torch.arange(S, device=DEV) + lens[0] - S >= tok
        assert torch.isnan(got[0, 4:][:, sees]).all() and torch.equal(got[0, 4:][:, ~sees], base[0, 4:][:, ~sees])
        assert torch.equal(got[0, :4], base[0, :4]) and torch.equal(got[1], base[1])


@pytest.mark.parametrize("win,sink", [(22, 1), (23, 1), (24, 0), (25, 0)])
def test_windows_around_the_pages_of_a_workgroup(win, sink):
    """Queries on both sides of a page's end see one page more together."""
    rng = np.random.default_rng(win)
    for S, lens in ((2, [64 * 40 + 1, 64 * 30]), (3, [64 * 33 + 2, 65]), (1, [64 * 40 + 1, 64 * 40])):
        P = sum(-(-n // 64) for n in lens) + 2
        pool, table = random_pool(rng, P, 2, 64, 122, 129), random_table(rng, lens, P)
        check_attention("window", pool, table, np.array(lens), bf16(rng, (2, 8, S, 64)), 0.125,
                        window_blocks=win, sink_blocks=sink)


@pytest.mark.parametrize("name,Hq,H,D,S,lens,kw", [
    ("one segment and several", 8, 2, 64, 300, [300, 2000, 9000, 1100], {}),
    ("wide table", 5, 1, 128, 100, [100, 6000], {"causal": False}),
    ("window", 7, 1, 64, 200, [3000, 250], {"window_blocks": 30, "sink_blocks": 1}),
    ("tiles of many heads", 32, 8, 128, 200, [1700, 210], {})])
def test_tiles_of_unequal_lists(name, Hq, H, D, S, lens, kw):
    """Tiles whose lists are and are not cut into segments, in one call."""
    rng = np.random.default_rng(S + D)
    P = sum(-(-n // 64) for n in lens) + 5
    pool, table = random_pool(rng, P, H, D, 122, 129), random_table(rng, lens, P, extra=100)
    check_attention(name, pool, table, np.array(lens), bf16(rng, (len(lens), Hq, S, D)), D ** -0.5, **kw)


@pytest.mark.parametrize("name,B,Hq,H,D,S,hi,zero,keep", [
    ("ragged", 300, 4, 2, 64, 1, 1900, 0.3, None), ("few of many", 1000, 2, 1, 128, 2, 1700, 0.97, None),
    ("one of many", 130, 4, 4, 64, 1, 1900, 1.0, None), ("masked", 40, 8, 4, 64, 1, 1900, 0.2, 0.3),
    ("masked drafts", 70, 8, 2, 128, 5, 1800, 0.1, 0.1), ("none", 90, 4, 2, 64, 1, 1900, 2.0, None)])
def test_many_sequences_and_empty_ones(name, B, Hq, H, D, S, hi, zero, keep):
    """More sequences or lists than a wave has lanes, many of them without a page."""
    rng = np.random.default_rng(B)
    lens = rng.integers(1, hi, B)
    lens[rng.random(B) < zero] = 0
    if zero == 1.0:
        lens[B - 1] = hi
    pool = random_pool(rng, 150, H, D, 122, 129)
    table = rng.integers(0, 150, (B, 30)).astype(np.int32)
    kw = {} if keep is None else {"block_mask": (rng.random((B, H, 30)) < keep).astype(np.uint8)}
    q = bf16(rng, (B, Hq, S, D))
    if zero > 1.0:
        out, lse = steel().attn_cache(gpu(q), gpu(pool), ints(table), ints(lens))
        assert not out.any() and torch.isneginf(lse).all()
    else:
        check_attention(name, pool, table, lens, q, D ** -0.5, **kw)


@pytest.mark.parametrize("S,D,keep", [(1, 128, 0.1), (2, 64, 0.3), (100, 128, 0.2)])
def test_long_with_a_page_mask(S, D, keep):
    rng = np.random.default_rng(S)
    lens, H = np.array([12000, 100, 3000, 7777]), 2
    P = sum(-(-n // 64) for n in lens) + 5
    pool, table = random_pool(rng, P, H, D, 122, 129), random_table(rng, lens, P)
    mask = (rng.random((4, H, table.shape[1])) < keep).astype(np.uint8)
    mask[3, 0] = 0
    check_attention("long mask", pool, table, lens, bf16(rng, (4, 8, S, D)), D ** -0.5, block_mask=mask)


@pytest.mark.parametrize("S", [1, 70])
def test_pool_beyond_four_gib(S):
    """Pages whose byte offsets pass 32 bits, and the writes into them."""
    H, D, P = 8, 128, 66000
    rng = np.random.default_rng(S)
    pd = torch.zeros((P, H, 68 * D), dtype=torch.uint8, device=DEV)
    lens = np.array([150])
    small = random_pool(rng, 3, H, D)
    high = [P - 1, 61700, P - 3]
    pd[high] = gpu(small)
    k, v = bf16(rng, (1, H, 1, D)), bf16(rng, (1, H, 1, D))
    s = steel()
    s.cache_append(gpu(k), gpu(v), pd, ints([high]), ints(lens))
    kv.append(k.double().numpy(), v.double().numpy(), small, np.array([[0, 1, 2]]), lens)
    assert np.array_equal(pd[high].cpu().numpy(), small)
    q = bf16(rng, (1, 16, S, D))
    out, lse = s.attn_cache(gpu(q), pd, ints([high]), ints(lens))
    ref, rl = s.attn_cache(gpu(q), gpu(small), ints([[0, 1, 2]]), ints(lens))
    assert torch.equal(out, ref) and torch.equal(lse, rl)
    s.pages_copy(pd, ints([P - 1, -1]), ints([1, 2]))
    assert torch.equal(pd[1], pd[P - 1]) and not pd[2].any()


def test_same_bits_every_run_and_in_the_log_sum_exp_merge():
    """Runs repeat bit for bit; a recent part in bf16 joins by attn_merge."""
    rng = np.random.default_rng(8)
    s, H, D = steel(), 2, 128
    lens = np.array([3000, 500])
    P = 60
    pool, table = random_pool(rng, P, H, D, 122, 129), random_table(rng, lens, P)
    q = bf16(rng, (2, 8, 1, D))
    args = (gpu(q), gpu(pool), ints(table), ints(lens))
    a, al = s.attn_cache(*args)
    for _ in range(3):
        b, bl = s.attn_cache(*args)
        assert torch.equal(a, b) and torch.equal(al, bl)
    k, v = bf16(rng, (2, H, 40, D)), bf16(rng, (2, H, 40, D))
    o2, l2 = s.attn_fwd_lse(gpu(q), gpu(k), gpu(v), causal=False)
    out, lse = s.attn_merge(torch.stack((a, o2)), torch.stack((al, l2)))
    # the same keys in one softmax
    ck, cv = kv.load(pool, table, lens, 3000)
    for b, n in enumerate(lens):
        kk = np.concatenate((ck[b, :, :n], k[b].double().numpy()), 1)
        vv = np.concatenate((cv[b, :, :n], v[b].double().numpy()), 1)
        for h in range(8):
            sc = kk[h // 4] @ q[b, h, 0].double().numpy() * D ** -0.5
            w = np.exp(sc - sc.max())
            want = w @ vv[h // 4] / w.sum()
            near = 2.0 ** -7 * (w @ np.abs(vv[h // 4]) / w.sum())
            assert (np.abs(out[b, h, 0].cpu().double().numpy() - want) <= near).all()


# ---- pages ----

def random_rows(rng, B, M, P, share=True):
    """A page table with shared pages and its counts."""
    lens = rng.integers(0, 64 * M - 70, B)
    lens[rng.random(B) < 0.2] = 0
    free = list(rng.permutation(P))
    table = np.full((B, M), -1, np.int32)
    for b in range(B):
        n = -(-int(lens[b]) // 64)
        src = rng.integers(0, b) if share and b and rng.random() < 0.5 else None
        if src is not None:
            lens[b] = lens[src]
            table[b] = table[src]
        else:
            if len(free) < n:
                lens[b], n = 0, 0
            for j in range(n):
                table[b, j] = free.pop()
    refs = np.zeros(P, np.int32)
    for b in range(B):
        for p in kv.held(table, lens, b):
            refs[p] += 1
    return table, lens.astype(np.int32), refs


@pytest.mark.parametrize("B_in,B_out,M,P", [(1, 1, 3, 5), (4, 4, 9, 40), (7, 30, 20, 90), (64, 5, 33, 1500),
                                            (300, 300, 4, 900)])
def test_fork(B_in, B_out, M, P):
    rng = np.random.default_rng(B_in)
    table, lens, refs = random_rows(rng, B_in, M, P)
    parent = rng.integers(-2, B_in + 2, B_out).astype(np.int32)
    s, rd = steel(), ints(refs)
    t, l = s.pages_fork(ints(table), ints(lens), rd, ints(parent))
    wt, wl, wr = kv.fork(table, lens, refs, parent)
    assert np.array_equal(t.cpu().numpy(), wt) and np.array_equal(l.cpu().numpy(), wl)
    assert np.array_equal(rd.cpu().numpy(), wr)


@pytest.mark.parametrize("B,M,P,most", [(1, 4, 6, 1), (5, 9, 60, 3), (40, 20, 900, 65), (200, 5, 500, 1),
                                        (1500, 4, 6000, 70), (3, 40, 9000, 800), (16, 30, 100, 200), (20, 30, 65536, 200),
                                        (20, 30, 70001, 200), (1024, 3, 4000, 2), (1025, 3, 4000, 2)])
@pytest.mark.parametrize("seed", [0, 1])
def test_grow(B, M, P, most, seed):
    rng = np.random.default_rng(B + 1000 * seed)
    table, lens, refs = random_rows(rng, B, M, P)
    new = rng.integers(-1, most + 1, B).astype(np.int32)
    s = steel()
    t, l, r = ints(table), ints(lens), ints(refs)
    src, dst, left = s.pages_grow(t, l, r, ints(new))
    wt, wl, wr, ws, wd, wleft = kv.grow(table, lens, refs, new)
    say(f"[cache] grow B={B} P={P}: left {int(left)}")
    assert int(left) == wleft
    for got, want in ((t, wt), (l, wl), (r, wr), (src, ws), (dst, wd)):
        assert np.array_equal(got.cpu().numpy(), want)


def test_grow_refuses_as_a_whole():
    """One page too few, and a row too narrow: nothing changes."""
    s = steel()
    table, lens, refs = np.array([[0, -1], [1, -1]]), [64, 64], [1, 1, 0]
    for new, left in (([1, 1], -1), ([65, 0], -2 ** 31), ([1, 0], 0), ([0, 0], 1)):
        t, l, r = ints(table), ints(lens), ints(refs)
        src, dst, free = s.pages_grow(t, l, r, ints(new))
        assert int(free) == left
        if left < 0:
            assert t.cpu().tolist() == table.tolist() and l.cpu().tolist() == lens
            assert r.cpu().tolist() == refs and src.tolist() == dst.tolist() == [-1, -1]


@pytest.mark.parametrize("layers,P,H,D,n", [(1, 5, 1, 64, 1), (3, 40, 2, 128, 11), (2, 300, 8, 128, 77)])
def test_copy(layers, P, H, D, n):
    rng = np.random.default_rng(n)
    pool = rng.integers(0, 256, (layers, P, H, 68 * D), dtype=np.uint8)
    ids = rng.permutation(P)
    src, dst = rng.choice(ids[:P // 2 + 1], n), np.resize(ids[P // 2 + 1:], n)
    src[dst == -1] = -1
    if n > 3:
        src[1], dst[2], src[3] = -1, -1, P
        dst[0] = src[0]  # onto itself
    live = {int(d): int(x) for x, d in zip(src, dst) if 0 <= x < P and 0 <= d < P}
    pd = gpu(pool) if layers > 1 else gpu(pool[0])
    steel().pages_copy(pd, ints(src), ints(dst))
    want = pool.copy()
    for d, x in live.items():
        want[:, d] = pool[:, x]
    assert np.array_equal(pd.cpu().numpy().reshape(want.shape), want)


@pytest.mark.parametrize("layers,B,M,P", [(1, 1, 2, 3), (2, 5, 9, 70), (1, 30, 30, 1000), (1, 40, 200, 9000),
                                          (1, 3, 2, 4096), (1, 300, 20, 12289), (1, 200, 300, 65536),
                                          (1, 200, 300, 70003)])
@pytest.mark.parametrize("crowded", [False, True])
def test_compact(layers, B, M, P, crowded):
    rng = np.random.default_rng(P + crowded)
    table, lens, refs = random_rows(rng, B, M, P)
    if crowded:  # pages that no row of this table holds, a few of them behind the live ones
        refs[rng.random(P) < 0.5] += 1
    pool = rng.integers(0, 256, (layers, P, 1, 48), dtype=np.uint8)
    pd, t, r = gpu(pool), ints(table), ints(refs)
    live = steel().pages_compact(pd, t, ints(lens), r)
    wp, wt, wr, wl = kv.compact(pool.reshape(layers, P, 48), table, lens, refs)
    assert int(live) == wl
    assert np.array_equal(t.cpu().numpy(), wt) and np.array_equal(r.cpu().numpy(), wr)
    held = np.flatnonzero(wr > 0)
    assert np.array_equal(pd.cpu().numpy().reshape(wp.shape)[:, held], wp[:, held])


def test_compact_of_an_empty_and_a_full_pool():
    s = steel()
    for refs in ([0] * 9, [1] * 9):
        pool = torch.arange(9 * 16, dtype=torch.uint8, device=DEV).view(9, 1, 16)
        t, r, before = ints([[0, 8]]), ints(refs), pool.clone()
        live = s.pages_compact(pool, t, ints([128 * refs[0]]), r)
        assert int(live) == sum(refs) and torch.equal(pool, before) and t.tolist() == [[0, 8]]


# ---- together ----

class Beams:
    """The same search twice: on the GPU and in the model."""

    def __init__(self, layers, B, M, P, H, D, seed):
        self.rng = np.random.default_rng(seed)
        self.layers, self.H, self.D, self.B = layers, H, D, B
        self.pool = np.zeros((layers, P, H, 68 * D), np.uint8)
        self.table, self.lens = np.full((B, M), -1, np.int32), np.zeros(B, np.int32)
        self.refs = np.zeros(P, np.int32)
        self.g = [gpu(self.pool), ints(self.table), ints(self.lens), ints(self.refs)]

    def step(self, s, S, new, Hq, parent=None):
        pool, t, l, r = self.g
        if parent is not None:
            t, l = s.pages_fork(t, l, r, ints(parent))
            self.table, self.lens, self.refs = kv.fork(self.table, self.lens, self.refs, parent)
        nd = ints(new)
        src, dst, left = s.pages_grow(t, l, r, nd)
        s.pages_copy(pool, src, dst)
        self.table, self.lens, self.refs, ws, wd, wleft = kv.grow(self.table, self.lens, self.refs, new)
        for a, b in zip(ws, wd):
            if a >= 0:
                self.pool[:, b] = self.pool[:, a]
        assert int(left) == wleft >= 0
        shape = (self.B, self.H, S, self.D)
        for layer in range(self.layers):
            k, v = bf16(self.rng, shape), bf16(self.rng, shape)
            q = bf16(self.rng, (self.B, Hq, S, self.D))
            s.cache_append(gpu(k), gpu(v), pool[layer], t, l, new=nd)
            out, lse = s.attn_cache(gpu(q), pool[layer], t, l, new=nd)
            kv.append(k.double().numpy(), v.double().numpy(), self.pool[layer], self.table, self.lens, new)
            wo, wl = kv.attention(q.double().numpy(), self.pool[layer], self.table, self.lens,
                                  self.D ** -0.5, new=new)
            # weights in bf16 (2^-8 of sum p |v| <= 2^-8 max |v|) and fp32 sums
            bound = 2.0 ** -8 * 1.01 * 8
            assert np.abs(out.cpu().double().numpy() - wo).max() <= bound
            fin = np.isfinite(wl)
            assert np.array_equal(np.isfinite(lse.cpu().numpy()), fin)
            assert np.abs(lse.cpu().double().numpy()[fin] - wl[fin]).max(initial=0) <= 1e-4
        self.g = [pool, t, l, r]

    def same(self):
        pool, t, l, r = self.g
        assert np.array_equal(t.cpu().numpy(), self.table) and np.array_equal(l.cpu().numpy(), self.lens)
        assert np.array_equal(r.cpu().numpy(), self.refs)
        assert np.array_equal(pool.cpu().numpy(), self.pool)


def test_beam_search_from_prompt_to_compaction():
    """Prompts of unequal lengths, forks, single tokens, drafts, ended beams, compaction, and on."""
    s = steel()
    x = Beams(2, 4, 8, 40, 2, 64, 5)
    x.step(s, 70, [70, 3, 64, 0], 4)
    x.step(s, 1, [1, 1, 1, 1], 4, parent=[0, 0, 2, 0])
    x.step(s, 1, [1, 0, 1, 1], 4, parent=[1, 0, 0, 3])
    x.step(s, 5, [5, 2, 1, 5], 4, parent=[3, 3, -1, 1])
    x.same()
    live = s.pages_compact(x.g[0], x.g[1], x.g[2], x.g[3])
    pool, x.table, x.refs, n = kv.compact(x.pool.reshape(2, 40, -1), x.table, x.lens, x.refs)
    x.pool = pool.reshape(x.pool.shape)
    assert int(live) == n
    x.same()
    x.step(s, 1, [1, 1, 1, 1], 4, parent=[0, 0, 1, 1])
    x.same()


def test_cached_prefix_through_the_dense_call():
    """What cache_load gives, attn_fwd_lse takes: the same attention from either."""
    rng = np.random.default_rng(1)
    s, H, D, n = steel(), 2, 128, 500
    pool, table = random_pool(rng, 9, H, D, 122, 129), random_table(rng, [n], 9)
    q = gpu(bf16(rng, (1, 8, 100, D)))
    args = (gpu(pool), ints(table), ints([n]))
    a, al = s.attn_cache(q, *args)
    k, v = s.cache_load(*args, n)
    b, bl = s.attn_fwd_lse(q, k, v)
    spread = float(v.abs().max())
    assert float((a - b).abs().max()) <= 2 * 2.0 ** -8 * 1.1 * spread
    assert float((al - bl).abs().max()) <= 2.0 ** -7


# ---- streams and graphs ----

def test_a_step_captured_into_a_graph():
    """Grow, copy, append and attend as one graph, replayed with eager work between: the
    lengths advance on the device."""
    s, H, D, B = steel(), 2, 128, 3
    rng = np.random.default_rng(2)
    lens = np.array([62, 130, 5], np.int32)
    pool, table = random_pool(rng, 30, H, D, 122, 129), random_table(rng, lens, 30, extra=4)
    refs = np.zeros(30, np.int32)
    refs[table[table >= 0]] = 1

    def state():
        return [gpu(pool), ints(table), ints(lens), ints(refs)]
    k, v, q, new = (gpu(bf16(rng, (B, H, 1, D))), gpu(bf16(rng, (B, H, 1, D))),
                    gpu(bf16(rng, (B, 8, 1, D))), ints([1, 1, 1]))

    def step(st):
        src, dst, _ = s.pages_grow(st[1], st[2], st[3], new)
        s.pages_copy(st[0], src, dst)
        s.cache_append(k, v, st[0], st[1], st[2], new=new)
        return s.attn_cache(q, *st[:3], new=new)

    eager, held = state(), state()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(state())
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = step(held)
    for i in range(5):
        k.copy_(gpu(bf16(rng, (B, H, 1, D))))
        graph.replay()
        want, wl = step(eager)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, wl), f"replay {i}"
        assert all(torch.equal(x, y) for x, y in zip(held, eager))
    assert held[2].tolist() == [67, 135, 10]


def test_reordering_and_compaction_captured_into_a_graph():
    """Fork, compaction, read-back and attention (long lists under a mask, a chunk) as one graph,
    replayed over states that are put back, with eager work between."""
    s, H, D, B, P = steel(), 2, 64, 3, 200
    rng = np.random.default_rng(3)
    lens = np.array([3000, 64, 2100], np.int32)
    pool, table = random_pool(rng, P, H, D, 122, 129), random_table(rng, lens, P)
    refs = np.zeros(P, np.int32)
    refs[table[table >= 0]] = 1
    M = table.shape[1]
    mask = gpu((rng.random((B, H, M)) < 0.6).astype(np.uint8))
    q1, qc = gpu(bf16(rng, (B, 4, 1, D))), gpu(bf16(rng, (B, 4, 50, D)))
    start = [gpu(pool), ints(table), ints(lens), ints(refs)]
    parent = ints([2, 0, 2])

    def step(st):
        t, l = s.pages_fork(*st[1:], parent)
        live = s.pages_compact(st[0], t, l, st[3])
        k, v = s.cache_load(st[0], t, l, 100)
        return (t, l, live, k, v, *s.attn_cache(q1, st[0], t, l, block_mask=mask),
                *s.attn_cache(q1, st[0], t, l), *s.attn_cache(qc, st[0], t, l))

    held = [x.clone() for x in start]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step([x.clone() for x in start])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(held)
    for i, order in enumerate(([2, 0, 2], [1, 1, 0], [-1, 2, 2], [0, 1, 2])):
        parent.copy_(ints(order))
        for x, y in zip(held, start):
            x.copy_(y)
        q1.copy_(gpu(bf16(rng, q1.shape)))
        graph.replay()
        eager = [x.clone() for x in start]
        want = step(eager)
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b), f"replay {i}"
        live = int(outs[2])
        assert torch.equal(held[3], eager[3]) and torch.equal(held[0][:live], eager[0][:live])
        ref = kv.fork(table, lens, refs, order)
        assert live == int((ref[2] > 0).sum())


def test_two_graphs_and_streams_do_not_share_anything():
    """Two captured calls replayed at one time on two streams, and calls by `stream=`."""
    s, D = steel(), 128
    rng = np.random.default_rng(4)
    sets = []
    for n in (4000, 2500):
        pool, table = random_pool(rng, 70, 2, D, 122, 129), random_table(rng, [n], 70)
        sets.append((gpu(bf16(rng, (1, 8, 1, D))), gpu(pool), ints(table), ints([n])))
    want = [s.attn_cache(*x) for x in sets]
    torch.cuda.synchronize()
    graphs, outs, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for x in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(s.attn_cache(*x))
        graphs.append(g)
    for _ in range(20):
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o[0], w[0]) and torch.equal(o[1], w[1])
    got = [[s.attn_cache(*x, stream=st) for x, st in zip(sets, streams)] for _ in range(10)]
    torch.cuda.synchronize()
    for pair in got:
        for o, w in zip(pair, want):
            assert torch.equal(o[0], w[0]) and torch.equal(o[1], w[1])


def test_binding_on_the_gpu_refuses():
    s = steel()
    pool, t, l = torch.zeros((4, 2, 68 * 64), dtype=torch.uint8, device=DEV), ints([[0, 1]]), ints([64])
    q = torch.zeros((1, 4, 1, 64), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(ValueError, match="page_table"):
        s.attn_cache(q, pool, t.long(), l)
    with pytest.raises(ValueError, match="lens"):
        s.attn_cache(q, pool, t, l.cpu())
    with pytest.raises(ValueError, match="block_mask"):
        s.attn_cache(q, pool, t, l, block_mask=torch.ones((1, 4, 2), dtype=torch.uint8, device=DEV))
    with pytest.raises(ValueError, match="q must be"):
        s.attn_cache(torch.zeros((1, 4, 1, 128), dtype=torch.bfloat16, device=DEV), pool, t, l)
    with pytest.raises(s.SteelError, match="multiple"):
        s.attn_cache(torch.zeros((1, 3, 1, 64), dtype=torch.bfloat16, device=DEV), pool, t, l)
    with pytest.raises(s.SteelError, match="window"):
        s.attn_cache(q, pool, t, l, sink_blocks=1)
    with pytest.raises(ValueError, match="k and v"):
        s.cache_append(q, q, pool, t, l)
    with pytest.raises(ValueError, match="new"):
        s.cache_append(q[:, :2], q[:, :2], pool, t, l, new=ints([1, 1]))
    with pytest.raises(ValueError, match="contiguous uint8"):
        s.cache_load(pool.transpose(0, 1), t, l, 1)
    with pytest.raises(s.SteelError, match=">= 1"):
        s.cache_load(pool, t, l, 0)
    with pytest.raises(ValueError, match="out must be"):
        s.attn_cache(q, pool, t, l, out=torch.empty((1, 4, 1, 64), dtype=torch.bfloat16, device=DEV))
    with pytest.raises(ValueError, match="refs"):
        s.pages_compact(pool, t, l, ints([1, 1, 1]))
