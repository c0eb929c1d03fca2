"""Float64 model of the paged 4-bit key/value cache.

Written from the format's definition, one value and one page at a time where that is
the plainest way: ``encode`` picks, for 32 channels, the smallest power of two that
brings the largest magnitude to 6 or less (exponent -125 .. 125) and the nearest of the
8 magnitudes (ties to the even code); ``decode`` looks the codes up; ``attention`` forms
every score of a row, masks it and takes a plain softmax; ``fork``, ``grow`` and
``compact`` walk the rows of the page table in order.
"""
from __future__ import annotations

import math

import numpy as np

PAGE = 64
MAGNITUDES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)


def scale_exponent(amax: float) -> int:
    e = -125
    while e < 125 and amax > 6.0 * 2.0 ** e:
        e += 1
    return e


def encode(x):
    """x float64 [D] -> (codes uint8 [D], scale bytes uint8 [D / 32])."""
    x = np.asarray(x, dtype=np.float64)
    if not np.isfinite(x).all():
        return np.zeros(x.size, np.uint8), np.full(x.size // 32, 255, np.uint8)
    codes, scales = np.zeros(x.size, np.uint8), np.zeros(x.size // 32, np.uint8)
    for g in range(x.size // 32):
        part = x[32 * g:32 * g + 32]
        e = scale_exponent(np.abs(part).max())
        scales[g] = e + 127
        for i, v in enumerate(part):
            y = abs(v) / 2.0 ** e
            d = np.abs(MAGNITUDES - y)
            near = np.flatnonzero(d == d.min())
            code = near[0] if near.size == 1 or near[0] % 2 == 0 else near[1]
            codes[32 * g + i] = code + (8 if math.copysign(1.0, v) < 0 else 0)
    return codes, scales


def decode(codes, scales):
    """codes [..., D], scales [..., D / 32] -> float64 [..., D]."""
    mag = MAGNITUDES[codes & 7]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return np.where(codes & 8, -mag, mag) * np.repeat(s, 32, axis=-1)


def pack(pages, page, head, token, which, codes, scales):
    """Store one token's vector (which: 0 key, 1 value) into pages [P, Hkv, 68 D]."""
    D = codes.size
    rec = pages[page, head]
    at = 32 * D * which + token * (D // 2)
    rec[at:at + D // 2] = codes[0::2] | (codes[1::2] << 4)
    at = 64 * D + 2 * D * which + token * (D // 32)
    rec[at:at + D // 32] = scales


def unpack(pages, page, head, which):
    """float64 [64, D]: a page's keys or values of one head."""
    D = pages.shape[2] // 68
    rec = pages[page, head]
    by = rec[32 * D * which:32 * D * (which + 1)].reshape(PAGE, D // 2)
    codes = np.stack((by & 15, by >> 4), axis=-1).reshape(PAGE, D)
    at = 64 * D + 2 * D * which
    return decode(codes, rec[at:at + 2 * D].reshape(PAGE, D // 32))


def count(new, b, S):
    return S if new is None else min(max(int(new[b]), 0), S)


def append(k, v, pages, table, lens, new=None):
    """k, v float64 [B, Hkv, S, D]; pages uint8 [P, Hkv, 68 D] is updated."""
    B, H, S, _ = k.shape
    for b in range(B):
        n = count(new, b, S)
        for i in range(n):
            pos = int(lens[b]) - n + i
            if pos < 0 or pos // PAGE >= table.shape[1]:
                continue
            page = int(table[b, pos // PAGE])
            if not 0 <= page < pages.shape[0]:
                continue
            for h in range(H):
                pack(pages, page, h, pos % PAGE, 0, *encode(k[b, h, i]))
                pack(pages, page, h, pos % PAGE, 1, *encode(v[b, h, i]))


def load(pages, table, lens, S, start=None):
    """float64 keys and values [B, Hkv, S, D], 0 where there is no token."""
    B, H, D = len(lens), pages.shape[1], pages.shape[2] // 68
    out = np.zeros((2, B, H, S, D))
    for b in range(B):
        for i in range(S):
            pos = (0 if start is None else int(start[b])) + i
            if pos < 0 or pos >= lens[b] or pos // PAGE >= table.shape[1]:
                continue
            page = int(table[b, pos // PAGE])
            if 0 <= page < pages.shape[0]:
                for h in range(H):
                    for w in (0, 1):
                        out[w, b, h, i] = unpack(pages, page, h, w)[pos % PAGE]
    return out[0], out[1]


def attention(q, pages, table, lens, scale, *, new=None, causal=True, window_blocks=0,
              sink_blocks=0, block_mask=None):
    """q float64 [B, Hq, S_q, D] -> (out [B, Hq, S_q, D], lse [B, Hq, S_q])."""
    B, Hq, S, D = q.shape
    P, H, M = pages.shape[0], pages.shape[1], table.shape[1]
    out, lse = np.zeros((B, Hq, S, D)), np.full((B, Hq, S), -np.inf)
    for b in range(B):
        n = count(new, b, S)
        keys = min(max(int(lens[b]), 0), PAGE * M)
        j = np.arange(keys)
        for h in range(H):
            k, v = np.zeros((keys, D)), np.zeros((keys, D))
            there = np.zeros(keys, dtype=bool)
            for kb in range(-(-keys // PAGE)):
                page = int(table[b, kb])
                if 0 <= page < P and (block_mask is None or block_mask[b, h, kb]):
                    at = slice(kb * PAGE, min(keys, kb * PAGE + PAGE))
                    k[at] = unpack(pages, page, h, 0)[:at.stop - at.start]
                    v[at] = unpack(pages, page, h, 1)[:at.stop - at.start]
                    there[at] = True
            p = int(lens[b]) - n + np.arange(n)[:, None]
            see = there & (p >= 0)
            if causal:
                see &= j <= p
            if window_blocks > 0:
                kb, qb = j // PAGE, p // PAGE
                see &= ((kb <= qb) & (kb > qb - window_blocks)) | (kb < sink_blocks)
            rows = np.flatnonzero(see.any(axis=1))
            if rows.size == 0:
                continue
            see = see[rows]
            for hq in range(h * (Hq // H), (h + 1) * (Hq // H)):
                s = np.where(see, q[b, hq, rows] @ k.T * scale, -np.inf)
                top = s.max(axis=1, keepdims=True)
                w = np.exp(s - top)
                tot = w.sum(axis=1, keepdims=True)
                bad = np.isnan(v).any(axis=1)
                o = w @ np.where(bad[:, None], 0.0, v) / tot
                o[(see & bad).any(axis=1)] = np.nan  # a row that sees a NaN value, and no other
                out[b, hq, rows] = o
                lse[b, hq, rows] = (top + np.log(tot))[:, 0]
    return out, lse


def held(table, lens, b):
    return [int(x) for x in table[b, :min(-(-max(int(lens[b]), 0) // PAGE), table.shape[1])]]


def fork(table, lens, refs, parent):
    """(table, lens, refs) of the new rows."""
    refs = np.array(refs, dtype=np.int32)
    M, P = table.shape[1], len(refs)
    for b in range(len(lens)):
        for p in held(table, lens, b):
            if 0 <= p < P:
                refs[p] -= 1
    out, outl = np.full((len(parent), M), -1, np.int32), np.zeros(len(parent), np.int32)
    for b, src in enumerate(parent):
        if 0 <= src < len(lens):
            row = held(table, lens, src)
            out[b, :len(row)] = row
            outl[b] = max(int(lens[src]), 0)
            for p in row:
                if 0 <= p < P:
                    refs[p] += 1
    return out, outl, refs


def grow(table, lens, refs, new):
    """(table, lens, refs, src, dst, left)."""
    B, M = table.shape
    P = len(refs)
    # pages behind the pool stand in for missing ones, to count them as if they were there
    t, l, r = np.array(table), np.array(lens), np.concatenate((refs, np.zeros(B * (M + 1), np.int32)))
    src, dst = np.full(B, -1, np.int32), np.full(B, -1, np.int32)
    free = [p for p in range(len(r)) if r[p] == 0]
    there = sum(p < P for p in free)
    used = 0
    narrow = False

    def take():
        nonlocal used
        used += 1
        return free[used - 1]

    for b in range(B):
        n, have = max(int(new[b]), 0), max(int(l[b]), 0)
        if have + n > PAGE * M:
            narrow = True
            continue
        last = -(-have // PAGE) - 1
        if n and have % PAGE and 0 <= t[b, last] < P and r[t[b, last]] > 1:
            p = take()
            src[b], dst[b] = t[b, last], p
            r[t[b, last]] -= 1
            r[p] += 1
            t[b, last] = p
        for kb in range(last + 1, -(-(have + n) // PAGE)):
            p = take()
            t[b, kb] = p
            r[p] += 1
        l[b] = have + n
    left = there - used
    if narrow or left < 0:
        none = np.full(B, -1, np.int32)
        return (np.array(table), np.array(lens), np.array(refs), none, none.copy(),
                -2 ** 31 if narrow else left)
    return t, l, r[:P], src, dst, left


def compact(pages, table, lens, refs):
    """(pages, table, refs, live); pages [layers, P, bytes]."""
    pages, table, refs = np.array(pages), np.array(table), np.array(refs)
    live = int((refs > 0).sum())
    holes = [p for p in range(live) if refs[p] <= 0]
    movers = [p for p in range(live, len(refs)) if refs[p] > 0]
    to = dict(zip(movers, holes))
    for p, h in to.items():
        pages[:, h] = pages[:, p]
        refs[h], refs[p] = refs[p], 0
    for b in range(len(lens)):
        for j, p in enumerate(held(table, lens, b)):
            table[b, j] = to.get(p, p)
    return pages, table, refs, live
