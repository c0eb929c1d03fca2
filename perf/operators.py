"""The operators of the paged 4-bit key/value cache: their cases, their plain forms and
their definitions in 64 bits.

A cache is a pool of pages of 64 tokens.  The record of a page and a key/value head is
68 * D bytes: key codes [64][D/2] (low nibble: even channel), value codes [64][D/2], key
scales [64][D/32], value scales [64][D/32].  A code is an E2M1 number (0 .5 1 1.5 2 3 4 6
and a sign), a scale byte b stands for 2^(b - 127): the smallest power of two that brings
the largest magnitude of its 32 channels to 6 or less.  A token's vector with a
non-finite element has scale bytes of 255, which stand for NaN.  A sequence is a row of
page numbers and a length; ``refs`` counts the rows that hold a page.

Kinds:
  attn     attention of new queries over the cached keys and values
  append   new keys and values written into the cache and read back
  step     beams reordered (rows forked or freed), grown by new tokens, and the shared
           pages that are written next copied
  compact  the live pages moved to the front of the pool
"""
import math
import random

import torch

own = False

BLK = 64


def _attn(name, B, Hq, Hkv, D, Sq, lo, hi, win=0, sink=0, keep=0.0, causal=True, mix=0):
    c = {"kind": "attn", "B": B, "Hq": Hq, "Hkv": Hkv, "D": D, "Sq": Sq, "lo": lo, "hi": hi,
         "win": win, "sink": sink, "keep": keep, "causal": causal, "mix": mix}
    return {"name": name, **c} if name else c


def _append(name, B, Hkv, D, S, lo, hi, ragged, mix=0):
    c = {"kind": "append", "B": B, "Hkv": Hkv, "D": D, "S": S, "lo": lo, "hi": hi,
         "ragged": ragged, "mix": mix}
    return {"name": name, **c} if name else c


def _step(name, B, Hkv, D, layers, new, lo, hi, mix=0):
    c = {"kind": "step", "B": B, "Hkv": Hkv, "D": D, "layers": layers, "new": new, "lo": lo,
         "hi": hi, "mix": mix}
    return {"name": name, **c} if name else c


def _compact(name, B, Hkv, D, layers, lo, hi, fill, mix=0):
    c = {"kind": "compact", "B": B, "Hkv": Hkv, "D": D, "layers": layers, "lo": lo, "hi": hi,
         "fill": fill, "mix": mix}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one token of one short sequence, BERT-sized heads: what a call costs beyond its work
        _attn("token_b1_mha12_s512_d64", 1, 12, 12, 64, 1, 512, 512),
        # one decoding step of a small batch, grouped heads
        _attn("token_b4_gqa32x8_s8000_d128", 4, 32, 8, 128, 1, 8000, 8000),
        # one decoding step of a full server: 64 sequences of very unequal lengths
        _attn("token_b64_gqa32x8_ragged_d128", 64, 32, 8, 128, 1, 70, 32768, mix=1),
        # four drafted tokens checked at once against long windowed sequences
        _attn("draft4_b8_mha24_window_d64", 8, 24, 24, 64, 4, 9000, 16384, win=16, sink=1, mix=2),
        # one decoding step that reads a tenth of the pages of each key/value head
        _attn("token_b8_gqa32x8_s32768_keep10_d128", 8, 32, 8, 128, 1, 32768, 32768, keep=0.1),
        # a chunk of a prompt against the cache that holds what came before and the chunk
        _attn("chunk1000_gqa32x8_s12000_d128", 1, 32, 8, 128, 1000, 12000, 12000),
        # the keys and values of one decoding step, one layer
        _append("append_token_b64_h8_d128", 64, 8, 128, 1, 70, 32768, False, mix=1),
        # prompts of unequal lengths in one padded batch
        _append("append_prompt_b4_h8_d128", 4, 8, 128, 8192, 1, 8192, True, mix=3),
        # a beam search of one short sequence
        _step("step_b4_h12_s500_d64", 4, 12, 64, 1, 1, 450, 500, mix=9),
        # many beams, pages of two layers
        _step("step_b64_h8_ragged_d128", 64, 8, 128, 2, 1, 70, 4096, mix=5),
        # a small pool after a few sequences ended
        _compact("compact_b4_h12_d64", 4, 12, 64, 1, 100, 1000, 0.5, mix=6),
        # a pool of two layers, two thirds in use
        _compact("compact_b32_h8_d128", 32, 8, 128, 2, 500, 8192, 0.67, mix=7),
    ]


_HEADS = {64: [(1, 1), (8, 8), (12, 12), (24, 24), (32, 8), (32, 4)],
          128: [(8, 2), (16, 4), (32, 8), (32, 32), (24, 6), (16, 8), (20, 4)]}


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw(rng):
    kind = rng.choice(["attn", "attn", "attn", "chunk", "append", "step", "compact"])
    D = rng.choice([64, 128])
    Hq, Hkv = rng.choice(_HEADS[D])
    mix = rng.randrange(1 << 30)
    B = _log(rng, 1, 64)
    if kind == "attn":
        Sq = rng.choice([1, 1, 1, 2, 4, 7])
        hi = _log(rng, 64, 32768)
        lo = hi if rng.random() < 0.4 else max(Sq, _log(rng, 1, hi))
        win = rng.choice([0, 0, 4, 16])
        keep = 0.0 if win else rng.choice([0.0, 0.0, 0.1, 0.25])
        return _attn("", B, Hq, Hkv, D, Sq, lo, hi, win, rng.choice([0, 1, 2]) if win else 0,
                     keep, rng.random() < 0.9, mix)
    if kind == "chunk":
        Sq = _log(rng, 17, 2000)
        hi = Sq + _log(rng, 1, 12000)
        win = rng.choice([0, 0, 8])
        return _attn("", rng.choice([1, 1, 2, 4]), Hq, Hkv, D, Sq, rng.choice([Sq, hi]), hi, win,
                     rng.choice([0, 1]) if win else 0, 0.0, True, mix)
    if kind == "append":
        S = rng.choice([1, 1, 4, _log(rng, 16, 8192)])
        return _append("", B if S < 16 else rng.choice([1, 2, 4]), Hkv, D, S, S,
                       S + _log(rng, 1, 16384), rng.random() < 0.5, mix)
    if kind == "step":
        hi = _log(rng, 64, 8192)
        return _step("", B, Hkv, D, rng.choice([1, 2]), rng.choice([1, 1, 4, 70]),
                     _log(rng, 1, hi), hi, mix)
    hi = _log(rng, 64, 8192)
    return _compact("", B, Hkv, D, rng.choice([1, 2]), _log(rng, 1, hi), hi,
                    rng.choice([0.3, 0.5, 0.9]), mix)


def draw(rng):
    most = [work(c) for c in listed()]
    flops, nbytes = max(w["flops"] for w in most), max(w["bytes"] for w in most)
    while True:
        c = _draw(rng)
        w = work(c)
        if w["flops"] <= flops and w["bytes"] <= nbytes and _pool_bytes(c) <= 1 << 31:
            return c


# ---- what a case's sequences are ----

def _pages(n):
    return -(-n // BLK)


def _lens(case):
    """Lengths, log-uniform between lo and hi with one sequence of each."""
    rng = random.Random(case["mix"])
    lens = [_log(rng, case["lo"], case["hi"]) for _ in range(case["B"])]
    if len(lens) > 1:
        lens[rng.randrange(len(lens))] = case["lo"]
    lens[0] = case["hi"]
    return lens


def _layout(case):
    """(lengths, columns of the page table, pages of the pool) before the call."""
    lens = _lens(case)
    held = sum(map(_pages, lens))
    if case["kind"] == "step":
        return lens, _pages(case["hi"] + case["new"]) + 1, 2 * held + case["B"] * (3 + _pages(case["new"]))
    if case["kind"] == "compact":
        return lens, _pages(case["hi"]) + 1, max(held + 1, int(held / case["fill"]))
    return lens, _pages(case["hi"]) + 1, held + 3


def _pool_bytes(case):
    return case.get("layers", 1) * _layout(case)[2] * case["Hkv"] * 68 * case["D"]


def _new(case):
    """Tokens that each sequence gets."""
    rng = random.Random(case["mix"] + 1)
    lens = _lens(case)
    if case["kind"] == "append":
        most = [min(n, case["S"]) for n in lens]
        return [m if not case["ragged"] else rng.choice([m, rng.randint(0, m)]) for m in most]
    return [rng.choice([case["new"], case["new"], 0]) if case["new"] > 1 else 1 for _ in lens]


def _parents(case):
    """For each beam the one that it continues: some twice, some ended, most their own."""
    rng = random.Random(case["mix"] + 2)
    B = case["B"]
    return [rng.choice([b, b, rng.randrange(B), rng.randrange(B), -1 if B > 2 else b])
            for b in range(B)]


def _moves(case):
    lens, _, P = _layout(case)
    live = sum(map(_pages, lens))
    return min(live, P - live) // 2


def _live_pages(case, pos):
    """Pages that a query at pos reads, window and sinks applied."""
    qb = pos // BLK
    return {kb for kb in range(qb + 1) if kb > qb - case["win"] or kb < case["sink"]}


# ---- inputs ----

_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _quantise(x):
    """x [..., D] -> (codes uint8 [..., D/2], scales uint8 [..., D/32])."""
    x = x.float()
    D = x.shape[-1]
    bad = ~torch.isfinite(x).all(-1, keepdim=True)
    g = torch.where(bad, 0.0, x).unflatten(-1, (D // 32, 32))
    top, ex = torch.frexp(g.abs().amax(-1))  # top * 2^ex, top in [0.5, 1)
    ex = torch.where(top > 0.75, ex - 2, ex - 3).clamp(-125, 125)
    y = torch.ldexp(g, -ex[..., None])
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = (torch.round(a / step) * step).clamp(max=6.0)
    code = (a > 0.25).to(torch.uint8)  # codes 1 .. 7: thresholds between neighbours
    for t in (0.75, 1.25, 1.75, 2.5, 3.5, 5.0):
        code += a > t
    code += torch.signbit(y).to(torch.uint8) * 8
    code = torch.where(bad[..., None], 0, code).flatten(-2)
    scale = torch.where(bad, 255, ex + 127).to(torch.uint8)
    return code[..., 0::2] + 16 * code[..., 1::2], scale


def _values(codes, scales, dtype=torch.float32):
    """What codes [..., D/2] and scales [..., D/32] stand for: [..., D]."""
    lut = torch.tensor(_E2M1 + tuple(-x for x in _E2M1), dtype=dtype, device=codes.device)
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    s = torch.exp2(scales.to(torch.int32).to(dtype) - 127)
    s = torch.where(scales == 255, math.nan, s)
    v = lut[c.to(torch.int32)].unflatten(-1, (scales.shape[-1], 32)) * s[..., None]
    return v.flatten(-2)


def _fields(rec, D):
    """Views of records [..., 68 D]: key codes, value codes, key scales, value scales."""
    kc, vc, ks, vs = rec.split((32 * D, 32 * D, 2 * D, 2 * D), -1)
    return (kc.unflatten(-1, (BLK, D // 2)), vc.unflatten(-1, (BLK, D // 2)),
            ks.unflatten(-1, (BLK, D // 32)), vs.unflatten(-1, (BLK, D // 32)))


def _table(case, g, dev):
    """Page table: the sequences' pages at random places of the pool, -1 behind them."""
    lens, M, P = _layout(case)
    n = sum(map(_pages, lens))
    ids = torch.randperm(P, generator=g, device=dev)[:n]
    if case["kind"] == "compact":  # a fixed number of live pages behind the first n
        m = _moves(case)
        low = torch.randperm(n, generator=g, device=dev)[:n - m]
        high = n + torch.randperm(P - n, generator=g, device=dev)[:m]
        ids = torch.cat((low, high))[torch.randperm(n, generator=g, device=dev)]
    table = torch.full((len(lens), M), -1, dtype=torch.int32, device=dev)
    refs = torch.zeros(P, dtype=torch.int32, device=dev)
    refs[ids] = 1
    at = 0
    for b, l in enumerate(lens):
        table[b, :_pages(l)] = ids[at:at + _pages(l)]
        at += _pages(l)
    return table, refs


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed))
    lens, M, P = _layout(case)
    B, Hkv, D = case["B"], case["Hkv"], case["D"]
    table, refs = _table(case, g, dev)
    st = {"case": case, "lens_host": lens, "table": table, "refs": refs,
          "lens": torch.tensor(lens, dtype=torch.int32, device=dev)}
    if case["kind"] in ("step", "compact"):
        shape = (case["layers"], P, Hkv, 68 * D)
        st["pages"] = torch.randint(0, 256, shape, generator=g, device=dev, dtype=torch.uint8)
        if case["kind"] == "step":
            st["parent"] = torch.tensor(_parents(case), dtype=torch.int32, device=dev)
            st["new"] = torch.tensor(_new(case), dtype=torch.int32, device=dev)
        return st
    pages = torch.empty((P, Hkv, 68 * D), dtype=torch.uint8, device=dev)
    for p0 in range(0, P, 1024):  # tokens N(0,1), keys with a few larger channels
        n = min(1024, P - p0)
        amp = 1 + 3 * (torch.rand((1, Hkv, 1, D), generator=g, device=dev) < 0.03)
        fields = _fields(pages[p0:p0 + n], D)
        for i, a in ((0, amp), (1, 1.0)):
            x = torch.randn((n, Hkv, BLK, D), generator=g, device=dev) * a
            codes, scales = _quantise(x)
            fields[i].copy_(codes)
            fields[2 + i].copy_(scales)
    st["pages"] = pages
    if case["kind"] == "append":
        new = _new(case)
        shape = (B, Hkv, case["S"], D)
        st["k"] = torch.randn(shape, generator=g, device=dev).to(torch.bfloat16)
        st["v"] = torch.randn(shape, generator=g, device=dev).to(torch.bfloat16)
        st["new_host"] = new
        st["new"] = torch.tensor(new, dtype=torch.int32, device=dev)
        st["start"] = st["lens"] - st["new"]
        return st
    st["q"] = torch.randn((B, case["Hq"], case["Sq"], D), generator=g, device=dev).to(torch.bfloat16)
    st["scale"] = D ** -0.5
    st["mask"] = None
    if case["keep"]:
        m = torch.rand((B, Hkv, M), generator=g, device=dev) < case["keep"]
        m[torch.arange(B, device=dev), :, (st["lens"].long() - 1) // BLK] = True
        st["mask"] = m.to(torch.uint8)
    return st


# ---- one pass ----

def run(st):
    return (_OWN if own else _PLAIN)[st["case"]["kind"]](st)


def _own_attn(st):
    import paper_2607_09385_amd as steel
    case = st["case"]
    out, lse = steel.attn_cache(st["q"], st["pages"], st["table"], st["lens"],
                                block_mask=st["mask"], window_blocks=case["win"],
                                sink_blocks=case["sink"], scale=st["scale"],
                                causal=case["causal"], out_dtype=torch.bfloat16)
    return {"out": out, "lse": lse}


def _own_append(st):
    import paper_2607_09385_amd as steel
    steel.cache_append(st["k"], st["v"], st["pages"], st["table"], st["lens"], new=st["new"])
    k, v = steel.cache_load(st["pages"], st["table"], st["lens"], st["case"]["S"],
                            start=st["start"])
    return {"k": k, "v": v}


def _own_step(st):
    import paper_2607_09385_amd as steel
    refs = st["refs"].clone()
    table, lens = steel.pages_fork(st["table"], st["lens"], refs, st["parent"])
    src, dst, left = steel.pages_grow(table, lens, refs, st["new"])
    steel.pages_copy(st["pages"], src, dst)
    return {"table": table, "lens": lens, "refs": refs, "src": src, "dst": dst, "left": left,
            "pages": st["pages"]}


def _own_compact(st):
    import paper_2607_09385_amd as steel
    table, refs = st["table"].clone(), st["refs"].clone()
    live = steel.pages_compact(st["pages"], table, st["lens"], refs)
    return {"live": live, "table": table, "refs": refs, "pages": st["pages"]}


_OWN = {"attn": _own_attn, "append": _own_append, "step": _own_step, "compact": _own_compact}


# The plain forms.

def _visible(case, pos, n, dev):
    """[rows, n] truth values: which of the first n keys queries at pos see."""
    j = torch.arange(n, device=dev)
    vis = torch.ones((len(pos), n), dtype=torch.bool, device=dev)
    if case["causal"]:
        vis = j <= pos[:, None]
    if case["win"]:
        qb, kb = pos[:, None] // BLK, j // BLK
        vis = vis & (((kb <= qb) & (kb > qb - case["win"])) | (kb < case["sink"]))
    return vis & (pos[:, None] >= 0)


def _plain_attn(st):
    case, q = st["case"], st["q"]
    B, Hq, Sq, D = q.shape
    Hkv, G = case["Hkv"], Hq // case["Hkv"]
    out, lse = [], []
    for b in range(B):
        n = st["lens_host"][b]
        pos = torch.arange(n - Sq, n, device=q.device)
        f = _fields(st["pages"][st["table"][b, :_pages(n)].long()].transpose(0, 1), D)
        k = _values(f[0], f[2]).flatten(1, 2)[:, :n]
        v = _values(f[1], f[3]).flatten(1, 2)[:, :n]
        qb = q[b].float().reshape(Hkv, G * Sq, D)
        s = torch.bmm(qb, k.transpose(1, 2)).view(Hkv, G, Sq, n) * st["scale"]
        vis = _visible(case, pos, n, q.device)
        if st["mask"] is not None:
            m = st["mask"][b, :, :_pages(n)].bool().repeat_interleave(BLK, 1)[:, None, None, :n]
            vis = vis & m
        s = torch.where(vis, s, -math.inf)
        top = s.amax(-1, keepdim=True)
        top = torch.where(top == -math.inf, 0.0, top)
        p = torch.exp(s - top)
        tot = p.sum(-1, keepdim=True)
        o = torch.bmm(p.view(Hkv, G * Sq, n), v).view(Hkv, G, Sq, D)
        out.append((o / torch.where(tot > 0, tot, 1.0)).reshape(Hq, Sq, D))
        lse.append((top + torch.log(tot)).reshape(Hq, Sq))
    return {"out": torch.stack(out).to(torch.bfloat16), "lse": torch.stack(lse)}


def _plain_append(st):
    case, pages, table = st["case"], st["pages"], st["table"].long()
    D, S = case["D"], case["S"]
    at = st["start"].long()[:, None] + torch.arange(S, device=pages.device)  # [B, S]
    there = torch.arange(S, device=pages.device) < st["new"][:, None]
    page = table.gather(1, torch.where(there, at // BLK, 0))
    b, i = there.nonzero(as_tuple=True)
    pg, tok = page[b, i], at[b, i] % BLK
    fields = _fields(pages, D)
    out = {}
    for name, f in (("k", 0), ("v", 1)):
        codes, scales = _quantise(st[name].transpose(1, 2)[b, i])  # [tokens, Hkv, ..]
        fields[f][pg, :, tok] = codes
        fields[2 + f][pg, :, tok] = scales
        x = torch.zeros((case["B"], S, case["Hkv"], D), dtype=torch.bfloat16, device=pages.device)
        x[b, i] = _values(fields[f][pg, :, tok], fields[2 + f][pg, :, tok]).to(torch.bfloat16)
        out[name] = x.transpose(1, 2).contiguous()
    return out


def _count(table, lens, P):
    """Rows of the table that hold each page."""
    j = torch.arange(table.shape[1], device=table.device)
    held = j < (lens[:, None] + BLK - 1) // BLK
    n = torch.zeros(P + 1, dtype=torch.int32, device=table.device)
    n.index_add_(0, torch.where(held, table, P).flatten().long(),
                 torch.ones(table.numel(), dtype=torch.int32, device=table.device))
    return n[:P]


def _plain_step(st):
    P, B = st["refs"].numel(), st["table"].shape[0]
    parent, new = st["parent"].long(), st["new"].long()
    dev = parent.device
    # fork: rows of the parents, ended beams empty
    gone = parent < 0
    lens = torch.where(gone, 0, st["lens"][parent.clamp(min=0)])
    j = torch.arange(st["table"].shape[1], device=dev)
    held = j < ((lens + BLK - 1) // BLK)[:, None]
    table = torch.where(held, st["table"][parent.clamp(min=0)], -1)
    refs = st["refs"] + _count(table, lens, P) - _count(st["table"], st["lens"], P)
    # grow: which beams write into a page that others hold as well
    have, want = (lens + BLK - 1) // BLK, (lens + new + BLK - 1) // BLK
    last = table.gather(1, (have - 1).clamp(min=0)[:, None].long())[:, 0].long()
    wide = torch.where((new > 0) & (lens % BLK != 0), last, P)  # P: none
    r1 = torch.cat((refs, refs.new_zeros(1)))
    writers = torch.zeros(P + 1, dtype=torch.int32, device=dev)
    writers.index_add_(0, wide, torch.ones(B, dtype=torch.int32, device=dev))
    top = torch.full((P + 1,), -1, dtype=torch.int64, device=dev)
    top.scatter_reduce_(0, wide, torch.arange(B, device=dev), "amax")
    alone = (writers[wide] == r1[wide]) & (top[wide] == torch.arange(B, device=dev))
    cow = (wide < P) & (r1[wide] > 1) & ~alone
    need = want - have + cow
    off = need.cumsum(0) - need
    free = torch.sort((refs != 0).to(torch.int32), stable=True).indices
    left = ((refs == 0).sum() - need.sum()).to(torch.int32).reshape(1)
    fits = left[0] >= 0
    rank = (off + cow)[:, None] + j - have[:, None]
    fresh = (j >= have[:, None]) & (j < want[:, None]) & fits
    first = torch.where(cow & fits, off, 0)
    copy = cow & fits
    grown = torch.where(fresh, free[rank.clamp(0, P - 1)].to(torch.int32), table)
    at_last = (j == (have - 1)[:, None]) & copy[:, None]
    grown = torch.where(at_last, free[first].to(torch.int32)[:, None], grown)
    src = torch.where(copy, last, -1).to(torch.int32)
    dst = torch.where(copy, free[first], -1).to(torch.int32)
    lens2 = torch.where(fits, lens + new, lens).to(torch.int32)
    refs = (refs + _count(grown, lens2, P) - _count(table, lens, P)).to(torch.int32)
    # copy
    i = copy.nonzero()[:, 0]
    st["pages"][:, dst[i].long()] = st["pages"][:, src[i].long()]
    return {"table": grown, "lens": lens2, "refs": refs, "src": src, "dst": dst, "left": left,
            "pages": st["pages"]}


def _plain_compact(st):
    refs, table = st["refs"], st["table"]
    P = refs.numel()
    at = torch.arange(P, device=refs.device)
    live = (refs > 0).sum()
    hole = ((refs == 0) & (at < live)).nonzero()[:, 0]
    mover = ((refs > 0) & (at >= live)).nonzero()[:, 0]
    st["pages"][:, hole] = st["pages"][:, mover]
    to = at.clone()
    to[mover] = hole
    new_refs = refs.clone()
    new_refs[hole] = refs[mover]
    new_refs[mover] = 0
    held = torch.arange(table.shape[1], device=refs.device) < ((st["lens"] + BLK - 1) // BLK)[:, None]
    return {"live": live.to(torch.int32).reshape(1),
            "table": torch.where(held, to[table.clamp(min=0).long()].to(torch.int32), table),
            "refs": new_refs, "pages": st["pages"]}


_PLAIN = {"attn": _plain_attn, "append": _plain_append, "step": _plain_step,
          "compact": _plain_compact}


# ---- what a pass cannot do without ----

def work(case):
    Hkv, D, lens = case["Hkv"], case["D"], _lens(case)
    vec, record = D + D / 16, Hkv * 68 * D  # bytes of a token's key and value; of a page
    if case["kind"] == "attn":
        nbytes = flops = 0.0
        for n in lens:
            share = max(case["keep"], 1.0 / _pages(n)) if case["keep"] else 1.0
            seen, pairs = set(), 0
            for pos in range(n - case["Sq"], n):
                if case["win"]:
                    pg = _live_pages(case, pos)
                    end = pos + 1 if case["causal"] else n
                    pairs += sum(min(BLK, end - kb * BLK) for kb in pg)
                    seen |= pg
                else:
                    pairs += pos + 1 if case["causal"] else n
            read = sum(min(BLK, n - kb * BLK) for kb in seen) if case["win"] else n
            nbytes += read * share * Hkv * vec
            flops += 4.0 * D * case["Hq"] * pairs * share
        rows = case["B"] * case["Hq"] * case["Sq"]
        return {"bytes": nbytes + rows * (4 * D + 4), "flops": flops}
    if case["kind"] == "append":  # written and read back
        tokens, padded = sum(_new(case)) * Hkv, case["B"] * Hkv * case["S"]
        return {"bytes": tokens * (4 * D + 2 * vec) + padded * 4 * D, "flops": 16.0 * tokens * D}
    _, M, P = _layout(case)
    if case["kind"] == "compact":
        moved, entries = _moves(case), sum(map(_pages, lens))
    else:
        moved, entries = _copies(case), case["B"] * M
    return {"bytes": 2.0 * case["layers"] * moved * record + 8 * (P + entries), "flops": float(P)}


def _copies(case):
    """Shared last pages that the beams of a step write into, all but one writer of each
    where all its holders write."""
    lens, parents, new = _lens(case), _parents(case), _new(case)
    total = 0
    for p, n in enumerate(lens):
        kids = [b for b, a in enumerate(parents) if a == p]
        writers = sum(new[b] > 0 for b in kids)
        if n % BLK and len(kids) > 1:
            total += writers - (writers == len(kids))
    return total


# ---- the definitions in 64 bits ----

def _decode64(rec, D):
    """Keys and values [Hkv, tokens, D] in 64 bits of records [pages, Hkv, 68 D], code by
    code: sign, exponent and mantissa bits."""
    P, H = rec.shape[:2]
    out = []
    for c0, s0 in ((0, 64 * D), (32 * D, 66 * D)):
        byte = rec[:, :, c0:c0 + 32 * D].reshape(P, H, BLK, D // 2, 1).int()
        c = torch.cat((byte % 16, byte // 16), -1).reshape(P, H, BLK, D)
        e, m = (c // 2) % 4, (c % 2).double()
        mag = torch.where(e == 0, m / 2, (1 + m / 2) * 2.0 ** (e - 1).double())
        b = rec[:, :, s0:s0 + 2 * D].reshape(P, H, BLK, D // 32, 1).expand(P, H, BLK, D // 32, 32)
        s = 2.0 ** (b.reshape(P, H, BLK, D).double() - 127)
        s = torch.where(s > 2.0 ** 127.5, math.nan, s)
        x = torch.where(c >= 8, -mag, mag) * s
        out.append(x.permute(1, 0, 2, 3).reshape(H, P * BLK, D))
    return out


def _exact_attn(case, st):
    q, B, Sq, D = st["q"], case["B"], case["Sq"], case["D"]
    Hq, G = case["Hq"], case["Hq"] // case["Hkv"]
    out = torch.zeros((B, Hq, Sq, D), dtype=torch.float64, device=q.device)
    lse = torch.full((B, Hq, Sq), -math.inf, dtype=torch.float64, device=q.device)
    for b in range(B):
        n = st["lens_host"][b]
        ids = st["table"][b, :_pages(n)].long()
        ks, vs = _decode64(st["pages"][ids], D)
        i, j = torch.arange(Sq, device=q.device)[:, None], torch.arange(n, device=q.device)
        pos = n - Sq + i
        hidden = (pos < 0) | (j > pos) if case["causal"] else (pos < 0) | (j < 0)
        if case["win"]:
            near = (j // BLK <= pos // BLK) & (j // BLK + case["win"] > pos // BLK)
            hidden = hidden | ~(near | (j < BLK * case["sink"]))
        for h in range(Hq):
            g = h // G
            dead = hidden
            if st["mask"] is not None:
                dead = hidden | (st["mask"][b, g][j // BLK] == 0)
            s = (q[b, h].double() @ ks[g, :n].T) * st["scale"]
            s = s.masked_fill(dead, -math.inf)
            l = torch.logsumexp(s, 1)
            p = torch.exp(s - torch.where(torch.isinf(l), 0.0, l)[:, None])
            out[b, h] = p @ vs[g, :n]
            lse[b, h] = l
    return {"out": out, "lse": lse}


def _exact_append(case, st):
    """Every value to the nearest of the 15 magnitudes' multiples (ties: even code)."""
    new = st["new_host"]
    grid = torch.tensor(_E2M1, dtype=torch.float64, device=st["k"].device)
    out = {}
    for name in ("k", "v"):
        x = st[name].double()
        g = x.reshape(*x.shape[:-1], -1, 32)
        top = g.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(torch.clamp(top, min=1e-300) / 6)).clamp(-125, 125)
        e = torch.where(6 * 2.0 ** (e - 1) >= top, e - 1, e).clamp(-125, 125)
        e = torch.where(6 * 2.0 ** e < top, e + 1, e).clamp(-125, 125)
        y = g / 2.0 ** e
        best = torch.full_like(y, math.inf)
        val = torch.zeros_like(y)
        for c in (0, 2, 4, 6, 1, 3, 5, 7):  # even codes first: they win ties
            d = (y.abs() - grid[c]).abs()
            val = torch.where(d < best, grid[c], val)
            best = torch.minimum(best, d)
        r = (torch.sign(y) * val * 2.0 ** e).reshape(x.shape)
        for b, n in enumerate(new):
            r[b, :, n:] = 0
        out[name] = r
    return out


def _exact_step(case, st):
    """The rows one after another, on the host."""
    table, lens, refs = st["table"].tolist(), st["lens"].tolist(), st["refs"].tolist()
    rows = []
    for p in st["parent"].tolist():
        rows.append(([], 0) if p < 0 else (table[p][:_pages(lens[p])], lens[p]))
    for r, n in zip(table, lens):
        for p in r[:_pages(n)]:
            refs[p] -= 1
    for r, _ in rows:
        for p in r:
            refs[p] += 1
    free = [p for p, r in enumerate(refs) if r == 0]
    spare = len(free)
    at, src, dst, out, outl = 0, [], [], [], []
    for (r, n), t in zip(rows, st["new"].tolist()):
        r, s, d = list(r), -1, -1
        if t and n % BLK and refs[r[-1]] > 1:
            s, d = r[-1], free[at]
            at += 1
            refs[s] -= 1
            refs[d] += 1
            r[-1] = d
        while len(r) < _pages(n + t):
            r.append(free[at])
            refs[free[at]] += 1
            at += 1
        src.append(s)
        dst.append(d)
        out.append(r + [-1] * (len(table[0]) - len(r)))
        outl.append(n + t)
    pages = st["pages"].clone()
    for s, d in zip(src, dst):
        if s >= 0:
            pages[:, d] = pages[:, s]

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device=pages.device)
    return {"table": ints(out), "lens": ints(outl), "refs": ints(refs), "src": ints(src),
            "dst": ints(dst), "left": ints([spare - at]), "pages": pages}


def _exact_compact(case, st):
    table, refs = st["table"].tolist(), st["refs"].tolist()
    live = sum(r > 0 for r in refs)
    holes = (p for p in range(live) if refs[p] == 0)
    to = {p: next(holes) for p in range(live, len(refs)) if refs[p] > 0}
    pages = st["pages"].clone()
    for p, h in to.items():
        pages[:, h] = pages[:, p]
        refs[h], refs[p] = refs[p], 0
    rows = [[to.get(p, p) for p in r] for r in table]

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device=pages.device)
    return {"live": ints([live]), "table": ints(rows), "refs": ints(refs), "pages": pages}


def exact(case, seed):
    st = prepare(case, seed)
    return {"attn": _exact_attn, "append": _exact_append, "step": _exact_step,
            "compact": _exact_compact}[case["kind"]](case, st)
