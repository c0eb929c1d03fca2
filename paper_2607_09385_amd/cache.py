"""The paged 4-bit key/value cache: writing, reading, attention, page bookkeeping.

``pages`` is a uint8 pool [n_pages, Hkv, 68 * D] (include/steel.h has the layout: 64
tokens a page, 4.25 bits a value), ``page_table`` int32 [B, max_pages] the pages of each
sequence, ``lens`` int32 [B] their tokens and ``refs`` int32 [n_pages] how many rows
hold each page (0: free).  A decoding step, its table shared by all layers' pools:

    src, dst, left = pages_grow(page_table, lens, refs, n_new, took=took)   # once a step
    for pool in pools:                                                      # every layer
        pages_copy(pool, src, dst)                # pages that forked rows write into
        cache_append(k, v, pool, page_table, lens, new=took)
        out, lse = attn_cache(q, pool, page_table, lens, new=took)

``took`` (int32 [B], like ``n_new``) is what there was room for: ``n_new``, or 0 everywhere
where the pool is too full.  Such a step changes nothing and its ``out`` is 0; ``left`` is
negative then, for the host to see when it looks next.  With ``n_new`` in the place of ``took``
it would write over tokens that are there, so ``left`` has to be looked at first.

Everything stays on the device: no call waits for the host, so a step may be captured
into a graph.  Tensors that a call makes belong to the stream it runs on.
"""
from __future__ import annotations

import functools
import math
from typing import Optional

from . import _lib
from . import STEEL_OUT_BF16, _check_bf16_rows, _on, _torch


def _ints(name, t, shape, device):
    torch = _torch()
    if isinstance(t, torch.Tensor) and t.dtype is torch.int32 and t.shape == shape \
            and t.device == device and t.is_contiguous():
        return t.data_ptr()
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device != device:
        raise ValueError(f"{name} must be on {device} (got {t.device})")
    raise ValueError(f"{name} must be a contiguous int32 tensor {list(shape)} "
                     f"(got {t.dtype} {tuple(t.shape)})")


def _numel(name, t):
    if not isinstance(t, _torch().Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    return t.numel()


def _table(page_table, lens, device):
    """(B, max_pages, pointer to the table, pointer to the lengths)."""
    if not isinstance(page_table, _torch().Tensor) or page_table.dim() != 2:
        raise ValueError("page_table must be an int32 tensor [B, max_pages]")
    B, M = page_table.shape
    return B, M, _ints("page_table", page_table, (B, M), device), _ints("lens", lens, (B,), device)


def _gpu(name, t):
    if not isinstance(t, _torch().Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be on a GPU device (got {t.device})")


def _pool(pages):
    """(n_pages, Hkv, D) of one layer's pool."""
    _gpu("pages", pages)
    if pages.dtype != _torch().uint8 or pages.dim() != 3 or not pages.is_contiguous() \
            or pages.shape[2] % 68 != 0:
        raise ValueError("pages must be a contiguous uint8 tensor [n_pages, Hkv, 68 * D] "
                         f"(got {pages.dtype} {tuple(pages.shape)})")
    n, h, r = pages.shape
    return n, h, r // 68


def _layers(pages):
    """(layers, n_pages, bytes of a page) of one pool, or of several of one size."""
    _gpu("pages", pages)
    if pages.dtype != _torch().uint8 or pages.dim() not in (3, 4) or not pages.is_contiguous():
        raise ValueError("pages must be a contiguous uint8 tensor [n_pages, Hkv, bytes] or "
                         f"[layers, n_pages, Hkv, bytes] (got {pages.dtype} {tuple(pages.shape)})")
    shape = pages.shape
    return (shape[0] if len(shape) == 4 else 1), shape[-3], shape[-2] * shape[-1]


def _empty(stream, like, *specs):
    """New tensors (shape, dtype) on like's device, allocated for the stream the call runs on."""
    if stream is None:
        return [like.new_empty(shape, dtype=dtype) for shape, dtype in specs]
    if stream.device != like.device:
        raise ValueError(f"stream must be on {like.device} (got {stream.device})")
    with _torch().cuda.stream(stream):
        return [like.new_empty(shape, dtype=dtype) for shape, dtype in specs]


def _call(fn, device, stream, *args):
    """fn(*args, stream handle) with the device current."""
    torch = _torch()
    if stream is None:
        handle = torch._C._cuda_getCurrentRawStream(device.index)
    elif stream.device != device:
        raise ValueError(f"stream must be on {device} (got {stream.device})")
    else:
        handle = int(stream.cuda_stream)
    if torch._C._cuda_getDevice() == device.index:
        st = fn(*args, handle)
    else:
        with _on(device):
            st = fn(*args, handle)
    if st:
        _lib.check(st)


@functools.lru_cache(maxsize=256)
def _bytes(name, *sizes):
    """Workspace bytes that the library asks for."""
    n = getattr(_lib.load(), name)(*sizes)
    if n == 0:
        raise _lib.SteelError(_lib.STEEL_ERR_INVALID_ARGUMENT, _lib.last_error())
    return n


def cache_pool(n_pages: int, Hkv: int, D: int, *, layers: Optional[int] = None, device=None):
    """An empty pool: uint8 [n_pages, Hkv, 68 * D], or [layers, ...] of them (pool[l]
    is layer l's)."""
    torch = _torch()
    if D not in (64, 128):
        raise ValueError(f"D must be 64 or 128 (got {D})")
    shape = (n_pages, Hkv, 68 * D)
    return torch.zeros(shape if layers is None else (layers, *shape), dtype=torch.uint8,
                       device=device or torch.device("cuda"))


def cache_append(k, v, pages, page_table, lens, *, new=None, stream=None):
    """Write keys and values bf16 [B, Hkv, S, D] (any strides with contiguous rows)
    into the cache, as tokens lens[b] - new[b] + i of sequence b (``new`` int32 [B]:
    tokens of each sequence; None: S)."""
    n_pages, Hkv, D = _pool(pages)
    device = pages.device
    B, M, tp, lp = _table(page_table, lens, device)
    ks = _check_bf16_rows("k", k, device)
    vs = _check_bf16_rows("v", v, device)
    S = k.shape[2]
    if k.shape != (B, Hkv, S, D) or v.shape != k.shape:
        raise ValueError(f"k and v must be [{B}, {Hkv}, S, {D}] (got {tuple(k.shape)}, {tuple(v.shape)})")
    _call(_lib.load().steel_cache_append, device, stream, k.data_ptr(), v.data_ptr(), *ks, *vs,
          pages.data_ptr(), tp, lp, None if new is None else _ints("new", new, (B,), device),
          B, Hkv, S, D, M, n_pages)


def cache_load(pages, page_table, lens, S: int, *, start=None, stream=None):
    """Keys and values bf16 [B, Hkv, S, D] of tokens start[b] + i (``start`` int32 [B];
    None: 0), exactly as the cache holds them; rows without a token are 0."""
    n_pages, Hkv, D = _pool(pages)
    device = pages.device
    B, M, tp, lp = _table(page_table, lens, device)
    sp = None if start is None else _ints("start", start, (B,), device)
    kv = ((B, Hkv, S, D), _torch().bfloat16)
    k, v = _empty(stream, pages, kv, kv)
    _call(_lib.load().steel_cache_load, device, stream, pages.data_ptr(), tp, lp, sp, k.data_ptr(),
          v.data_ptr(), B, Hkv, S, D, M, n_pages)
    return k, v


def attn_cache(q, pages, page_table, lens, *, new=None, block_mask=None, window_blocks: int = 0,
               sink_blocks: int = 0, scale: Optional[float] = None, causal: bool = True,
               out_dtype=None, out=None, lse=None, stream=None):
    """Attention of queries bf16 [B, Hq, S_q, D] (any strides with contiguous rows) over
    the cached keys and values of their sequences; query i stands at position
    lens[b] - new[b] + i (``new`` int32 [B]: queries of each sequence; None: S_q).

    block_mask: uint8 [B, Hkv, max_pages] or None, pages that the heads of a key/value
    head see; window_blocks, sink_blocks: as for ``attn_fwd_window`` (0: no window).
    Returns (out [B, Hq, S_q, D] in ``out_dtype``, float32 or bfloat16, lse fp32
    [B, Hq, S_q]); rows without a visible key are 0 and -inf."""
    torch = _torch()
    n_pages, Hkv, D = _pool(pages)
    device = pages.device
    B, M, tp, lp = _table(page_table, lens, device)
    qs = _check_bf16_rows("q", q, device)
    _, Hq, S_q, _ = q.shape
    if q.shape != (B, Hq, S_q, D):
        raise ValueError(f"q must be [{B}, Hq, S_q, {D}] (got {tuple(q.shape)})")
    np_ = None if new is None else _ints("new", new, (B,), device)
    mp = None
    if block_mask is not None:
        if not isinstance(block_mask, torch.Tensor) or block_mask.dtype != torch.uint8 \
                or block_mask.shape != (B, Hkv, M) or not block_mask.is_contiguous() \
                or block_mask.device != device:
            raise ValueError(f"block_mask must be a contiguous uint8 [{B}, {Hkv}, {M}] on {device}")
        mp = block_mask.data_ptr()
    odt = torch.float32 if out_dtype is None else out_dtype
    if odt is not torch.float32 and odt is not torch.bfloat16:
        raise ValueError("out_dtype must be torch.float32 or torch.bfloat16")
    rows = (B, Hq, S_q)
    if out is None:
        out, = _empty(stream, pages, ((B, Hq, S_q, D), odt))
    elif out.dtype != odt or out.shape != (B, Hq, S_q, D) or not out.is_contiguous() \
            or out.device != device:
        raise ValueError(f"out must be a contiguous {odt} tensor [B, Hq, S_q, D] on {device}")
    if lse is None:
        lse, = _empty(stream, pages, (rows, torch.float32))
    elif lse.dtype != torch.float32 or lse.shape != rows or not lse.is_contiguous() \
            or lse.device != device:
        raise ValueError(f"lse must be a contiguous float32 tensor [B, Hq, S_q] on {device}")
    nbytes = _bytes("steel_attn_cache_workspace_bytes_ex", B, Hq, Hkv, S_q, D, M, mp is not None)
    ws = None  # 256 bytes: none is used
    if nbytes > 256:
        ws, = _empty(stream, pages, ((nbytes,), torch.uint8))
    _call(_lib.load().steel_attn_cache, device, stream, q.data_ptr(), *qs, pages.data_ptr(), tp, lp,
          np_, mp, out.data_ptr(), lse.data_ptr(), B, Hq, Hkv, S_q, D, M, n_pages,
          1.0 / math.sqrt(D) if scale is None else float(scale), 1 if causal else 0,
          int(window_blocks), int(sink_blocks), STEEL_OUT_BF16 if odt is torch.bfloat16 else 0,
          None if ws is None else ws.data_ptr(), nbytes)
    return out, lse


def pages_fork(page_table, lens, refs, parent, *, stream=None):
    """New rows (page_table [B_out, max_pages], lens [B_out]): row b continues old row
    parent[b] (int32 [B_out]), sharing its pages, or is empty (-1).  ``refs`` is
    updated: pages that no new row holds become free."""
    _gpu("page_table", page_table)
    device = page_table.device
    B, M, tp, lp = _table(page_table, lens, device)
    n_pages, B_out = _numel("refs", refs), _numel("parent", parent)
    rp = _ints("refs", refs, (n_pages,), device)
    pp = _ints("parent", parent, (B_out,), device)
    i32 = page_table.dtype
    table, length = _empty(stream, page_table, ((B_out, M), i32), ((B_out,), i32))
    _call(_lib.load().steel_pages_fork, device, stream, tp, lp, rp, pp, table.data_ptr(),
          length.data_ptr(), B, B_out, M, n_pages)
    return table, length


def pages_grow(page_table, lens, refs, new, *, took=None, stream=None):
    """Room for new[b] (int32 [B]) more tokens of every sequence: page_table, lens and
    refs are updated, the lowest free pages taken first.  Returns (src, dst, left): the
    pages that ``pages_copy`` has to copy before the new tokens are written (int32
    [B], -1: none; rows that write into a page which other rows hold get their own) and
    the free pages that remain (int32 [1]; negative: too few, nothing has changed).

    took: int32 [B] that is filled with the tokens each sequence got room for, max(new[b], 0)
    or 0 where nothing has changed: what the calls that follow take as their ``new``."""
    _gpu("page_table", page_table)
    device = page_table.device
    B, M, tp, lp = _table(page_table, lens, device)
    n_pages = _numel("refs", refs)
    rp = _ints("refs", refs, (n_pages,), device)
    np_ = _ints("new", new, (B,), device)
    kp = None if took is None else _ints("took", took, (B,), device)
    nbytes = _bytes("steel_pages_grow_workspace_bytes", n_pages, B)
    ws = None  # 256 bytes: none is used
    if nbytes > 256:
        ws, = _empty(stream, page_table, ((nbytes,), _torch().uint8))
    made, = _empty(stream, page_table, ((2 * B + 1,), page_table.dtype))
    src, dst, left = made.split_with_sizes((B, B, 1))
    _call(_lib.load().steel_pages_grow_ex, device, stream, tp, lp, rp, np_, src.data_ptr(),
          dst.data_ptr(), left.data_ptr(), kp, B, M, n_pages,
          None if ws is None else ws.data_ptr(), nbytes)
    return src, dst, left


def pages_copy(pages, src, dst, *, stream=None):
    """Copy page src[i] onto page dst[i] (int32 [n]; pairs with -1 are skipped) in one
    pool or in every layer of a [layers, ...] pool.  Destinations are distinct and no
    sources."""
    layers, n_pages, nbytes = _layers(pages)
    n, device = _numel("src", src), pages.device
    _call(_lib.load().steel_pages_copy, device, stream, pages.data_ptr(),
          _ints("src", src, (n,), device), _ints("dst", dst, (n,), device), n, layers, n_pages, nbytes)


def pages_compact(pages, page_table, lens, refs, *, to=None, stream=None):
    """Move the live pages (refs > 0) of a pool, or of every layer of a [layers, ...]
    pool, to its front; page_table and refs follow.  Returns their number (int32 [1]).

    to: int32 [n_pages] that is filled with the number each live page has now, by the one it
    had (-1: free).  Pages that no row of ``page_table`` holds (a kept prefix, another table)
    move too, and this is where their holders find them."""
    layers, n_pages, page_bytes = _layers(pages)
    device = pages.device
    B, M, tp, lp = _table(page_table, lens, device)
    rp = _ints("refs", refs, (n_pages,), device)
    op = None if to is None else _ints("to", to, (n_pages,), device)
    nbytes = _bytes("steel_pages_workspace_bytes", n_pages, B)
    ws, live = _empty(stream, pages, ((nbytes,), _torch().uint8), ((1,), page_table.dtype))
    _call(_lib.load().steel_pages_compact_ex, device, stream, pages.data_ptr(), tp, lp, rp,
          live.data_ptr(), op, B, M, layers, n_pages, page_bytes, ws.data_ptr(), nbytes)
    return live
