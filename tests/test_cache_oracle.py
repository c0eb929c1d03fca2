"""The cache's float64 model against closed forms, and the refusals of the cache's entry
points (no GPU needed: every check runs before any HIP call)."""
import numpy as np
import pytest
import torch

import oracle.kv_cache as kv
import paper_2607_09385_amd as steel
from paper_2607_09385_amd import _lib

FAKE = 0x100000  # 16-byte aligned, never dereferenced on the checked paths


def test_every_code_and_tie():
    x = np.zeros(32)
    x[:17] = [6, 0.25, 0.2501, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 5.001, -0.25, -0.75, -6, 0.0, -0.0, 1, 4]
    codes, scales = kv.encode(x)
    want = [6, 0, 0.5, 1, 1, 2, 2, 4, 4, 6, 0, -1, -6, 0, 0, 1, 4]
    assert scales[0] == 127
    assert kv.decode(codes, scales)[:17].tolist() == want


@pytest.mark.parametrize("amax,e", [(0.0, -125), (6.0, 0), (6.0001, 1), (3.0, -1), (1.5, -2),
                                    (2.0 ** -130, -125), (3.3e38, 125), (12.0, 1)])
def test_scale_is_the_smallest_that_holds_the_maximum(amax, e):
    assert kv.scale_exponent(amax) == e


@pytest.mark.parametrize("seed", range(3))
def test_values_are_off_by_half_a_step_at_most(seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(128) * 10.0 ** rng.uniform(-6, 6)
    codes, scales = kv.encode(x)
    y, s = kv.decode(codes, scales), np.repeat(2.0 ** (scales.astype(float) - 127), 32)
    a = np.abs(x) / s
    step = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))
    assert (np.abs(x - y) <= 0.5 * step * s).all() and a.max() <= 6


def test_non_finite_vectors_stand_for_nan():
    for bad in (np.nan, np.inf, -np.inf):
        x = np.ones(64)
        x[40] = bad
        assert np.isnan(kv.decode(*kv.encode(x))).all()


def test_attention_without_quantisation_error_is_the_plain_one():
    """Values on the E2M1 grid survive the cache, so attention over it is softmax(QK)V."""
    rng = np.random.default_rng(0)
    B, H, n, D = 1, 2, 150, 64
    grid = np.concatenate((kv.MAGNITUDES, -kv.MAGNITUDES))
    k, v = grid[rng.integers(0, 16, (B, H, n, D))], grid[rng.integers(0, 16, (B, H, n, D))]
    k[..., 0::32] = v[..., 0::32] = 6
    pages = rng.integers(0, 256, (5, H, 68 * D), dtype=np.uint8)
    table, lens = np.array([[3, 0, 4]]), np.array([n])
    kv.append(k, v, pages, table, lens)
    lk, lv = kv.load(pages, table, lens, n)
    assert np.array_equal(lk, k) and np.array_equal(lv, v)
    q = rng.standard_normal((B, 4, 3, D))
    out, lse = kv.attention(q, pages, table, lens, 0.1)
    for h in range(4):
        for i in range(3):
            s = k[0, h // 2, :n - 2 + i] @ q[0, h, i] * 0.1
            assert np.allclose(out[0, h, i], np.exp(s) @ v[0, h // 2, :n - 2 + i] / np.exp(s).sum())
            assert np.isclose(lse[0, h, i], np.log(np.exp(s).sum()))


def test_beam_step_by_hand():
    table = np.array([[5, 2, -1], [7, -1, -1]], np.int32)
    lens, refs = np.array([70, 64], np.int32), np.zeros(9, np.int32)
    refs[[5, 2, 7]] = 1
    t, l, r = kv.fork(table, lens, refs, [0, 0, -1])  # the second row ends, the first twice
    assert t.tolist() == [[5, 2, -1], [5, 2, -1], [-1, -1, -1]] and l.tolist() == [70, 70, 0]
    assert r[5] == r[2] == 2 and r[7] == 0
    t, l, r, src, dst, left = kv.grow(t, l, r, [1, 60, 1])
    # row 0 copies page 2 to page 0, row 1 is then alone with it and takes 1, row 2 takes 3
    assert t.tolist() == [[5, 0, -1], [5, 2, 1], [3, -1, -1]] and l.tolist() == [71, 130, 1]
    assert src.tolist() == [2, -1, -1] and dst.tolist() == [0, -1, -1] and left == 4
    pages = np.arange(9, dtype=np.uint8).reshape(1, 9, 1)
    p, t2, r2, live = kv.compact(pages, t, l, r)
    assert live == 5 and t2.tolist() == [[4, 0, -1], [4, 2, 1], [3, -1, -1]]
    assert p[0, 4, 0] == 5 and r2[:5].tolist() == [1, 1, 1, 1, 2] and not r2[5:].any()


# ---- refusals ----

def append(**kw):
    a = dict(k=FAKE, v=FAKE, st=(8192, 1024, 64, 8192, 1024, 64), pages=FAKE, table=FAKE, lens=FAKE,
             new=None, B=2, Hkv=8, S=16, D=64, M=4, P=9)
    a.update(kw)
    st = _lib.load().steel_cache_append(a["k"], a["v"], *a["st"], a["pages"], a["table"], a["lens"],
                                        a["new"], a["B"], a["Hkv"], a["S"], a["D"], a["M"], a["P"], None)
    return st, _lib.last_error()


@pytest.mark.parametrize("kw,code,text", [
    (dict(k=None), 1, "non-NULL"), (dict(table=None), 1, "non-NULL"), (dict(v=FAKE + 8), 1, "aligned"),
    (dict(pages=FAKE + 4), 1, "aligned"), (dict(D=96), 2, "D=96"), (dict(S=0), 1, ">= 1"),
    (dict(P=0), 1, ">= 1"), (dict(B=-1), 1, ">= 1"), (dict(M=1 << 25), 2, "max_pages"),
    (dict(st=(8192, 1024, 68, 8192, 1024, 64)), 1, "strides of k"),
    (dict(st=(8192, 1024, 64, 8192, -8, 64)), 1, "strides of v"),
    (dict(B=1 << 20, Hkv=1 << 10, S=1 << 10), 2, "too large"),
    (dict(B=1 << 12, Hkv=1 << 8, S=1 << 8, D=128), 2, "too large"), (dict(B=1 << 24, Hkv=1, S=1), 2, "too large"),
])
def test_append_refuses(kw, code, text):
    st, msg = append(**kw)
    assert st == code and text in msg


def attn(**kw):
    a = dict(q=FAKE, st=(4096, 512, 64), pages=FAKE, out=FAKE, B=2, Hq=8, Hkv=4, S=8, D=64, M=4, P=9,
             scale=0.1, causal=1, win=0, sink=0, flags=0, ws=FAKE, n=1 << 40)
    a.update(kw)
    st = _lib.load().steel_attn_cache(a["q"], *a["st"], a["pages"], FAKE, FAKE, None, None, a["out"],
                                      None, a["B"], a["Hq"], a["Hkv"], a["S"], a["D"], a["M"], a["P"],
                                      a["scale"], a["causal"], a["win"], a["sink"], a["flags"],
                                      a["ws"], a["n"], None)
    return st, _lib.last_error()


@pytest.mark.parametrize("kw,code,text", [
    (dict(q=None), 1, "non-NULL"), (dict(out=FAKE + 8), 1, "aligned"), (dict(Hq=6), 1, "multiple"),
    (dict(scale=0.0), 1, "scale"), (dict(scale=float("nan")), 1, "scale"), (dict(causal=2), 1, "causal"),
    (dict(win=-1), 1, "window_blocks"), (dict(sink=1), 1, "needs a window"), (dict(flags=2), 1, "flags"),
    (dict(D=32), 2, "D=32"), (dict(ws=None, M=64), 1, "workspace"),
    (dict(ws=FAKE + 16, M=64), 1, "256-byte"),
    (dict(n=256, M=64), 1, "smaller"), (dict(st=(4096, 512, 4)), 1, "strides of q"),
    (dict(B=1 << 20, Hq=1 << 10, Hkv=1, S=1 << 10), 2, "many"), (dict(B=1 << 24, Hq=1, Hkv=1), 2, "too large"),
    (dict(B=1 << 20, Hq=1 << 3, Hkv=1 << 3, M=1 << 10), 2, "too large"),
])
def test_attention_refuses(kw, code, text):
    st, msg = attn(**kw)
    assert st == code and text in msg


def test_attention_workspace_of_bad_sizes_is_zero():
    lib = _lib.load()
    assert lib.steel_attn_cache_workspace_bytes(1, 3, 2, 1, 64, 4) == 0
    assert "multiple" in _lib.last_error()
    assert lib.steel_attn_cache_workspace_bytes(1, 4, 2, 1, 64, 4) == 256  # none is used


def test_load_refuses():
    lib = _lib.load()
    assert lib.steel_cache_load(FAKE, FAKE, FAKE, None, None, FAKE, 1, 1, 1, 64, 1, 1, None) == 1
    assert lib.steel_cache_load(FAKE, FAKE, FAKE, None, FAKE + 8, FAKE, 1, 1, 1, 64, 1, 1, None) == 1
    assert lib.steel_cache_load(FAKE, FAKE, FAKE, None, FAKE, FAKE, 1, 1, 1, 80, 1, 1, None) == 2
    assert lib.steel_cache_load(FAKE, FAKE, FAKE, None, FAKE, FAKE, 1 << 10, 1 << 10, 1 << 9, 64, 1, 1, None) == 2


def test_page_calls_refuse():
    lib = _lib.load()
    f = FAKE
    g = FAKE + 0x1000
    assert lib.steel_pages_fork(f, f, f, None, g, g, 1, 1, 4, 8, None) == 1
    assert lib.steel_pages_fork(f, f, f, f, f, g, 1, 1, 4, 8, None) == 1 and "alias" in _lib.last_error()
    assert lib.steel_pages_fork(f, f, f, f, g, g, 0, 1, 4, 8, None) == 1
    assert lib.steel_pages_fork(f, f, f, f, g, g, 1, 1, 4, (1 << 22) + 1, None) == 2
    assert lib.steel_pages_fork(f, f, f, f, g, g, 1, (1 << 23) + 1, 4, 8, None) == 2
    n = lib.steel_pages_workspace_bytes(8, 2)
    assert n > 0 and lib.steel_pages_workspace_bytes(0, 2) == 0
    assert lib.steel_pages_grow(f, f, f, f, f, f, None, 2, 4, 8, f, n, None) == 1
    assert lib.steel_pages_grow(f, f, f, f, f, f, f, 2, 4, 8, f, n - 256, None) == 1
    assert "smaller" in _lib.last_error()
    assert lib.steel_pages_grow(f, f, f, f, f, f, f, 1 << 20, 1 << 12, 8, f, 1 << 40, None) == 2
    assert lib.steel_pages_copy(f, f, f, 1, 1, 8, 40, None) == 1 and "multiple of 16" in _lib.last_error()
    assert lib.steel_pages_copy(f + 4, f, f, 1, 1, 8, 64, None) == 1
    assert lib.steel_pages_copy(f, f, f, 0, 1, 8, 64, None) == 1
    assert lib.steel_pages_copy(f, f, f, 1, 0, 8, 64, None) == 1
    assert lib.steel_pages_copy(f, f, f, 1 << 30, 1, 8, 1 << 20, None) == 2
    assert lib.steel_pages_compact(f, f, f, f, None, 2, 4, 1, 8, 64, f, n, None) == 1
    assert lib.steel_pages_compact(f, f, f, f, f, 2, 4, 1, 8, 64, None, n, None) == 1


def test_binding_refuses():
    pages = torch.zeros((4, 2, 68 * 64), dtype=torch.uint8)
    t, l = torch.zeros((1, 2), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    q = torch.zeros((1, 2, 1, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        steel.attn_cache(q, pages, t, l)
    with pytest.raises(ValueError, match="GPU"):
        steel.cache_append(q, q, pages, t, l)
    with pytest.raises(TypeError):
        steel.cache_load(None, t, l, 1)
    with pytest.raises(ValueError, match="GPU"):
        steel.pages_fork(t, l, l, l)
    with pytest.raises(ValueError, match="GPU"):
        steel.pages_grow(t, l, l, l)
    with pytest.raises(ValueError, match="GPU"):
        steel.pages_copy(pages, l, l)
    with pytest.raises(ValueError, match="D must be"):
        steel.cache_pool(4, 2, 96, device="cpu")
    assert tuple(steel.cache_pool(4, 2, 64, layers=3, device="cpu").shape) == (3, 4, 2, 68 * 64)


def test_binding_checks_rows():
    t = torch.zeros((2, 4, 8, 64), dtype=torch.bfloat16)
    dev = t.device
    assert steel._check_bf16_rows("q", t, dev) == (2048, 512, 64)
    assert steel._check_bf16_rows("q", t.transpose(1, 2), dev) == (2048, 64, 512)
    assert steel._check_bf16_rows("q", t[:1, :, :1], dev) == (0, 512, 0)
    assert steel._check_bf16_rows("q", t[:, :1].expand(2, 4, 8, 64), dev) == (2048, 0, 64)
    with pytest.raises(ValueError, match="contiguous"):
        steel._check_bf16_rows("q", t.transpose(2, 3), dev)
    with pytest.raises(ValueError, match="bfloat16"):
        steel._check_bf16_rows("q", t.float(), dev)
    with pytest.raises(ValueError, match="on cuda"):
        steel._check_bf16_rows("q", t, torch.device("cuda", 0))
