"""Refusals of the page calls' longer forms (no GPU needed: every check runs before any HIP
call)."""
from paper_2607_09385_amd import _lib

F, G = 0x100000, 0x101000  # aligned, never dereferenced on the checked paths


def test_growth_refuses_a_took_that_is_its_input():
    lib = _lib.load()
    n = lib.steel_pages_workspace_bytes(8, 2)
    assert lib.steel_pages_grow_ex(F, F, F, G, F, F, F, G, 2, 4, 8, F, n, None) == 1
    assert "alias" in _lib.last_error()
    assert lib.steel_pages_grow_ex(F, F, F, G, F, F, None, F, 2, 4, 8, F, n, None) == 1
    assert lib.steel_pages_grow_ex(F, F, F, G, F, F, F, F, 2, 4, 8, F, n - 256, None) == 1
    assert "smaller" in _lib.last_error()
    assert lib.steel_pages_grow_ex(F, F, F, G, F, F, F, F, 0, 4, 8, F, n, None) == 1


def test_compaction_refuses_a_map_over_its_counts():
    lib = _lib.load()
    n = lib.steel_pages_workspace_bytes(8, 2)
    assert lib.steel_pages_compact_ex(F, F, F, G, F, G, 2, 4, 1, 8, 64, F, n, None) == 1
    assert "alias" in _lib.last_error()
    assert lib.steel_pages_compact_ex(F, F, F, G, None, F, 2, 4, 1, 8, 64, F, n, None) == 1
    assert lib.steel_pages_compact_ex(F, F, F, G, F, F, 2, 4, 1, 8, 64, F, n - 256, None) == 1


def test_growth_without_a_workspace():
    """Only where none is used: up to 1024 rows and 65,536 pages."""
    lib = _lib.load()
    need = lib.steel_pages_grow_workspace_bytes
    assert need(8, 2) == need(65536, 1024) == 256
    for sizes in ((65537, 1), (8, 1025)):
        assert need(*sizes) == lib.steel_pages_workspace_bytes(*sizes) > 256
        assert lib.steel_pages_grow_ex(F, F, F, G, F, F, F, None, sizes[1], 4, sizes[0], None, 1 << 40, None) == 1
        assert "workspace" in _lib.last_error()
    assert need(0, 2) == 0 and need(8, 0) == 0


def test_attention_workspace_with_and_without_a_mask():
    """The lists of live pages, 8 bytes an entry of the table and key/value head and a count a
    list, are asked for with a mask only."""
    lib = _lib.load()
    need = lib.steel_attn_cache_workspace_bytes_ex
    B, Hq, H, M = 64, 32, 8, 16384
    masked, plain = need(B, Hq, H, 1, 128, M, 1), need(B, Hq, H, 1, 128, M, 0)
    assert masked == lib.steel_attn_cache_workspace_bytes(B, Hq, H, 1, 128, M)
    assert masked - plain == 8 * B * H * M + 4 * B * H and plain < 1 << 23
    assert need(B, Hq, H, 1, 128, 24, 0) == need(B, Hq, H, 1, 128, 24, 1) == 256
    assert need(B, Hq, H, 100, 128, M, 0) == need(B, Hq, H, 100, 128, M, 1)  # no lists are made
    assert need(B, Hq, 3, 1, 128, M, 0) == 0 and "multiple" in _lib.last_error()

    def call(mask, n):
        return lib.steel_attn_cache(F, 0, 0, 0, F, F, F, None, mask, F, None, B, Hq, H, 1, 128, M, 9, 0.1,
                                    1, 0, 0, 0, F, n, None)
    assert call(F, masked - 256) == 1 and "smaller" in _lib.last_error()
    assert call(F, plain) == 1 and "smaller" in _lib.last_error()
    assert call(None, plain - 256) == 1 and "smaller" in _lib.last_error()
