"""Sizes whose products pass 31, 32 and 64 bits: refused on the host, before anything is launched or divided by; the pointers here are never followed."""
import ctypes

import pytest

from test_operator_arguments import APPEND, ATTENTION, OK, UNSUPPORTED, call, lib, pointer  # noqa: F401

MOST = 0x7fffff00


@pytest.mark.parametrize("batch,q_len,q_heads,heads", [
    (1, 1 << 16, 1 << 16, 1),                   # rows of a key head: 2^32
    (1 << 21, 1 << 21, 1 << 22, 1 << 10),       # all rows: 2^64
    (1 << 16, 1 << 15, 1, 1),                   # 2^31
    (1, MOST + 1, 1, 1), (MOST + 1, 1, 1, 1), (1, 0x7fffffff, 1, 1), (0x7fffffff, 0x7fffffff, 0x7fffffff, 1),
])
def test_rows_beyond_31_bits(lib, batch, q_len, q_heads, heads):  # noqa: F811
    size = lib.amq_cache_attention_workspace_bytes
    size.argtypes, size.restype = [ctypes.c_int] * 6, ctypes.c_size_t
    for tokens in (1, 1024, 4096, MOST):
        assert size(batch, q_len, q_heads, heads, 64, tokens) == 0
    assert call(lib.amq_cache_attention, ATTENTION, batch=batch, q_len=q_len, q_heads=q_heads, heads=heads) == UNSUPPORTED


def test_the_largest_workspaces(lib):  # noqa: F811
    """The workspace does not grow with the batch, the queries or the tokens beyond what the GPU's CTAs hold."""
    size = lib.amq_cache_attention_workspace_bytes
    size.argtypes, size.restype = [ctypes.c_int] * 6, ctypes.c_size_t
    for batch, q_len, q_heads, heads in ((1, MOST, 1, 1), (MOST, 1, 1, 1), (1, 1, MOST // 256 * 256, 256), (7, 4096, 128, 8)):
        rows = q_len * q_heads // heads
        blocks = heads * ((rows + 3) // 4)
        assert 0 < size(batch, q_len, q_heads, heads, 128, MOST) <= max(blocks, 592) * 2 * 8 * (128 * 4 + 8)


def test_append_to_a_cache_without_pages(lib):  # noqa: F811
    """Rows on no page are left out: all of them, and a cache without pages has no addresses."""
    none = {"cache_" + part: pointer(0) for part in ("kcodes", "kcoeffs", "vcodes", "vcoeffs")}
    assert call(lib.amq_cache_append, APPEND, pages=0, **none) == OK
