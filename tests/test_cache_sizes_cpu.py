"""Sizes of a cache whose products an int, or 64 bits, do not hold: refused before anything is computed with them."""
import ctypes

import pytest

from paper_2412_15803_gb300 import wq4
from test_cache_calls_cpu import A, INVALID, UNSUPPORTED, cache, pool

# heads of 128 past an int's elements of a row; rows of a pool past 2^64 (their product's low bits are 0)
MANY_HEADS = dict(num_pages=1, n_kv_heads=1 << 25)
MANY_ROWS = dict(num_pages=1 << 30, n_kv_heads=1 << 16, page_size=1 << 18, page_table_stride=1)


@pytest.mark.parametrize("sizes,heads", [(MANY_HEADS, 1 << 25), (MANY_HEADS, 1 << 27), (dict(num_pages=1, n_kv_heads=1 << 24), 1 << 24),
                                         (MANY_ROWS, 1 << 16), (MANY_ROWS, 1 << 19)])
def test_attention_refuses(sizes, heads):
    L, c, wide = wq4.load(), cache(**sizes), (1 << 31) - 8
    assert L.wq4_paged_attention(ctypes.byref(c), 4 * A, wide, 5 * A, 6 * A, wide, 1, heads, 0.1, 7 * A, 1 << 40, None) == UNSUPPORTED
    assert L.wq4_window_attention(ctypes.byref(c), 4 * A, wide, 5 * A, 6 * A, wide, 1, heads, 0.1, 5, 1, 7 * A, 1 << 40, None) == UNSUPPORTED
    assert L.wq4_prompt_attention(ctypes.byref(c), 4 * A, wide, 8 * A, 5 * A, 6 * A, wide, 1, 1, heads, 0.1, 5, 1, 7 * A, 1 << 40,
                                  None) == UNSUPPORTED
    assert L.wq4_prompt_append(ctypes.byref(c), 4 * A, wide, 6 * A, wide, 8 * A, 5 * A, 1, 1, heads, 1e4, None) == UNSUPPORTED


@pytest.mark.parametrize("sizes", [MANY_HEADS, dict(num_pages=1, n_kv_heads=1 << 24), dict(num_pages=1, n_kv_heads=(1 << 31) - 1)])
def test_append_of_one_token_refuses(sizes):
    L, c = wq4.load(), cache(**sizes)
    assert L.wq4_kv_append(ctypes.byref(c), 4 * A, 5 * A, (1 << 31) - 8, 6 * A, 1, None) == UNSUPPORTED


def test_pool_refuses():
    L, p = wq4.load(), pool(layers=1, caches=[cache(**MANY_ROWS)])
    assert L.wq4_kv_compact(ctypes.byref(p), None) == UNSUPPORTED


def test_the_largest_row_is_still_checked():
    """One head less than an int's worth of elements is no matter of size: a row shorter than its heads is invalid."""
    c, heads = cache(num_pages=1, n_kv_heads=(1 << 24) - 1), (1 << 24) - 1
    L = wq4.load()
    for call in (lambda s: L.wq4_paged_attention(ctypes.byref(c), 4 * A, s, 5 * A, 6 * A, s, 1, heads, 0.1, 7 * A, 1 << 40, None),
                 lambda s: L.wq4_window_attention(ctypes.byref(c), 4 * A, s, 5 * A, 6 * A, s, 1, heads, 0.1, 5, 1, 7 * A, 1 << 40, None)):
        assert call(heads * 128 - 8) == INVALID
