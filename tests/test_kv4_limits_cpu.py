"""Sizes at which attention over the 4-bit cache would count past 32 bits are refused on the host (no GPU needed)."""
import ctypes

import pytest

from paper_2607_13511_amd import binding

D256 = ctypes.c_void_p(256)          # never dereferenced: validation fails first


def call(heads_q, heads_kv, tokens, batch, table_pages, page=1024):
    d = D256
    return binding.lib().externd_kv4_attention(d, 4, heads_kv, 64, page, d, 1, 64 * heads_q, 64, heads_q, d, d, tokens, batch, 1, 32,
                                               d, d, d, table_pages, 0.125, 0, d, 1 << 40, None)


@pytest.mark.parametrize("heads_kv,table_pages", [(64, 1 << 21), (64, 1 << 30), (128, 1 << 20), (4096, 1 << 15), (1000, 140000)])
def test_tiles_of_all_cache_heads(heads_kv, table_pages):
    """A row block's tiles over all cache heads: the last head's would begin past 2^31."""
    assert (min(table_pages * 1024, (1 << 31) - 1) // 64 + 8) * heads_kv >= 1 << 31
    assert call(heads_kv, heads_kv, 1, 1, table_pages) == binding.EUNSUPPORTED


def test_rows_in_whole_blocks():
    """Rows rounded up to blocks of 256, and one block more."""
    assert call(1, 1, (1 << 31) - 100, 1, 4) == binding.EUNSUPPORTED
    assert call(64, 1, (1 << 25) - 1, 1, 4) == binding.EUNSUPPORTED


def test_block_rows():
    """Which kernel a call takes: fp32 and few rows or little work 4, many rows of a 16-bit type 256."""
    f = binding.lib().externd_kv4_attention_block_rows
    assert f(32, 8, 128, 1, 4096, 2, 2048, 12001) == 256 and f(32, 8, 128, 2, 4096, 2, 2048, 0) == 256
    assert f(32, 8, 128, 0, 4096, 2, 2048, 12001) == 4               # fp32
    assert f(32, 8, 128, 1, 32, 32, 1, 16384) == 4                   # single tokens
    assert f(8, 2, 128, 1, 64, 1, 64, 64) == 4                       # little work
    for bad in [(33, 8, 128, 1, 1, 1, 1, 0), (32, 8, 96, 1, 1, 1, 1, 0), (32, 8, 128, 3, 1, 1, 1, 0), (32, 8, 128, 1, -1, 1, 1, 0),
                (32, 8, 128, 1, 1, 0, 1, 0), (32, 8, 128, 1, 1, 1, 0, 0), (32, 8, 128, 1, 1, 1, 1, -1)]:
        assert f(*bad) == 0
