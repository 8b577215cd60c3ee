"""Lengths and batches that no launch holds are refused before anything is enqueued (no GPU)."""
import pytest

from paper_2412_20105_amd import binding as st3
from test_block_host import FAKE, UNSUPPORTED, cache, rows, shape

MOST = 2 ** 31 - 1
FAR = 1 << 50


def big(**more):
    return cache(table_blocks=1 << 25, table_stride=1 << 25, **more)


@pytest.mark.parametrize("max_len", [MOST, MOST - 62, 65535 * 64 + 1])
def test_store(max_len):
    assert st3.lib().st3_block_store(shape(batch=1), rows(), rows(), FAKE, MOST, max_len, big(), None) == UNSUPPORTED


@pytest.mark.parametrize("max_len,keep", [(MOST, MOST), (MOST, 100), (MOST, MOST - 62), (2 ** 30, 100), (2 ** 30 - 1, 65535 * 64 + 1)])
def test_evict(max_len, keep):
    n = 1 << 31
    assert st3.lib().st3_block_evict(shape(batch=1), big(), big(k_tail=1 << 40, v_tail=1 << 41), max_len, keep, 0, 0, FAKE, n, n, FAR, n, n, 2 * FAR, n, n,
                                     None) == UNSUPPORTED


@pytest.mark.parametrize("heads,kv_heads,max_len,scored", [(1, 1, 2 ** 30 - 1, False), (8, 2, 2 ** 30 - 1, True), (64, 64, 300_000_000, True)])
def test_decode(heads, kv_heads, max_len, scored):
    """More chunks than a grid has in y, or more workgroups behind them than it has in x."""
    new = rows(FAR, 1 << 13, 128)
    assert st3.lib().st3_block_decode(shape(1, heads, kv_heads), rows(FAKE, 1 << 13), new, new, big(), max_len, rows(2 * FAR, 1 << 13), FAKE if scored else None,
                                      1 << 31, 1 << 31, FAKE, 1 << 62, None) == UNSUPPORTED


@pytest.mark.parametrize("dtype", [st3.ST3_BF16, st3.ST3_F32])
def test_packed_attention(dtype):
    r = rows(FAKE, 32 * 128)
    assert st3.lib().st3_packed_attention(shape(1024, 32, 32, 128, dtype), r, r, r, FAKE, 1 << 30, 1 << 20, rows(FAR, 32 * 128), 0, None, 0, 0, None, 0,
                                          None) == UNSUPPORTED
