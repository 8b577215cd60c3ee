"""A turn without rows is no error, though an empty tensor has no address (no GPU: nothing is enqueued)."""
import ctypes as C

import pytest

from paper_2412_20105_amd import binding as st3

FAKE = 0x10000


@pytest.mark.parametrize("layout", [st3.ST3_ROTARY_HALVES, st3.ST3_ROTARY_ADJACENT])
def test_no_rows_with_a_table_of_none(layout):
    none, empty = st3.Rows(None, 1024, 128), st3.Rotary(None, 128, 64, layout)
    shape = st3.gqa_shape(2, 8, 2, 128)
    cache = st3.BlockCache(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 8, FAKE, 8, 4, st3.ST3_BLOCK_INT8)
    L, at = st3.lib(), C.byref
    assert L.st3_rotary_table(1, 64, None, FAKE, None, 0, 0, None, 128, None) == st3.ST3_OK
    assert L.st3_rotate_rows(at(none), at(none), 8, 0, 128, st3.ST3_BF16, at(empty), 0, None) == st3.ST3_OK
    assert L.st3_block_append(at(shape), at(none), at(none), FAKE, 0, 0, at(cache), 100, at(empty), None) == st3.ST3_OK
    assert L.st3_block_attend(at(shape), at(none), FAKE, 0, 0, at(cache), 100, at(none), 1, None, 0, 0, None, 0, None) == st3.ST3_OK
    # with rows the table has to be somewhere
    some = st3.Rows(FAKE, 1024, 128)
    assert L.st3_block_append(at(shape), at(some), at(some), FAKE, 10, 5, at(cache), 100, at(empty), None) == 1
