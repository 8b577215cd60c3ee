"""Page tables whose rows the library could not reach by their stride (no GPU: the binding's own checks)."""
from unittest import mock

import pytest
import torch

from paper_2412_20105_amd import binding as st3


def describe(table, batch):
    codes = [torch.zeros(s, dtype=torch.int8) for s in ((4, 2, 64, 64), (4, 2, 64, 64))]
    tails = [torch.zeros((batch, 2, 64, 64), dtype=torch.bfloat16) for _ in range(2)]
    with mock.patch.object(torch.Tensor, "is_cuda", True):
        return st3.block_cache(*codes, torch.zeros(4, 2), torch.zeros(4, 2), *tails, table, torch.zeros(batch, dtype=torch.int32))


@pytest.mark.parametrize("blocks", [1, 5])
def test_a_table_of_rows_that_lie_on_each_other_is_refused(blocks):
    """One row for all sequences: with a stride of its own length the second one would lie behind the tensor."""
    with pytest.raises(ValueError):
        describe(torch.zeros((1, blocks), dtype=torch.int32).expand(3, blocks), 3)
    with pytest.raises(ValueError):
        describe(torch.zeros(20, dtype=torch.int32).as_strided((3, blocks + 1), (blocks, 1)), 3)


def test_tables_that_are_taken():
    assert describe(torch.zeros((3, 5), dtype=torch.int32), 3).table_stride == 5
    assert describe(torch.zeros((3, 9), dtype=torch.int32)[:, 2:7], 3).table_stride == 9
    one = describe(torch.zeros((1, 5), dtype=torch.int32).as_strided((1, 5), (0, 1)), 1)      # one sequence: any stride
    assert one.table_stride >= 5 and one.table_blocks == 5
