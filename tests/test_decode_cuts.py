"""The rule by which decode over blocks is cut, against the workspaces that the library asks for (no GPU)."""
import pytest

import decode_cut
from paper_2412_20105_amd import binding as st3


@pytest.mark.parametrize("batch,heads,kv_heads", [(1, 32, 8), (2, 4, 1), (8, 40, 40), (10, 30, 30), (24, 8, 8), (23, 24, 8), (25, 16, 8), (32, 32, 8),
                                                  (40, 80, 2), (2, 17, 1), (2, 40, 1), (64, 64, 4), (65, 64, 4)])
@pytest.mark.parametrize("d", [64, 128])
def test_workspaces_are_those_of_the_rule(batch, heads, kv_heads, d):
    shape = st3.gqa_shape(batch, heads, kv_heads, d)
    for n in [*range(0, 1700, 61), 2047, 2048, 3500, 5000, 16255, 16256, 20000, 48895, 48896, 49087, 49088, 70000, 131072]:
        assert st3.st3_block_workspace_bytes(shape, n) == decode_cut.workspace(batch, heads, kv_heads, d, n), n
        for scored in (False, True):        # chunks of every length up to this one have room
            _, chunk, most = decode_cut.cut(batch, heads, kv_heads, d, n, scored)
            assert chunk == 0 or -(-(n // 64 + 1) // chunk) <= most
