"""BlockGeneration refuses prompts once rows have come behind them (no GPU: the checks come before any call of the library)."""
import pytest
import torch

from paper_2412_20105_amd import binding as st3
from paper_2412_20105_amd.block_pipeline import BlockGeneration


def begun(lens):
    gen = BlockGeneration.__new__(BlockGeneration)          # (its buffers are on a device)
    gen.L, gen.H, gen.Hk, gen.d, gen.B, gen.capacity, gen.budget, gen.device = 0, 8, 2, 128, len(lens), 256, 128, "cpu"
    gen.shape = st3.gqa_shape(len(lens), 8, 2, 128)
    gen._turn_ws = gen._prompt_ws = torch.empty(0, dtype=torch.uint8)
    gen.len, gen.live = (torch.zeros(len(lens), dtype=torch.int32) for _ in range(2))
    gen.begin(lens)
    return gen


def rows(n):
    return tuple(torch.zeros((n, h, 128), dtype=torch.bfloat16) for h in (8, 2, 2))


def a_turn(gen, new):
    gen.begin_turn(new)
    gen.finish_turn()


@pytest.mark.parametrize("behind,n", [
    (lambda gen: a_turn(gen, [14, 0, 6]), 20),              # as many rows as the turn had: they would be taken for prompts, from row 0 on
    (lambda gen: a_turn(gen, [14, 0, 6]), 50), (lambda gen: a_turn(gen, [0, 0, 0]), 0), (lambda gen: gen.finish_step(), 50), (lambda gen: gen.evict(), 50)],
    ids=["turn", "turn_prompts_rows", "turn_of_none", "step", "eviction"])
def test_prompts_come_before_everything_else(behind, n):
    gen = begun([20, -1, 30])
    gen.evictions = 0
    behind(gen)
    with pytest.raises(ValueError, match="begin"):
        gen.prefill_layer(0, *rows(n))


def test_a_new_batch_takes_prompts_again():
    gen = begun([20, -1, 30])
    a_turn(gen, [14, 0, 6])
    gen.begin([0, -1, 0])
    assert gen.prefill_layer(0, *rows(0)).shape == (0, 8, 128)
    gen.retire(2)                                           # (an ended sequence leaves the others' prompts as they are)
    assert gen.prefill_layer(0, *rows(0)).shape == (0, 8, 128)
