"""BlockGeneration's own checks (no GPU: they come before any call of the library)."""
import pytest
import torch

from paper_2412_20105_amd.block_pipeline import BlockGeneration


def begun(total, H=4, Hk=2, d=64):
    gen = BlockGeneration.__new__(BlockGeneration)         # (its buffers are on a device)
    gen.H, gen.Hk, gen.d, gen.total, gen.lens = H, Hk, d, total, [total]
    return gen


def packed(q, k=None, v=None, H=4, Hk=2, d=64):
    k, v = q if k is None else k, q if v is None else v
    return tuple(torch.zeros((n, h, d), dtype=torch.bfloat16) for n, h in ((q, H), (k, Hk), (v, Hk)))


@pytest.mark.parametrize("total,rows", [(200, (150,)), (200, (250,)), (200, (199,)), (200, (0,)), (0, (3,)), (200, (200, 150)), (200, (200, 200, 250)),
                                        (200, (150, 200, 200)), (0, (0, 1))])
def test_prompts_of_another_number_of_rows_than_begin_was_told(total, rows):
    with pytest.raises(ValueError, match="rows"):
        begun(total).prefill_layer(0, *packed(*rows))


def test_no_rows_at_all():
    out = begun(0).prefill_layer(0, *packed(0))
    assert out.shape == (0, 4, 64)
