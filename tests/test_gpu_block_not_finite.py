"""Decode over blocks where logits are not finite: NaN reaches the output and every weight of the heads that meet it, and no other key head's."""
import numpy as np
import pytest
import torch

from block_util import filled
from gpu_util import DEV
from paper_2412_20105_amd import binding as st3

pytestmark = pytest.mark.gpu


def step(dev, H, top, q, k, v, score):
    shape = st3.gqa_shape(dev.batch, H, dev.kv_heads, dev.dim)
    out = torch.full((dev.batch, H, dev.dim), 7.0, dtype=torch.bfloat16, device=DEV)
    ws = torch.full((st3.st3_block_workspace_bytes(shape, top),), 0xff, dtype=torch.uint8, device=DEV)
    st3.st3_block_decode(shape, q, k, v, dev.c, top, out, score, ws)
    torch.cuda.synchronize()
    return out


# strips of few blocks (one launch), and of so many that they are cut into chunks
@pytest.mark.parametrize("lens", [[150, 300], [3000, 2500]], ids=["whole", "chunks"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("where", ["new", "tail", "query"])
def test_nan_reaches_every_weight_of_its_heads(lens, bad, where):
    """(An infinite key gives infinite logits, and the weights of those are inf - inf.)"""
    rng, H, Hk, d = np.random.default_rng(7), 4, 2, 64
    dev, _ = filled(rng, lens, Hk, d, "int8", max(lens) // 64 + 1)
    q, k, v = (torch.from_numpy(rng.standard_normal((2, h, d)).astype(np.float32)).to(DEV).bfloat16() for h in (H, Hk, Hk))
    q.abs_()
    if where == "new":
        k[0, 1] = bad
    elif where == "tail":
        dev.k_tail[0, 1, 5] = bad
    else:
        q[0, 3] = float("nan")
    old = torch.rand((2, Hk, max(lens) + 3), device=DEV)
    score = old.clone()
    out = step(dev, H, max(lens), q, k, v, score)
    n = lens[0]
    assert bool(out[0, 3].isnan().all()) and bool(torch.isfinite(out[0, :2]).all()) and bool(torch.isfinite(out[1]).all())
    assert bool(out[0, 2].isnan().all()) == (where != "query")
    assert bool(score[0, 1, :n + 1].isnan().all())
    assert torch.equal(score[0, 1, n + 1:], old[0, 1, n + 1:])
    assert bool(torch.isfinite(score[0, 0]).all()) and bool(torch.isfinite(score[1]).all())


@pytest.mark.parametrize("lens", [[0, 64], [2304, 64]], ids=["whole", "chunks"])
def test_logits_that_are_all_minus_infinity_weigh_nothing(lens):
    rng, H, Hk, d = np.random.default_rng(8), 4, 2, 64
    dev, _ = filled(rng, lens, Hk, d, "e4m3", max(lens) // 64 + 1)
    dev.table[0] = -1                               # the new row is all that there is
    q, k, v = (torch.from_numpy(rng.standard_normal((2, h, d)).astype(np.float32)).to(DEV).bfloat16() for h in (H, Hk, Hk))
    q.abs_()
    k[0] = -float("inf")
    score = torch.ones((2, Hk, max(lens) + 3), device=DEV)
    out = step(dev, H, max(lens), q, k, v, score)
    n = lens[0]
    assert not bool(out[0].any()) and bool(torch.isfinite(out[1]).all())
    assert bool((score[0, :, :n] == 1).all()) and bool((score[0, :, n] == 0).all()) and bool((score[0, :, n + 1:] == 1).all())
