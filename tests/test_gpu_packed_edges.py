"""Packed prompts: what lies behind a row's own position reaches no row before it, also in the row's own tile of keys and rows."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, TORCH_DTYPE, rand_values
from paper_2412_20105_amd import binding as st3

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,Hk,d", [(4, 2, 128), (5, 1, 64), (32, 8, 128)])
@pytest.mark.parametrize("at", [1, 15, 16, 31, 32, 33, 64, 100, 129])
def test_rows_before_the_edge_are_the_same_bit_for_bit(at, H, Hk, d, dtype):
    rng, n, dt = np.random.default_rng(at), 130, TORCH_DTYPE[dtype]
    x = torch.from_numpy(rand_values(rng, (n, H + 2 * Hk, d), dtype)).to(DEV).to(dt)
    y = x.clone()
    y[at:, :H] = float("nan")
    y[at:, H:H + Hk] = float("inf")
    y[at:, H + Hk:] = float("nan")
    shape = st3.gqa_shape(1, H, Hk, d, st3.ST3_F32 if dtype == "f32" else st3.ST3_BF16)
    cu = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    got = []
    for z in (x, y):
        out = torch.zeros((n, H, d), dtype=dt, device=DEV)
        st3.st3_packed_attention(shape, z[:, :H], z[:, H:H + Hk], z[:, H + Hk:], cu, n, out)
        got.append(out)
    torch.cuda.synchronize()
    assert torch.equal(got[0][:at], got[1][:at]) and bool(torch.isfinite(got[0]).all())
