"""Evictions of rows whose values are a few of the smallest float32: the new block's scale is rounded there, and a quotient by it can pass the largest code."""
import numpy as np
import pytest
import torch

from block_util import BLOCK, DeviceCache
from gpu_util import DEV
from oracle import block_oracle as bo
from test_gpu_block_cache import do_evict

pytestmark = pytest.mark.gpu

UNIT = 2.0 ** -149
# (old scale in units, largest code kept): 516 and 146 are the scales of blocks whose largest value was 2^-133
KINDS = {"int8": [(516, 1), (516, 2), (516, 5), (516, 127), (200, 1), (1, 127), (3, 40), (64, 1), (63, 1), (190, 1), (191, 1), (318, 1), (95, 2), (700, 1)],
         "e4m3": [(146, 7), (146, 10), (146, 3), (146, 16), (1, 448), (224, 1), (223, 1), (671, 1), (672, 1), (96, 7), (500, 2), (1119, 1), (100, 9), (700, 1)]}


def largest_quotient(units, code, top):
    x = np.float32(code) * np.float32(units * UNIT)
    scale = x * (np.float32(1) / np.float32(top))
    return x / scale if scale > 0 else 0.0


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
def test_codes_of_the_smallest_values_are_saturated(code, d):
    rng, top = np.random.default_rng(5), 127.0 if code == "int8" else 448.0
    # some of these pass the largest code by more than a rounding to it
    assert max(largest_quotient(u, m, top) for u, m in KINDS[code]) > (128.5 if code == "int8" else 480.0)
    Hk, n, keep = len(KINDS[code]), 4 * BLOCK, 2 * BLOCK
    dev = DeviceCache(rng, 1, Hk, d, code, 4)
    ref = bo.BlockCache(1, Hk, d, code)
    for j in range(4):
        page = int(dev.table[0, j])
        for h, (units, most) in enumerate(KINDS[code]):
            pair = []
            for codes, scale, turned in ((dev.k_codes, dev.k_scale, False), (dev.v_codes, dev.v_scale, True)):
                x = rng.integers(-min(most, 16), min(most, 16) + 1, size=(BLOCK, d)).astype(np.float64)     # (whole numbers up to 16 are codes of E4M3)
                x[1, :2], x[-1, -2:] = [most, -most], [-most, most]
                t = torch.from_numpy(np.ascontiguousarray(x.T if turned else x)).float()
                t = t.to(torch.int8) if code == "int8" else t.to(torch.float8_e4m3fn).view(torch.uint8)
                codes[page, h].copy_(t)
                scale[page, h] = float(units * UNIT)
                pair.append((x, np.float32(units * UNIT)))
            ref.blocks[0][h].append(tuple(pair))
    dev.set_len([n])
    assert all(float(dev.k_scale[int(dev.table[0, 0]), h]) == u * UNIT for h, (u, _) in enumerate(KINDS[code]))
    score = np.zeros((1, Hk, n + 1))
    score[:, :, 1:n:2] = 1.0                        # every other row, the ones with the largest codes among them
    do_evict(rng, dev, ref, [n], keep, 0, 0, score)
