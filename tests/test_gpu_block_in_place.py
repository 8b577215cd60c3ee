"""Decode over blocks whose output is the queries themselves, row for row: the same as into memory of its own, in every form of the launch."""
import numpy as np
import pytest
import torch

import decode_cut
from gpu_util import DEV
from paper_2412_20105_amd import binding as st3
from test_gpu_decode_dispatch import LONG, SHORT, random_cache, some

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,H,Hk,d,scored,form", [
    (some(SHORT, 8), 8, 2, 128, True, (12, True)), (some(SHORT, 10), 60, 30, 64, True, (4, True)), (some(LONG, 10), 30, 30, 128, False, (4, True)),
    (some(SHORT, 8), 40, 1, 128, False, (12, True)), ([5000, 300], 4, 1, 64, True, (4, False)), ([5000, 300], 40, 1, 128, True, (4, False))])
def test_queries_that_become_the_output(lens, H, Hk, d, scored, form):
    waves, chunk, _ = decode_cut.cut(len(lens), H, Hk, d, max(lens), scored)
    assert (waves, chunk == 0) == form
    rng, B = np.random.default_rng(H + d), len(lens)
    dev, shape = random_cache(rng, lens, Hk, d, "int8"), st3.gqa_shape(B, H, Hk, d)
    x = torch.from_numpy(rng.standard_normal((B, H + 2 * Hk, d)).astype(np.float32)).to(DEV).bfloat16()
    ws = torch.empty(st3.st3_block_workspace_bytes(shape, max(lens)), dtype=torch.uint8, device=DEV)
    got = []
    for in_place in (False, True):
        y = x.clone()
        q, k, v = y[:, :H], y[:, H:H + Hk], y[:, H + Hk:]
        out = q if in_place else torch.zeros((B, H, d), dtype=torch.bfloat16, device=DEV)
        score = torch.zeros((B, Hk, max(lens) + 1), device=DEV) if scored else None
        st3.st3_block_decode(shape, q, k, v, dev.c, max(lens), out, score, ws)
        torch.cuda.synchronize()
        got.append((out.clone(), score))
        assert torch.equal(y[:, H:], x[:, H:])
    assert torch.equal(got[0][0], got[1][0]) and (not scored or torch.equal(got[0][1], got[1][1]))
