"""Up to 32 rows of a key head (new tokens times its query heads) are attended as exactly as single tokens: weights as two bf16 terms, 2^-16 of each left
out at most."""
import numpy as np
import pytest
import torch

from gpu_util import DEV
from paper_2412_20105_amd import binding as st3
from test_gpu_block_attend import run
from test_gpu_block_attend_odd import FORMS, check, prepared

pytestmark = pytest.mark.gpu

# A weight is cut off at 8 significant bits; the rest, below 2^-7 of the power of two under the weight, is rounded to 8 more: off by 2^-16 of it at most.
TERMS = 2.0 ** -16
FEW = [f for f, (old, new, H, Hk, d) in FORMS.items() if new * H // Hk <= 32]


@pytest.mark.parametrize("form", FEW)
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_outputs_are_off_by_their_own_rounding(form, code):
    old, new, H, Hk, d = FORMS[form]
    shape, q, at, most, dev, top, ws, before = prepared(form, code, 50, 11)
    out, score = torch.full((q.shape[0], H, d), 7.0, dtype=torch.bfloat16, device=DEV), before.clone()
    st3.st3_block_attend(shape, q, at, most, dev.c, top, out, 50, score, ws)
    torch.cuda.synchronize()
    check(dev, q, old, new, 50, out, score, before, weight=TERMS)


@pytest.mark.parametrize("old", [0, 5, 63, 130, 700, 5000])
@pytest.mark.parametrize("H,Hk,d,code", [(8, 2, 128, "int8"), (7, 1, 64, "e4m3"), (32, 1, 128, "e4m3")])
def test_one_token_is_as_exact_as_a_decode_step(old, H, Hk, d, code):
    shape, q, at, most, dev, top, ws, before = run(np.random.default_rng(old + H), [old], [1], H, Hk, d, code, 1, pad=0)[2]
    for call in ("attend", "decode"):
        out, score = torch.full((1, H, d), 7.0, dtype=torch.bfloat16, device=DEV), before.clone()
        if call == "attend":
            st3.st3_block_attend(shape, q, at, most, dev.c, top, out, 1, score, ws)
        else:
            dev.set_len([old + 1])
            score[0, :, old] = 0.0                          # (a row that is no new one adds to what is there)
            dws = torch.empty(max(256, st3.st3_block_workspace_bytes(shape, old + 1)), dtype=torch.uint8, device=DEV)
            st3.st3_block_decode(shape, q, None, None, dev.c, old + 1, out, score, dws)
        torch.cuda.synchronize()
        check(dev, q, old, 1, 1, out, score, before, weight=TERMS)
