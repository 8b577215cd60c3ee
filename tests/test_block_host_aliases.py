"""Refusals of buffers that share memory where a call writes what another part of it still reads (no GPU: all of them come before the launch)."""
import ctypes as C

import pytest

from paper_2412_20105_amd import binding as st3
from test_block_host import FAKE, INVALID, cache, rows, shape

FAR = FAKE + (1 << 30)


def decode(k, v, out):
    return st3.lib().st3_block_decode(shape(), rows(FAR, 1024, 128), k, v, cache(), 50, out, None, 0, 0, FAKE, 1 << 30, None)


@pytest.mark.parametrize("out", [rows(FAKE), rows(FAKE + 256), rows(FAKE + 2048), rows(FAKE - 2 * 1024 * 2 + 16)], ids=["same", "a row on", "second sequence", "last row"])
@pytest.mark.parametrize("which", ["k", "v"])
def test_decode_refuses_an_output_on_the_new_rows(out, which):
    new, far = rows(FAKE, 1024, 128), rows(2 * FAR, 1024, 128)
    assert decode(new if which == "k" else far, far if which == "k" else new, out) == INVALID


def evict(score, sb, sh, to_score, tb, th, top=50, keep=20):
    return st3.lib().st3_block_evict(shape(), cache(), cache(k_tail=1 << 40, v_tail=1 << 41), top, keep, 0, 0, score, sb, sh, to_score, tb, th, FAKE, 20, 20, None)


@pytest.mark.parametrize("args", [
    (FAKE, 200, 100, FAKE + 4, 200, 100), (FAKE, 200, 100, FAKE + 4 * 49, 200, 100), (FAKE + 4 * 19, 200, 100, FAKE, 200, 100),
    (FAKE, 200, 100, FAKE, 200, 90), (FAKE, 200, 100, FAKE + 4 * 100, 200, 100), (FAKE, 100, 50, FAKE + 4 * 90, 40, 20)], ids=str)
def test_evict_refuses_scores_that_overlap(args):
    assert evict(*args) == INVALID
