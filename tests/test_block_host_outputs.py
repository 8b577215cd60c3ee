"""Outputs whose rows lie on each other (no GPU: refused before the launch; what is not is told by a refusal that comes later)."""
import pytest

from paper_2412_20105_amd import binding as st3
from test_block_host import FAKE, INVALID, SMALL, cache, packed, rows, shape

FAR = FAKE + (1 << 30)

# strides (of rows, of heads) of an output of 8 heads of 128: (100, or 2, rows of them)
ON_EACH_OTHER = [(128, 128), (256, 128), (1016, 128), (512, 256), (128, 1024), (1024, 256)]
APART = [(1024, 128), (2048, 128), (2048, 256), (1032, 128)]


def decode(out, **more):
    return st3.lib().st3_block_decode(shape(**more), rows(), rows(2 * FAR), rows(3 * FAR), cache(), 50, out, None, 0, 0, FAKE, 0, None)


@pytest.mark.parametrize("strides", ON_EACH_OTHER, ids=str)
def test_packed_attention_refuses(strides):
    assert packed(out=rows(FAR, *strides)) == INVALID
    assert packed(out=rows(FAR, *strides), wb=0) == INVALID


@pytest.mark.parametrize("strides", [*APART, (128, 128 * 100), (256, 256 * 100), (128, 128 * 100 + 8)], ids=str)
def test_packed_attention_takes(strides):
    assert packed(out=rows(FAR, *strides), wb=0) == SMALL


@pytest.mark.parametrize("strides", [*ON_EACH_OTHER[:4], (128, 128 + 8), (1024, 256)], ids=str)
def test_decode_refuses(strides):
    assert decode(rows(FAR, *strides)) == INVALID


@pytest.mark.parametrize("strides", [*APART, (128, 256), (256, 512)], ids=str)
def test_decode_takes(strides):
    assert decode(rows(FAR, *strides)) == SMALL


def test_one_sequence_or_one_head_has_no_stride():
    assert decode(rows(FAR, 128, 128), batch=1) == SMALL and decode(rows(FAR, 128, 128), heads=1, kv_heads=1) == SMALL
    assert decode(rows(FAR, 1024, 120), batch=1) == INVALID


def test_inputs_may_lie_on_each_other():
    """Keys that several heads or rows share are read alone."""
    assert packed(k=rows(FAKE, 128, 128), v=rows(FAKE, 128, 128), wb=0) == SMALL
