"""Scores of packed prompts where there are so many keys that the rows come through LDS in chunks: windows that end on, before and behind a chunk."""
import numpy as np
import pytest

from test_gpu_packed_attention import run

pytestmark = pytest.mark.gpu

MANY = 1024     # blocks of 64 keys, over all sequences at the bound's length, from which on rows go through LDS


@pytest.mark.parametrize("window", [1, 15, 16, 17, 32, 33, 64, 65, 130, 1000])
@pytest.mark.parametrize("G,d,dtype", [(1, 128, "bf16"), (4, 128, "bf16"), (3, 64, "bf16"), (1, 64, "f32"), (3, 128, "f32")])
def test_windows_around_the_chunks(window, G, d, dtype):
    Hk, lens = 29, [523, 1, 0, 257, 300]
    assert len(lens) * Hk * ((max(lens) + 63) // 64) > MANY
    run(np.random.default_rng(window + G), lens, Hk * G, Hk, d, dtype, window)


@pytest.mark.parametrize("layout", ["heads", "wide"])
def test_strides_of_the_rows(layout):
    Hk, lens = 33, [300, 64, 280, 5, 299, 77, 1]
    assert len(lens) * Hk * ((max(lens) + 63) // 64) > MANY
    run(np.random.default_rng(3), lens, 2 * Hk, Hk, 128, "bf16", 40, layout=layout)
