"""Which rows an eviction keeps where many scores share their leading bits: bins that hold just as many rows as are counted directly, one more, ties in them."""
import numpy as np
import pytest
import torch

from gpu_util import DEV
from block_util import BLOCK, DeviceCache, filled
from paper_2412_20105_amd import binding as st3

pytestmark = pytest.mark.gpu


def kept_rows(score, n, keep, n_sink, n_recent):
    """By the definition: a stable sort, greatest first, a NaN last."""
    mid = np.arange(n_sink, n - n_recent)
    s = score[mid] + 0.0                                    # (-0 is 0)
    order = np.lexsort((mid, -np.where(np.isnan(s), 0, s), np.isnan(s)))
    return np.sort(np.concatenate([np.arange(n_sink), mid[order[:keep - n_sink - n_recent]], np.arange(n - n_recent, n)]))


def check(rng, lens, score, keep, n_sink=0, n_recent=0):
    B, Hk, top = score.shape
    dev, _ = filled(rng, [BLOCK] * B, Hk, 64, "int8", top // BLOCK + 1, pages=B * (top // BLOCK + keep // BLOCK + 3))
    dev.set_len(lens)
    to = DeviceCache(rng, B, Hk, 64, "int8", max(keep // BLOCK, 1), pool=dev)
    dev.table[:, 1:] = dev.table[:, :1]                     # (which values move does not matter here)
    s = torch.from_numpy(score.astype(np.float32)).to(DEV)
    kept = torch.full((B, Hk, keep), 77, dtype=torch.int32, device=DEV)
    t = torch.full((B, Hk, keep), -5.0, device=DEV)
    st3.st3_block_evict(st3.gqa_shape(B, Hk, Hk, 64), dev.c, to.c, max(lens), keep, n_sink, n_recent, s, t, kept)
    torch.cuda.synchronize()
    for b, n in enumerate(lens):
        for h in range(Hk):
            want = kept_rows(score[b, h].astype(np.float32), n, keep, n_sink, n_recent)
            np.testing.assert_array_equal(kept[b, h].cpu().numpy(), want, err_msg=f"{b} {h}")
            np.testing.assert_array_equal(t[b, h].cpu().numpy(), score[b, h, want].astype(np.float32))


@pytest.mark.parametrize("n", [700, 1200, 4096, 4097, 8192, 9000, 16384, 17000, 32768])
@pytest.mark.parametrize("many", [1, 127, 128, 129, 500])
def test_scores_that_share_their_leading_bits(n, many):
    """`many` scores in [1, 1 + 2^-10), all others above or below; keep so many that the last row kept is among them."""
    rng = np.random.default_rng(n + many)
    score = np.zeros((1, 4, n))
    for h, step in enumerate((2.0 ** -23, 2.0 ** -20, 2.0 ** -13, 0.0)):     # all different, some alike, few different, all the same
        close = 1.0 + rng.permutation(many) % 1024 * step
        above = 100
        rest = np.concatenate([close, rng.uniform(2, 9, above), rng.uniform(0, 0.9, n - many - above)])
        score[0, h] = rng.permutation(rest)
    check(rng, [n], score, 100 + (many + 1) // 2)
    check(rng, [n], score, 100 + many)
    check(rng, [n], score, 101)


@pytest.mark.parametrize("n", [300, 3000, 6000])
def test_scores_of_every_kind(n):
    rng = np.random.default_rng(n)
    score = np.stack([rng.normal(size=n), rng.exponential(size=n) * 1e-40, np.where(rng.random(n) < 0.5, -0.0, 0.0), np.full(n, np.nan),
                      np.where(rng.random(n) < 0.3, np.inf, -np.inf), np.where(rng.random(n) < 0.3, np.nan, rng.normal(size=n))])[None]
    for keep, first, last in ((n // 3, 4, 20), (n - 1, 0, 0), (150, 75, 75), (1, 0, 0)):
        check(rng, [n], score, keep, first, last)


@pytest.mark.parametrize("n,keep", [(16385, 16000), (30000, 20000), (33000, 16500), (40000, 300), (40000, 39990)])
def test_long_sequences_in_place(n, keep):
    """More rows than a workgroup holds at a time, scores written over those that are read; ties everywhere."""
    rng = np.random.default_rng(n + keep)
    score = rng.integers(0, 50, size=(2, 2, n)) / 8.0
    score[1, 1] = 1.0
    lens = [n, n - 700]
    dev, _ = filled(rng, [BLOCK] * 2, 2, 64, "int8", n // BLOCK + 1, pages=2 * (n // BLOCK + keep // BLOCK + 3))
    dev.set_len(lens)
    to = DeviceCache(rng, 2, 2, 64, "int8", keep // BLOCK, pool=dev)
    dev.table[:, 1:] = dev.table[:, :1]
    s = torch.from_numpy(score.astype(np.float32)).to(DEV)
    kept = torch.full((2, 2, keep), 77, dtype=torch.int32, device=DEV)
    st3.st3_block_evict(st3.gqa_shape(2, 2, 2, 64), dev.c, to.c, n, keep, 5, 60, s, s, kept)
    torch.cuda.synchronize()
    for b, m in enumerate(lens):
        for h in range(2):
            want = np.arange(m) if m <= keep else kept_rows(score[b, h].astype(np.float32), m, keep, 5, 60)
            got = kept[b, h].cpu().numpy()
            np.testing.assert_array_equal(got[:len(want)], want, err_msg=f"{b} {h}")
            assert (got[len(want):] == -1).all()
            np.testing.assert_array_equal(s[b, h, :len(want)].cpu().numpy(), score[b, h, want].astype(np.float32))


def test_scores_beside_each_other_in_one_buffer():
    rng = np.random.default_rng(8)
    n, keep, B, Hk = 300, 130, 2, 3
    dev, _ = filled(rng, [BLOCK] * B, Hk, 64, "int8", n // BLOCK + 1, pages=B * (n // BLOCK + keep // BLOCK + 3))
    dev.set_len([n] * B)
    to = DeviceCache(rng, B, Hk, 64, "int8", keep // BLOCK, pool=dev)
    dev.table[:, 1:] = dev.table[:, :1]
    score = rng.exponential(size=(B, Hk, n))
    both = torch.full((B, Hk, n + keep), -5.0, device=DEV)
    both[..., :n] = torch.from_numpy(score.astype(np.float32)).to(DEV)
    kept = torch.full((B, Hk, keep), 77, dtype=torch.int32, device=DEV)
    st3.st3_block_evict(st3.gqa_shape(B, Hk, Hk, 64), dev.c, to.c, n, keep, 4, 10, both[..., :n], both[..., n:], kept)
    torch.cuda.synchronize()
    for b in range(B):
        for h in range(Hk):
            want = kept_rows(score[b, h].astype(np.float32), n, keep, 4, 10)
            np.testing.assert_array_equal(kept[b, h].cpu().numpy(), want)
            np.testing.assert_array_equal(both[b, h, n:].cpu().numpy(), score[b, h, want].astype(np.float32))
            np.testing.assert_array_equal(both[b, h, :n].cpu().numpy(), score[b, h].astype(np.float32))
