"""Turns whose rows' attention does not count as weight: the pieces of a prompt before its last."""
import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from paper_2412_20105_amd import binding as st3
from paper_2412_20105_amd.block_pipeline import BlockGeneration


def test_rows_of_a_turn_that_does_not_count_begin_with_no_weight():
    gen = BlockGeneration.__new__(BlockGeneration)          # (no GPU: up to the library's first call)
    gen.L, gen.B, gen.capacity, gen.budget, gen.device = 2, 4, 256, 128, "cpu"
    gen.lens, gen.shape, gen._turn_ws = [20, -1, 30, 0], st3.gqa_shape(4, 8, 2, 128), torch.empty(0, dtype=torch.uint8)
    gen.len, gen.live = torch.tensor(gen.lens, dtype=torch.int32), torch.tensor([1, 0, 1, 1], dtype=torch.int32)
    gen.score = torch.rand((2, 4, 2, 256)) + 1
    want = gen.score.clone()
    gen.begin_turn([7, 0, 100, 0])
    assert torch.equal(gen.score, want) and gen.counts
    gen.finish_turn()
    gen.begin_turn([0, 0, 0, 0], counts=False)
    assert torch.equal(gen.score, want)
    gen.finish_turn()
    gen.begin_turn([5, 0, 60, 3], counts=False)
    want[:, 0, :, 27:32] = want[:, 2, :, 130:190] = want[:, 3, :, :3] = 0.0
    assert torch.equal(gen.score, want) and not gen.counts
    gen.finish_turn()
    assert gen.lens == [32, -1, 190, 3]


@pytest.mark.gpu
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_weights_of_a_prompt_do_not_hang_on_its_pieces(code):
    """Two layers, two sequences, the last piece the same: weights of the prompt's last `window` rows, against the oracle, and the rows that an eviction keeps."""
    from block_util import fp32_slack
    from gpu_util import DEV, rand_values, to_np64
    rng = np.random.default_rng(4)
    L, H, Hk, d, window, lens, last = 2, 8, 2, 128, 8, (300, 170), (40, 33)
    x = [[rand_values(rng, (n, H + 2 * Hk, d), "bf16", 1.0) for n in lens] for _ in range(L)]
    cuts = ([(260, 137)], [(100, 0), (1, 70), (63, 67), (96, 0)], [(130, 64), (130, 73)])
    scores, kept = [], []
    for pieces in cuts:
        gen = BlockGeneration(L, H, Hk, d, 2, 512, 100, 2, 4, window, {"int8": st3.ST3_BLOCK_INT8, "e4m3": st3.ST3_BLOCK_E4M3}[code])
        gen.score.fill_(float("nan"))                       # (whatever an earlier batch left)
        gen.begin([0, 0])
        at = [0, 0]
        for i, new in enumerate([*pieces, last]):
            gen.begin_turn(new, counts=i == len(pieces))
            for l in range(L):
                rows = torch.from_numpy(np.concatenate([x[l][b][at[b]:at[b] + new[b]] for b in range(2)])).to(DEV).bfloat16()
                gen.extend_layer(l, rows[:, :H], rows[:, H:H + Hk], rows[:, H + Hk:])
            gen.finish_turn()
            at = [a + m for a, m in zip(at, new)]
        assert tuple(at) == lens
        scores.append([[to_np64(gen.score[l, b, :, :n]) for b, n in enumerate(lens)] for l in range(L)])
        gen.evict()
        kept.append(gen.kept.clone())
    for l in range(L):
        for b, n in enumerate(lens):
            ref = bo.BlockCache(1, Hk, d, code)
            q, k, v = (np.asarray(y, np.float64) for y in (x[l][b][:, :H], x[l][b][:, H:H + Hk], x[l][b][:, H + Hk:]))
            first = n - last[b]
            for h in range(Hk):
                ref.append(0, h, k[:first, h], v[:first, h])
            weights = bo.extend(ref, 0, q[first:], k[first:], v[first:], 1 / np.sqrt(d), window)[1]
            worst = float((np.abs(q).max() * np.abs(k).max()) * d / np.sqrt(d))
            for got in scores:
                assert np.all(np.abs(got[l][b] - weights) <= 2 * fp32_slack(worst, d, n) * weights + 1e-30)
                assert np.array_equal(got[l][b], scores[0][l][b])       # (the same cache, bit for bit, and the same call)
    assert all(torch.equal(k, kept[0]) for k in kept)
