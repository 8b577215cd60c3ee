"""New tokens over a cache where a launch is cut differently, where memory is large, and where calls run side by side."""
from functools import partial

import numpy as np
import pytest
import torch

import test_gpu_block_append as append
import test_gpu_block_attend as attend
from block_util import BLOCK, DeviceCache, filled
from gpu_util import DEV, rand_values
from paper_2412_20105_amd import binding as st3

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("old,new", [([20000], [3]), ([20000], [40]), ([9000, 30], [2, 100])])
def test_many_more_rows_than_the_sequences_have(old, new):
    """A buffer for the largest batch, nearly empty: no room for as many parts as its length is worth."""
    attend.run(np.random.default_rng(old[0] + new[0]), old, new, 32, 8, 64, "int8", 3, pad=3000)


def test_parts_of_a_large_batch():
    """More sequences than a wave has lanes, empty and left out ones among them, whose rows lie in parts."""
    rng = np.random.default_rng(2)
    old = [int(x) for x in rng.integers(0, 1500, size=70)]
    new = [int(x) for x in rng.integers(9, 14, size=70)]
    for b in (0, 62, 63, 64, 65, 69):
        new[b] = 0
    old[3] = old[66] = -1
    attend.run(rng, old, new, 4, 1, 64, "e4m3", 4)


@pytest.mark.parametrize("old,new,B,H,Hk", [(1251, 8, 1, 8, 2), (1250, 3, 2, 4, 4), (1290, 3, 2, 4, 4), (600, 1, 65, 8, 4), (600, 5, 60, 16, 4), (100, 32, 2, 2, 2),
                                            (100, 33, 2, 2, 2), (5000, 16, 5, 4, 2), (1251, 9, 1, 8, 2),
                                            (600, 9, 3, 7, 1), (5000, 16, 2, 8, 2), (17000, 9, 2, 28, 4), (700, 13, 70, 15, 3), (1000, 65, 2, 3, 3), (2000, 4, 200, 2, 1), (17000, 1, 200, 1, 1)])
@pytest.mark.parametrize("window", [0, 2, 50])
def test_either_side_of_every_cut(old, new, B, H, Hk, window):
    """Few rows: by 4, 8 and 12 waves, whole and in pieces, with their logits in LDS and formed again, in one group and in two (which may part a token's
    heads)."""
    rng = np.random.default_rng(old + new + B)
    olds = [old] * B
    for b in range(1, B):
        olds[b] = int(rng.integers(-1, 200))
    attend.run(rng, olds, [new] * B, H, Hk, 64 if B > 100 else 128, "int8" if B % 2 else "e4m3", window)


@pytest.mark.parametrize("B,old,new,H,Hk,d", [(1, 70, 40, 8, 2, 128), (3, 10, 300, 16, 1, 128), (5, 2, 90, 12, 4, 64), (1, 3000, 17, 4, 1, 128),
                                              # (up to here no more than 256 blocks)
                                              (40, 150, 40, 8, 2, 128), (30, 200, 30, 32, 2, 64), (60, 5, 300, 16, 1, 128)])
@pytest.mark.parametrize("window", [5, 33, 1000])
def test_scores_of_few_blocks_and_of_many(B, old, new, H, Hk, d, window):
    """Windows of up to thousands of rows, which do not lie in LDS at once; a workgroup's waves with a block each, and with one together."""
    rng = np.random.default_rng(B + old)
    olds, news = [int(x) for x in rng.integers(0, old + 1, size=B)], [int(x) for x in rng.integers(1, new, size=B - 1)] + [new]
    attend.run(rng, olds, news, H, Hk, d, "int8" if d == 64 else "e4m3", window)


@pytest.mark.parametrize("old,new", [([200], [3]), ([130, 700], [4, 9]), ([20] * 110, [2] * 110)])
def test_values_that_are_not_finite_with_few_rows(old, new):
    attend.test_values_that_are_not_finite_reach_the_rows_that_see_them(old, new)


@pytest.mark.parametrize("new", [2, 40])
def test_pages_beyond_32_bits(monkeypatch, new):
    """Pools of more than 2^32 bytes, the pages in use at their end."""
    pages, blocks = 2 ** 19 + 200, 3 + 100 // BLOCK
    names = np.random.default_rng(3).permutation(np.arange(2 ** 19 + 10, 2 ** 19 + 190)).astype(np.int32)
    far = partial(filled, pages=pages)
    monkeypatch.setattr(append, "filled", lambda rng, lens, Hk, d, code, n: far(rng, lens, Hk, d, code, n, names=names[:len(lens) * n]))
    monkeypatch.setattr(attend, "filled", append.filled)
    append.run(np.random.default_rng(4), [100, 20], [new, 64], 1, 128, "int8", 64)
    attend.run(np.random.default_rng(5), [150, 70], [new, 1], 4, 1, 128, "int8", 2)


@pytest.mark.parametrize("new", [2, 40])
def test_strides_beyond_32_bits(new):
    """Rows that lie 2^31 elements apart between the first and the last."""
    rng, H, Hk, d = np.random.default_rng(6), 4, 1, 64
    out, score, (shape, q, at, most, dev, top, ws, before) = attend.run(rng, [100], [new], H, Hk, d, "e4m3", 2, pad=0)
    step = (2 ** 31 // (new - 1) + 64) // 8 * 8
    far = torch.empty((new - 1) * step + H * d, dtype=torch.bfloat16, device=DEV).as_strided((new, H, d), (step, d, 1))
    far.copy_(q)
    o, s = torch.zeros_like(out), before.clone()
    st3.st3_block_attend(shape, far, at, most, dev.c, top, o, 2, s, ws)
    assert torch.equal(o, out) and torch.equal(s, score)
    st3.st3_block_attend(shape, q, at, most, dev.c, top, far, 2, before.clone(), ws)
    assert torch.equal(far, out)
    cs = torch.from_numpy(append.angles(rng, new, 32)).to(DEV)
    want = torch.empty_like(out)
    st3.st3_rotate_rows(out, want, st3.rotary(cs))
    st3.st3_rotate_rows(far, far, st3.rotary(cs))
    assert torch.equal(far, want)
    # as keys and values of a cache, against the same rows side by side
    caches = []
    for rows in (far[:, :Hk], far[:, :Hk].contiguous()):
        c, _ = filled(np.random.default_rng(7), [50], Hk, d, "e4m3", 3, names=np.int32([2, 0, 1]))
        c.k_tail.nan_to_num_(nan=0.0), c.v_tail.nan_to_num_(nan=0.0)
        st3.st3_block_append(shape, rows, rows, at, most, c.c, 50 + new, st3.rotary(cs))
        caches.append(c)
    full = torch.tensor([2], device=DEV)[:(50 + new) // BLOCK]
    for name in ("k_tail", "v_tail"):
        assert torch.equal(getattr(caches[0], name), getattr(caches[1], name))
    for name in ("k_codes", "v_codes", "k_scale", "v_scale"):
        assert torch.equal(getattr(caches[0], name)[full], getattr(caches[1], name)[full])


@pytest.mark.parametrize("new", [2, 20, 40])
def test_a_long_batch_is_its_sequences_alone(new):
    """Waves that walk up to 64 blocks for the scores, and few: the same sums."""
    rng, B, Hk, H, d = np.random.default_rng(11), 4, 8, 16, 128
    old = [130000, 129990, 100000, 64]
    blocks = (max(old) + new) // BLOCK + 1
    dev = DeviceCache(rng, B, Hk, d, "int8", blocks, pages=B * blocks)
    for x in (dev.k_scale, dev.v_scale):
        x.copy_(torch.rand(x.shape, device=DEV) * 0.02 + 0.001)
    for x in (dev.k_tail, dev.v_tail):
        x.copy_(torch.randn(x.shape, device=DEV))
    dev.set_len(old)
    q = torch.from_numpy(rand_values(rng, (B * new, H, d), "bf16", 1.0)).to(DEV).bfloat16()
    top = max(old) + new

    def go(tokens, c, batch):
        shape, out, score = st3.gqa_shape(batch, H, Hk, d), torch.empty_like(tokens), torch.zeros((batch, Hk, top), device=DEV)
        cu = torch.arange(0, batch * new + 1, new, dtype=torch.int32, device=DEV)
        ws = torch.empty(st3.st3_block_attend_workspace_bytes(shape, batch * new, new, top), dtype=torch.uint8, device=DEV)
        st3.st3_block_attend(shape, tokens, cu, new, c, top, out, new, score, ws)
        torch.cuda.synchronize()
        return out.double(), score.double()

    out, score = go(q, dev.c, B)
    v_most = float(dev.v_scale.max()) * 128 + float(dev.v_tail.abs().max())
    for b in range(B):
        c = st3.block_cache(dev.k_codes, dev.v_codes, dev.k_scale, dev.v_scale, dev.k_tail[b:b + 1], dev.v_tail[b:b + 1], dev.table[b:b + 1], dev.len[b:b + 1])
        o, s = go(q[b * new:(b + 1) * new], c, 1)
        # either sum of up to `top` weights in float32, in another order
        assert bool(((score[b] - s[0]).abs() <= 2 * (top + 32) * 2.0 ** -24 * s[0] + 1e-30).all())
        assert float((score[b, :, :old[b] + new].sum(-1) / (new * H // Hk) - 1).abs().max()) <= 2 * (top + 32) * 2.0 ** -24
        assert not score[b, :, old[b] + new:].any()
        assert bool(((out[b * new:(b + 1) * new] - o).abs() <= 2 * attend.HALF * 1.01 * (o.abs() + v_most)).all())


def test_two_at_once_and_two_graphs():
    """Calls on two streams, and two graphs, with workspaces of their own."""
    rng = np.random.default_rng(8)
    sets = [attend.run(rng, old, new, 8, 2, 128, "int8", 8) for old, new in (([6000, 50], [40, 200]), ([9000], [6]))]
    outs, scores, graphs = [torch.empty_like(o) for o, _, _ in sets], [s.clone() for _, s, _ in sets], []

    def call(i, stream=None):
        shape, q, at, most, dev, top, ws, before = sets[i][2]
        st3.st3_block_attend(shape, q, at, most, dev.c, top, outs[i], 8, scores[i], ws, stream)

    def check():
        torch.cuda.synchronize()
        for i, (o, s, _) in enumerate(sets):
            T = sets[i][2][2].tolist()[-1]
            assert torch.equal(outs[i][:T], o[:T]) and torch.equal(scores[i], s)

    def clear():
        for i in range(2):
            outs[i].zero_()
            scores[i].copy_(sets[i][2][-1])
        torch.cuda.synchronize()

    side = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        clear()
        for i in (0, 1):
            call(i, side[i])
        check()
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(i)
    for _ in range(4):
        clear()
        for i in (0, 1):
            with torch.cuda.stream(side[i]):
                graphs[i].replay()
        check()


def test_several_pieces_give_what_one_call_gives():
    """Appended and attended in two calls, the weights of the last rows are those of one."""
    rng, Hk, H, d, n, m = np.random.default_rng(9), 2, 8, 128, 300, 90
    k, v, q = (torch.from_numpy(rand_values(rng, (m, h, d), "bf16", 1.5)).to(DEV).bfloat16() for h in (Hk, Hk, H))
    shape, results = st3.gqa_shape(1, H, Hk, d), []
    for cuts in ([0, m], [0, 50, m]):
        dev, _ = filled(np.random.default_rng(10), [n], Hk, d, "int8", 8)
        out, score = torch.empty_like(q), torch.zeros((1, Hk, n + m), device=DEV)
        for a, b in zip(cuts, cuts[1:]):
            dev.set_len([n + a])
            cu = torch.tensor([0, b - a], dtype=torch.int32, device=DEV)
            st3.st3_block_append(shape, k[a:b], v[a:b], cu, b - a, dev.c, n + b)
            ws = torch.empty(st3.st3_block_attend_workspace_bytes(shape, b - a, b - a, n + b), dtype=torch.uint8, device=DEV)
            st3.st3_block_attend(shape, q[a:b], cu, b - a, dev.c, n + b, out[a:b], 4 if b == m else 0, score if b == m else None, ws)
        results.append((out, score))
    # Rows below the first cut differ: they see their block as bf16 rows then, as codes here.  The rest see the same cache; either side rounds its weights,
    # relative to a reference point of its own, and its output, so each is off by half a step of |out| + sum p |v|, which is at most the largest |v|.
    one, two = (r[0][50:].double() for r in results)
    v_most = max(float(v.abs().max()), float((dev.v_scale[dev.table[0, :(n + m) // BLOCK].long()] * 127).max()))
    assert bool(((one - two).abs() <= 2 * attend.HALF * 1.01 * (one.abs() + v_most)).all())
    # sums of 4 x 4 weights of at most 1 in float32, each within a slack far below 2^-16
    assert float((results[0][1] - results[1][1]).abs().max()) <= 2 * 16 * 2.0 ** -16


@pytest.mark.parametrize("pairs", [8, 24, 40, 64])
@pytest.mark.parametrize("more", [0, 1, 13])
def test_a_large_table_is_that_of_its_halves(pairs, more):
    rng = np.random.default_rng(12)
    T = 2 ** 20 // pairs + more                     # (from 2^20 pairs on threads make several tokens)
    positions = torch.from_numpy(rng.integers(-1000, 200000, (2, T)).astype(np.int32)).to(DEV)
    f, axis = torch.rand(pairs, device=DEV), rng.integers(0, 2, pairs).tolist()
    whole, halves = (torch.full((T + 70, pairs, 2), 7.0, device=DEV) for _ in range(2))
    st3.st3_rotary_table(positions, f, axis, whole[:T])
    for a, b in ((0, T // 2), (T // 2, T)):
        st3.st3_rotary_table(positions[:, a:b], f, axis, halves[a:b])
    assert torch.equal(whole, halves) and bool((whole[T:] == 7.0).all()) and not bool((whole[:T] == 7.0).any())


def test_components_that_are_all_the_same():
    """One row of positions stretched over the axes, without a copy: the table of one axis."""
    pos, f = torch.arange(50, 117, dtype=torch.int32, device=DEV), torch.rand(32, device=DEV)
    one, three = (torch.zeros((67, 32, 2), device=DEV) for _ in range(2))
    st3.st3_rotary_table(pos, f, None, one)
    st3.st3_rotary_table(pos.expand(3, 67), f, [c % 3 for c in range(32)], three)
    assert torch.equal(one, three)
