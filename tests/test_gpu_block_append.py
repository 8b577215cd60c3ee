"""st3_block_append against the oracle's cache, bit for bit."""
import numpy as np
import pytest
import torch

from block_util import BLOCK, DeviceCache, bf16, filled
from gpu_util import DEV, rand_values, to_np64
from oracle import block_oracle as bo
from paper_2412_20105_amd import binding as st3

pytestmark = pytest.mark.gpu


def angles(rng, T, pairs):
    a = rng.uniform(0, 2 * np.pi, (T, pairs))
    return np.stack([np.cos(a), np.sin(a)], -1).astype(np.float32)


def new_rows(rng, new, Hk, d, layout="fused"):
    T = sum(new)
    rows = rand_values(rng, (T, 2 * Hk + 1, d), "bf16", 1.5)
    dev = torch.from_numpy(rows).to(DEV).bfloat16()
    k, v = dev[:, :Hk], dev[:, Hk:2 * Hk]
    if layout == "heads":
        k, v = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (k, v))
    return rows[:, :Hk], rows[:, Hk:2 * Hk], k, v


def run(rng, old, new, Hk, d, code, pairs=0, adjacent=False, layout="fused", max_len=None, max_new=None):
    """Through the binding and against the oracle."""
    blocks = (max(old) + max(new)) // BLOCK + 2
    dev, ref = filled(rng, [max(n, 0) for n in old], Hk, d, code, blocks)
    dev.set_len(old)
    kn, vn, k, v = new_rows(rng, new, Hk, d, layout)
    rotary = None
    if pairs:
        cs = angles(rng, sum(new), pairs)
        kn = bf16(bo.rotate(kn, cs, adjacent))
        rotary = st3.rotary(torch.from_numpy(cs).to(DEV), int(adjacent))
    shape = st3.gqa_shape(len(old), Hk, Hk, d)
    cu = torch.tensor([0, *np.cumsum(new)], dtype=torch.int32, device=DEV)
    st3.st3_block_append(shape, k, v, cu, max(new) if max_new is None else max_new, dev.c,
                         max(n + m for n, m in zip(old, new)) if max_len is None else max_len, rotary)
    torch.cuda.synchronize()
    start = 0
    for b, (n, m) in enumerate(zip(old, new)):
        for h in range(Hk):
            if n >= 0:
                ref.append(b, h, np.asarray(kn[start:start + m, h], np.float64), np.asarray(vn[start:start + m, h], np.float64))
        start += m
    dev.check(ref)
    assert dev.len.tolist() == old
    return dev, ref


SIZES = [([0], [1]), ([0], [64]), ([0], [65]), ([63], [1]), ([63], [2]), ([64], [63]), ([1], [130]), ([10, 0, 64, 100], [54, 7, 64, 0]),
         ([70, -1, 5], [0, 9, 200]), ([127] * 3, [1, 2, 66]), ([5] * 70, [3] * 70), ([300, 20], [1, 500])]


@pytest.mark.parametrize("old,new", SIZES, ids=lambda x: "-".join(map(str, x[:5])))
@pytest.mark.parametrize("Hk,d", [(1, 64), (8, 128), (3, 128)])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_appended_rows(old, new, Hk, d, code):
    run(np.random.default_rng(sum(new) + d), old, new, Hk, d, code)


@pytest.mark.parametrize("old,new", [([0], [1]), ([63, 10], [2, 140]), ([64, 30, -1], [64, 5, 3])], ids=lambda x: "-".join(map(str, x)))
@pytest.mark.parametrize("d,pairs", [(64, 32), (64, 16), (64, 8), (128, 64), (128, 24), (128, 40), (128, 8)])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_keys_turned_on_the_way(old, new, d, pairs, adjacent, code):
    run(np.random.default_rng(sum(new) + pairs), old, new, 4, d, code, pairs, adjacent, ["fused", "heads"][pairs // 8 % 2])


@pytest.mark.parametrize("seed", range(20))
def test_random_batches(seed):
    rng = np.random.default_rng(500 + seed)
    B, d = int(rng.integers(1, 7)), int(rng.choice([64, 128]))
    old = [int(x) - 1 for x in np.exp(rng.uniform(0, np.log(400), B))]
    new = [int(x) - 1 for x in np.exp(rng.uniform(0, np.log(300), B))]
    new[-1] += 1
    run(rng, old, new, int(rng.integers(1, 6)), d, ["int8", "e4m3"][seed % 2], int(rng.choice([0, d // 2, 8])), bool(seed // 2 % 2), max_len=max(old) + max(new),
        max_new=max(new) + 9 if sum(new) > max(new) + 9 else None)


@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_any_way_of_cutting_gives_the_same_cache(code):
    """At once, in pieces, through the store, and the last rows one by one through decode."""
    rng = np.random.default_rng(9)
    lens, Hk, d, pairs = [200, 131], 2, 128, 32
    kn, vn, k, v = new_rows(rng, lens, Hk, d)
    table = torch.from_numpy(angles(rng, sum(lens), pairs)).to(DEV)
    shape = st3.gqa_shape(2, Hk, Hk, d)
    turned = torch.empty_like(k)
    st3.st3_rotate_rows(k, turned, st3.rotary(table))
    caches = [DeviceCache(np.random.default_rng(1), 2, Hk, d, code, 4) for _ in range(4)]
    cu = torch.tensor([0, 200, 331], dtype=torch.int32, device=DEV)
    st3.st3_block_append(shape, k, v, cu, 200, caches[0].c, 200, st3.rotary(table))
    st3.st3_block_store(shape, turned, v, cu, 200, caches[1].c)
    done, ws = [0, 0], torch.empty(st3.st3_block_workspace_bytes(shape, 200), dtype=torch.uint8, device=DEV)
    starts = [0, 200]
    for cut in ([10, 70], [50, 2], [4, 0], [130, 59], [6, 0]):      # to 64, 128, and inside
        rows = torch.cat([torch.arange(starts[b] + done[b], starts[b] + done[b] + cut[b]) for b in range(2)]).to(DEV)
        part = torch.tensor([0, cut[0], sum(cut)], dtype=torch.int32, device=DEV)
        caches[2].set_len(done)
        st3.st3_block_append(shape, k[rows], v[rows], part, max(cut), caches[2].c, max(n + m for n, m in zip(done, cut)), st3.rotary(table[rows]))
        done = [n + m for n, m in zip(done, cut)]
    assert done == lens
    out = torch.empty((2, Hk, d), dtype=torch.bfloat16, device=DEV)
    part = torch.tensor([0, 60, 60], dtype=torch.int32, device=DEV)
    st3.st3_block_append(shape, k[:60], v[:60], part, 60, caches[3].c, 60, st3.rotary(table[:60]))
    for i in range(140):
        now = [60 + i, i if i < 131 else -1]
        caches[3].set_len(now)
        rows = torch.tensor([60 + i, 200 + min(i, 130)], device=DEV)
        st3.st3_block_decode(shape, turned[rows], turned[rows], v[rows], caches[3].c, max(now), out, None, ws)
    torch.cuda.synchronize()
    ref = bo.BlockCache(2, Hk, d, code)
    t = to_np64(turned)
    for b, s in enumerate(starts):
        for h in range(Hk):
            ref.append(b, h, t[s:s + lens[b], h], vn[s:s + lens[b], h].astype(np.float64))
    for c in caches:
        c.check(ref)


def snapshot(dev):
    return [t.clone() for t in (dev.k_codes, dev.v_codes, dev.k_scale.view(torch.int32), dev.v_scale.view(torch.int32), dev.k_tail.view(torch.int16),
                                dev.v_tail.view(torch.int16), dev.len)]


def test_nothing_else_is_written():
    """Pages, scales and tail rows that the new rows do not touch keep their bits, empty places and sequences without new rows all of theirs."""
    rng = np.random.default_rng(10)
    old, new, Hk, d = [70, -1, 30, 64], [60, 5, 0, 10], 2, 64
    dev, ref = filled(rng, [70, 0, 30, 64], Hk, d, "int8", 4)
    dev.set_len(old)
    before = snapshot(dev)
    kn, vn, k, v = new_rows(rng, new, Hk, d)
    cu = torch.tensor([0, 60, 65, 65, 75], dtype=torch.int32, device=DEV)
    st3.st3_block_append(st3.gqa_shape(4, Hk, Hk, d), k, v, cu, 60, dev.c, 130)
    after = snapshot(dev)
    page = int(dev.table[0, 1])         # the one block that is whole now
    same = torch.arange(len(dev.k_codes), device=DEV) != page
    for a, b in list(zip(before, after))[:4]:
        assert torch.equal(a[same], b[same]) and not torch.equal(a[page], b[page])
    assert torch.equal(before[4][1:3], after[4][1:3]) and torch.equal(before[5][1:3], after[5][1:3])
    # (two rows are the tail of the first one now)
    assert torch.equal(before[4][0, :, 2:], after[4][0, :, 2:]) and torch.equal(before[4][3, :, 10:], after[4][3, :, 10:])
    assert torch.equal(before[5][0, :, :, 2:], after[5][0, :, :, 2:]) and torch.equal(before[5][3, :, :, 10:], after[5][3, :, :, 10:])


@pytest.mark.parametrize("bad", [-1, 10 ** 6])
def test_a_block_without_a_page_is_not_written(bad):
    rng = np.random.default_rng(11)
    old, new, Hk, d = [40, 10], [120, 130], 2, 128
    dev, ref = filled(rng, old, Hk, d, "e4m3", 4)
    dev.table[0, 1] = bad
    before = snapshot(dev)
    kn, vn, k, v = new_rows(rng, new, Hk, d)
    cu = torch.tensor([0, 120, 250], dtype=torch.int32, device=DEV)
    st3.st3_block_append(st3.gqa_shape(2, Hk, Hk, d), k, v, cu, 130, dev.c, 160)
    start = 0
    for b, (n, m) in enumerate(zip(old, new)):
        for h in range(Hk):
            ref.append(b, h, kn[start:start + m, h].astype(np.float64), vn[start:start + m, h].astype(np.float64))
            if b == 0:
                ref.blocks[b][h] = ref.blocks[b][h][:1]
        start += m
    dev.check(ref)                      # the block before, the tail, and the other sequence
    used = {int(dev.table[0, 0]), int(dev.table[1, 0]), int(dev.table[1, 1])}
    same = torch.tensor([i not in used for i in range(len(dev.k_codes))], device=DEV)
    assert all(torch.equal(a[same], b[same]) for a, b in list(zip(before, snapshot(dev)))[:4])


def test_lengths_that_lie_are_cut():
    rng = np.random.default_rng(12)
    Hk, d = 2, 64
    got = []
    # (the second sequence has 17 new rows in all of these: of 30, those that its bound, max_new or max_len leaves; one of 300 rows has none)
    for cu, n, max_new, max_len in (([0, 20, 37], [5, 64], 20, 90), ([-7, 20, 37], [5, 64], 30, 90), ([0, 20, 900], [5, 64], 30, 81), ([0, 17, 17], [5, 300], 17, 90),
                                    ([0, 17, 50], [5, 300], 30, 90)):
        dev, _ = filled(np.random.default_rng(2), [5, 64], Hk, d, "int8", 4)
        dev.set_len(n)
        _, _, k, v = new_rows(np.random.default_rng(3), [20, 30], Hk, d)
        st3.st3_block_append(st3.gqa_shape(2, Hk, Hk, d), k, v, torch.tensor(cu, dtype=torch.int32, device=DEV), max_new, dev.c, max_len)
        got.append([t.view(torch.int16).clone() for t in (dev.k_tail, dev.v_tail)])
    for first, g in ((0, 1), (0, 2), (3, 4)):
        assert all(torch.equal(a, b) for a, b in zip(got[first], got[g]))


def test_values_that_are_not_finite():
    """Infinities saturate, NaN as the format says; a turned infinity is one, or NaN."""
    rng = np.random.default_rng(13)
    Hk, d, pairs = 1, 64, 16
    for code in ("int8", "e4m3"):
        dev, ref = filled(rng, [30], Hk, d, code, 3)
        kn, vn, k, v = new_rows(rng, [60], Hk, d)
        for x, at in ((k, (3, 0, 5)), (k, (50, 0, 40)), (v, (7, 0, 9)), (v, (59, 0, 63))):
            x[at] = float(rng.choice([np.inf, -np.inf, np.nan]))
        cs = angles(rng, 60, pairs)
        st3.st3_block_append(st3.gqa_shape(1, 1, 1, d), k, v, torch.tensor([0, 60], dtype=torch.int32, device=DEV), 60, dev.c, 90,
                             st3.rotary(torch.from_numpy(cs).to(DEV)))
        turned = torch.empty_like(k)
        st3.st3_rotate_rows(k, turned, st3.rotary(torch.from_numpy(cs).to(DEV)))
        ref.append(0, 0, to_np64(turned)[:, 0], to_np64(v)[:, 0])
        dev.check(ref)


def test_captured_into_a_graph():
    rng = np.random.default_rng(14)
    Hk, d, old, new = 2, 128, [70, 10], [80, 40]
    kn, vn, k, v = new_rows(rng, new, Hk, d)
    table = torch.from_numpy(angles(rng, 120, 64)).to(DEV)
    dev, _ = filled(np.random.default_rng(4), old, Hk, d, "int8", 5)
    first = snapshot(dev)
    shape, cu = st3.gqa_shape(2, Hk, Hk, d), torch.tensor([0, 80, 120], dtype=torch.int32, device=DEV)
    rotary = st3.rotary(table)
    def restore():
        for t, s in zip((dev.k_codes, dev.v_codes, dev.k_scale.view(torch.int32), dev.v_scale.view(torch.int32), dev.k_tail.view(torch.int16),
                         dev.v_tail.view(torch.int16), dev.len), first):
            t.copy_(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st3.st3_block_append(shape, k, v, cu, 110, dev.c, 150, rotary)
    for i in range(4):
        if i == 2:
            cu.copy_(torch.tensor([0, 10, 120], dtype=torch.int32))
        restore()
        st3.st3_block_append(shape, k, v, cu, 110, dev.c, 150, rotary)
        want = snapshot(dev)
        restore()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, snapshot(dev))), i
