"""st3_block_attend against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from block_util import BLOCK, filled, fp32_slack
from gpu_util import DEV, rand_values, to_np64
from oracle import block_oracle as bo
from paper_2412_20105_amd import binding as st3

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8            # half a step of bf16, relative


def reference(q, rows, cu, old, scale, window, there=None):
    """out, sum of p |v| (what a relative error of the weights is worth), weights of the window's rows; float64 on the device.  rows(b, h): K and V;
    there(b): which rows have a page."""
    H = q.shape[1]
    out, spread, weights, worst = torch.zeros(q.shape, dtype=torch.float64, device=DEV), torch.zeros(q.shape, dtype=torch.float64, device=DEV), [], 0.0
    for b, n in enumerate(old):
        s, m = cu[b], cu[b + 1] - cu[b]
        got = None
        if n >= 0 and m > 0:
            heads = rows(b)
            got = torch.zeros((len(heads), n + m), dtype=torch.float64, device=DEV)
            see = torch.arange(n + m, device=DEV) <= n + torch.arange(m, device=DEV)[:, None]
            if there is not None:
                see &= there(b)
            for kh, (k, v) in enumerate(heads):
                for h in range(kh * (H // len(heads)), (kh + 1) * (H // len(heads))):
                    x = q[s:s + m, h].double()
                    a = (x @ k.t() * scale).masked_fill(~see, -torch.inf)
                    a = torch.softmax(a, -1).nan_to_num(nan=0.0)            # (a row that sees nothing)
                    worst = max(worst, float((x.abs() @ k.abs().t()).max()) * scale)
                    out[s:s + m, h], spread[s:s + m, h] = a @ v, a @ v.abs()
                    got[kh] += a[max(0, m - window):].sum(0) if window else 0
        weights.append(got)
    return out, spread, weights, worst


def run(rng, old, new, H, Hk, d, code, window=5, layout="fused", scale=0.0, sigma=1.5, max_len=None, max_new=None, pad=3, hide=None, compare=True):
    """Through the binding and against the reference; returns what the library left."""
    both = [n + m if n >= 0 else 0 for n, m in zip(old, new)]
    blocks = max(max(both), max_len or 0) // BLOCK + 1
    dev, ref = filled(rng, both, Hk, d, code, blocks)
    dev.set_len(old)
    for b, j in hide or []:
        dev.table[b, j] = -1 if j % 2 else 10 ** 6
    T, cu = sum(new), [0, *np.cumsum(new).tolist()]
    wide = torch.full((T + pad, H + 2, d), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:T, :H] = torch.from_numpy(rand_values(rng, (T, H, d), "bf16", sigma)).to(DEV).bfloat16()
    q, out = wide[:, :H], torch.full((T + pad, H, d), 7.0, dtype=torch.bfloat16, device=DEV)
    if layout == "heads":
        q = q.transpose(0, 1).contiguous().transpose(0, 1)
        out = torch.full((H, T + pad, d), 7.0, dtype=torch.bfloat16, device=DEV).transpose(0, 1)
    elif layout == "wide":
        out = torch.full((T + pad, H + 3, d), 7.0, dtype=torch.bfloat16, device=DEV)[:, 2:2 + H]
    shape = st3.gqa_shape(len(old), H, Hk, d, softmax_scale=scale)
    most, top = (max(new) if max_new is None else max_new), (max(both) if max_len is None else max_len)
    before = torch.rand((len(old), Hk, top + 5), device=DEV) * 3 if window else None
    score = None if before is None else before.clone()
    ws = torch.full((st3.st3_block_attend_workspace_bytes(shape, T + pad, most, top),), 255, dtype=torch.uint8, device=DEV)     # (NaN in every word)
    at = torch.tensor(cu, dtype=torch.int32, device=DEV)
    print(old[:4], new[:4], H, Hk, d, code, window, flush=True)
    st3.st3_block_attend(shape, q, at, most, dev.c, top, out, window, score, ws)
    torch.cuda.synchronize()
    state = (shape, q, at, most, dev, top, ws, before)
    if not compare:
        return out, score, state
    hidden = {}
    for b, j in hide or []:
        hidden.setdefault(b, []).append(j)
    there = lambda b: torch.tensor([i // BLOCK not in hidden.get(b, []) or i >= both[b] // BLOCK * BLOCK for i in range(both[b])], device=DEV)  # noqa: E731
    rows = lambda b: [tuple(torch.from_numpy(x).to(DEV) for x in ref.values(b, h)) for h in range(Hk)]  # noqa: E731
    real = scale if scale else 1.0 / np.sqrt(d)
    want, spread, weights, worst = reference(q, rows, cu, old, real, window, there)
    slack = fp32_slack(worst, d, max(both))
    got = out[:T].double()
    # the output's rounding, and that of every weight
    want, spread = want[:T], spread[:T]
    bound = HALF * (want.abs() + spread) * 1.01 + slack * spread + 1e-30
    assert bool(torch.isfinite(got).all())
    assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() / bound).max())
    assert bool((out[T:] == 7.0).all())
    if window:
        for b, (n, m) in enumerate(zip(old, new)):
            s, first = score[b].double(), before[b].double()
            end = n + m if n >= 0 and m > 0 else 0
            assert torch.equal(s[:, end:], first[:, end:]), b
            if end:
                given = weights[b].clone()
                given[:, :n] += first[:, :n]
                room = 2 * slack * weights[b] + 2.0 ** -23 * given + 1e-30
                assert bool(((s[:, :end] - given).abs() <= room).all()), (b, float(((s[:, :end] - given).abs() / room).max()))
    return out, score, state


SIZES = [([0], [1]), ([5], [1]), ([63], [1]), ([64], [1]), ([62, 0], [1, 3]), ([63, 130], [2, 70]), ([0, 0], [64, 65]), ([10, -1, 0, 300], [3, 4, 0, 33]),
         ([-1], [2]), ([200, 0, 1] * 25, [1, 2, 5] * 25), ([700, 64, 65], [130, 16, 17])]


@pytest.mark.parametrize("old,new", SIZES, ids=lambda x: "-".join(map(str, x[:6])))
@pytest.mark.parametrize("H,Hk,d", [(4, 4, 64), (8, 2, 128), (7, 1, 128), (6, 2, 64)])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_against_the_definition(old, new, H, Hk, d, code):
    run(np.random.default_rng(sum(new) + H + d), old, new, H, Hk, d, code)


@pytest.mark.parametrize("H,Hk", [(32, 1), (40, 40), (20, 5), (28, 4), (33, 3), (70, 1)])
@pytest.mark.parametrize("window", [0, 1, 40])
def test_groups_and_windows(H, Hk, window):
    run(np.random.default_rng(H + window), [70, 3, 141], [1, 30, 41], H, Hk, 128, "int8", window)


@pytest.mark.parametrize("layout", ["fused", "heads", "wide"])
def test_strides(layout):
    run(np.random.default_rng(5), [65, 20], [10, 60], 8, 4, 128, "e4m3", 3, layout)


def test_window_of_all_rows_and_a_scale_of_its_own():
    run(np.random.default_rng(6), [90, 150], [70, 5], 4, 2, 64, "int8", 1000, scale=0.3, sigma=1.0)


def test_bounds_above_the_longest():
    run(np.random.default_rng(7), [50, 10], [4, 9], 4, 2, 64, "int8", 4, max_len=3000, max_new=13)


@pytest.mark.parametrize("old,new,H,Hk,d", [([5000], [3], 8, 2, 128), ([9000], [1], 4, 4, 64), ([4100, 100], [17, 200], 8, 2, 128), ([2500] * 3, [5, 1, 64], 16, 8, 64),
                                            ([30000], [2], 4, 1, 128), ([1000], [900], 8, 2, 128), ([6000], [300], 4, 2, 64), ([40, 8000], [600, 40], 6, 1, 128)])
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_long(old, new, H, Hk, d, code):
    run(np.random.default_rng(sum(old)), old, new, H, Hk, d, code, 33)


@pytest.mark.parametrize("old,new,B", [(739, 4, 1), (739, 5, 1), (300, 8, 3), (1251, 1, 8), (700, 16, 2), (900, 33, 4), (200, 4, 40), (70, 2, 300)])
@pytest.mark.parametrize("d", [64, 128])
def test_few_and_many_rows(old, new, B, d):
    """However a launch is cut."""
    rng = np.random.default_rng(old + new)
    olds = [int(rng.integers(old // 2, old + 1)) for _ in range(B)]
    olds[-1] = old
    run(rng, olds, [new] * B, 32 if B < 100 else 8, 8 if B < 100 else 2, d, "int8" if d == 64 else "e4m3", 2)


@pytest.mark.parametrize("seed", range(24))
def test_random_batches(seed):
    rng = np.random.default_rng(1000 + seed)
    H, Hk = [(8, 2), (4, 4), (12, 4), (7, 1), (16, 8), (5, 5)][seed % 6]
    B = int(rng.integers(1, 9))
    old = [int(x) - 1 for x in np.exp(rng.uniform(0, np.log(900), size=B))]
    new = [int(x) - 1 for x in np.exp(rng.uniform(0, np.log(300), size=B))]
    new[0] += 1
    run(rng, old, new, H, Hk, int(rng.choice([64, 128])), ["int8", "e4m3"][seed // 2 % 2], int(rng.integers(0, 70)), ["fused", "heads", "wide"][seed % 3])


@pytest.mark.parametrize("old,new,hide", [([200, 130], [10, 5], [(0, 0), (0, 2), (1, 1)]), ([128], [3], [(0, 0), (0, 1)]), ([64], [64], [(0, 0), (0, 1)]),
                                          ([5000], [3], [(0, j) for j in range(0, 78, 3)]), ([0], [200], [(0, 0)])])
@pytest.mark.parametrize("window", [0, 7])
def test_blocks_without_pages_are_not_attended(old, new, hide, window):
    """Also where all are missing, and a row that sees none gets 0."""
    out, _, _ = run(np.random.default_rng(8), old, new, 8, 2, 128, "e4m3", window, hide=hide)
    if hide == [(0, 0), (0, 1)] and old == [64]:
        assert not out[:64].any()
    if new == [200]:
        assert not out[:64].any() and out[64:200].any()


def test_lengths_that_lie_are_cut():
    rng = np.random.default_rng(13)
    out, score, (shape, q, at, most, dev, top, ws, before) = run(rng, [100, 30], [20, 30], 4, 2, 64, "int8", 4)
    def go(cu, n, most, top):
        dev.set_len(n)
        o, s = torch.full_like(out, 7.0), before.clone()
        st3.st3_block_attend(shape, q[:50], torch.tensor(cu, dtype=torch.int32, device=DEV), most, dev.c, top, o[:50], 4, s, ws)
        torch.cuda.synchronize()
        return o, s
    o, s = go([-4, 20, 900], [100, 30], most, top)
    assert torch.equal(o, out) and torch.equal(s, score)
    # a row past either bound is no new row: 17 of 20, 27 of 30
    want = go([0, 17, 50], [100, 30], most, 117)
    o, s = go([0, 20, 50], [100, 30], most, 117)
    assert torch.equal(o[:17], want[0][:17]) and bool((o[17:20] == 7.0).all()) and torch.equal(s[0], want[1][0])
    o, s = go([0, 20, 50], [100, 30], 27, top)
    assert torch.equal(o[:47], out[:47]) and bool((o[47:] == 7.0).all())
    # more rows than the bound says: nothing of that sequence is touched
    o, s = go([0, 20, 50], [5000, 30], most, top)
    assert bool((o[:20] == 7.0).all()) and torch.equal(o[20:], out[20:]) and torch.equal(s[0], before[0]) and torch.equal(s[1], score[1])


@pytest.mark.parametrize("old,new", [([40], [90]), ([64, 10], [130, 3]), ([4000], [5])])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(old, new):
    """Infinities and NaN in single elements of the tail's V, NaN codes in pages: 0 times them is no part of any sum."""
    rng = np.random.default_rng(sum(old))
    H, Hk, d = 4, 2, 64
    out, _, (shape, q, at, most, dev, top, ws, _) = run(rng, old, new, H, Hk, d, "e4m3", 0)
    clean, cu, bad = out.double(), at.tolist(), []
    for b, (n, m) in enumerate(zip(old, new)):
        both = n + m
        for j in {both - 1, both - 2, n, both // BLOCK * BLOCK} & set(range(both)):
            h, col = int(rng.integers(Hk)), int(rng.integers(d))
            if j >= both // BLOCK * BLOCK:
                dev.v_tail[b, h, col, j % BLOCK] = float(rng.choice([np.inf, -np.inf, np.nan]))
            else:
                dev.v_codes[int(dev.table[b, j // BLOCK]), h, col, j % BLOCK] = 0x7f
            bad.append((b, j, h, col))
    got = torch.empty_like(out)
    st3.st3_block_attend(shape, q, at, most, dev.c, top, got, 0, None, ws)
    torch.cuda.synchronize()
    odd = torch.zeros(out.shape, dtype=torch.bool, device=DEV)
    for b, j, h, col in bad:
        odd[cu[b] + max(0, j - old[b]):cu[b + 1], h * (H // Hk):(h + 1) * (H // Hk), col] = True
    T = cu[-1]
    assert bool((~torch.isfinite(got[:T].double()))[odd[:T]].all())
    # all others are what they were (a row that was taken again rounds the same sums)
    assert torch.equal(got[:T][~odd[:T]], out[:T][~odd[:T]])


def test_logits_that_are_not_finite():
    """NaN or +infinity among the logits of a head: its output is NaN; -infinity weighs nothing, and where all are, the output is 0."""
    rng = np.random.default_rng(20)
    out, score, (shape, q, at, most, dev, top, ws, before) = run(rng, [10], [30], 4, 2, 64, "int8", 30)
    x = q.clone()
    x[:, :, 0] = x[:, :, 0].abs() + 0.5
    for value in (float("inf"), float("nan")):
        k = dev.k_tail.clone()
        dev.k_tail[0, 0, 25, 0] = value             # row 25: new row 15 is the first that sees it
        o, s = torch.empty_like(out), before.clone()
        st3.st3_block_attend(shape, x, at, most, dev.c, top, o, 30, s, ws)
        torch.cuda.synchronize()
        nan = torch.isnan(o[:30])
        assert bool(nan[15:, :2].all()) and not nan[:15].any() and not nan[:, 2:].any()
        assert bool(torch.isnan(s[0, 0, :40]).all()) and not torch.isnan(s[0, 1]).any() and not torch.isnan(s[0, 0, 40:]).any()
        dev.k_tail.copy_(k)
    dev.k_tail[0, 0, :, 0] = -float("inf")
    o, s = torch.empty_like(out), before.clone()
    st3.st3_block_attend(shape, x, at, most, dev.c, top, o, 30, s, ws)
    torch.cuda.synchronize()
    assert not o[:30, :2].any() and bool(torch.isfinite(o[:30, 2:]).all())
    assert torch.equal(s[0, 0, :10], before[0, 0, :10]) and not s[0, 0, 10:40].any()


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("value", [0.0, 1e-38, 3e33])       # (sums of 160 weights, up to 2^8 each before they are normalised, have to stay below 2^128)
def test_blocks_of_zeros_and_of_extremes(code, value):
    """A block's scale may be 0, or near either end of float32: at the causal edge too, where masked logits are -infinity."""
    rng = np.random.default_rng(21)
    H, Hk, d, old, new = 4, 2, 64, 100, 60
    out, score, (shape, q, at, most, dev, top, ws, before) = run(rng, [old], [new], H, Hk, d, code, 60)
    for j in range(2):
        page = int(dev.table[0, j])
        dev.k_scale[page] = 0.0 if value == 0.0 else 1e-38
        dev.v_scale[page] = value / 448
    q2 = (q.float() * 0.25).bfloat16()
    o, s = torch.empty_like(out), before.clone()
    st3.st3_block_attend(shape, q2, at, most, dev.c, top, o, 60, s, ws)
    torch.cuda.synchronize()
    kind = torch.int8 if code == "int8" else torch.float8_e4m3fn
    def rows(b):
        pairs = []
        for h in range(Hk):
            x = []
            for name in ("k", "v"):
                pages = dev.table[0, :2].long()
                y = getattr(dev, name + "_codes")[pages, h].view(kind).double() * getattr(dev, name + "_scale")[pages, h].double()[:, None, None]
                t = getattr(dev, name + "_tail")[0, h].double()
                x.append(torch.cat([(y if name == "k" else y.transpose(1, 2)).reshape(-1, d), (t if name == "k" else t.t())[:32]]))
            pairs.append(tuple(x))
        return pairs
    want, spread, weights, worst = reference(q2, rows, [0, new], [old], 1 / np.sqrt(d), 60)
    slack, got = fp32_slack(worst, d, 160), o[:new].double()
    # below the smallest normal bf16 (2^-126) a weight's or the output's rounding is a step of 2^-133 instead
    bound = HALF * (want[:new].abs() + spread[:new]) * 1.01 + slack * spread[:new] + 160 * 127 * 2.0 ** -126
    assert bool(torch.isfinite(got).all()) and bool(((got - want[:new]).abs() <= bound).all())
    given = weights[0] + torch.cat([before[0, :, :old].double(), torch.zeros((Hk, new), dtype=torch.float64, device=DEV)], 1)
    assert bool(((s[0, :, :160].double() - given).abs() <= 2 * slack * weights[0] + 2.0 ** -23 * given).all())


def test_other_sequences_do_not_leak():
    rng = np.random.default_rng(22)
    H, Hk, d, old, new = 4, 2, 64, [70, 20, 100], [10, 40, 30]
    out, score, (shape, q, at, most, dev, top, ws, before) = run(rng, old, new, H, Hk, d, "e4m3", 8)
    dev.k_tail[1], dev.v_tail[1] = float("nan"), float("inf")
    x = q.clone()
    x[10:50] = float("nan")
    o, s = torch.full_like(out, 7.0), before.clone()
    st3.st3_block_attend(shape, x, at, most, dev.c, top, o, 8, s, ws)
    torch.cuda.synchronize()
    keep = torch.tensor([*range(10), *range(50, 83)], device=DEV)
    assert torch.equal(o[keep], out[keep]) and torch.equal(s[0], score[0]) and torch.equal(s[2], score[2])


def test_same_result_every_time_and_on_another_stream():
    rng = np.random.default_rng(14)
    out, score, (shape, q, at, most, dev, top, ws, before) = run(rng, [400, 3, 2500], [5, 30, 2], 8, 2, 128, "int8", 16)
    side = torch.cuda.Stream()
    for stream in (None, side, side.cuda_stream):
        o, s = torch.full_like(out, 7.0), before.clone()
        torch.cuda.synchronize()
        st3.st3_block_attend(shape, q, at, most, dev.c, top, o, 16, s, ws, stream)
        torch.cuda.synchronize()
        assert torch.equal(o, out) and torch.equal(s, score)


def test_captured_into_a_graph():
    rng = np.random.default_rng(15)
    out, score, (shape, q, at, most, dev, top, ws, before) = run(rng, [3000, 77], [13, 70], 8, 2, 128, "int8", 8, pad=0)
    graph, o, s = torch.cuda.CUDAGraph(), torch.zeros_like(out), before.clone()
    with torch.cuda.graph(graph):
        st3.st3_block_attend(shape, q, at, most, dev.c, top, o, 8, s, ws)
    for i in range(4):
        if i == 2:
            at.copy_(torch.tensor([0, 40, 83], dtype=torch.int32))      # other lengths within the bounds, and tails no longer than what is there
            dev.set_len([46 * 64 + 3 - 40, 128 + 15 - 43])
        want_o, want_s = torch.full_like(out, 7.0), before.clone()
        st3.st3_block_attend(shape, q, at, most, dev.c, top, want_o, 8, want_s, ws)
        o.fill_(7.0), s.copy_(before)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want_o) and torch.equal(s, want_s), i


def test_one_token_is_a_decode_step():
    """A single new token: what st3_block_decode gives over a cache that holds it."""
    rng = np.random.default_rng(16)
    old, H, Hk, d = [130, 1, 700], 8, 2, 128
    out, score, (shape, q, at, most, dev, top, ws, before) = run(rng, old, [1, 1, 1], H, Hk, d, "int8", 1, pad=0)
    o, s = torch.empty_like(out), before.clone()
    dws = torch.empty(st3.st3_block_workspace_bytes(shape, 701), dtype=torch.uint8, device=DEV)
    dev.set_len([n + 1 for n in old])
    for b, n in enumerate(old):
        s[b, :, n] = 0.0
    st3.st3_block_decode(shape, q, None, None, dev.c, 701, o, s, dws)
    torch.cuda.synchronize()
    # either side's output is rounded, here each weight too: at most half a step of the largest |v| (codes of 127 scales, or the tail)
    v = max(float((dev.v_scale[dev.table[b, :(n + 1) // BLOCK].long()] * 127).max()) if n >= BLOCK else 0.0 for b, n in enumerate(old))
    v = max(v, float(dev.v_tail.nan_to_num(nan=0.0).abs().max()))
    assert float((out.double() - o.double()).abs().max()) <= (3 * HALF + 2 * 2.0 ** -16) * 1.01 * v
    # (both were compared with the definition in other tests; here: sums of 4 weights of at most 1, in float32 either way)
    for b, n in enumerate(old):
        assert float((score[b, :, :n + 1] - s[b, :, :n + 1]).abs().max()) <= 1e-4


def test_against_the_oracle():
    """The oracle's own row-by-row form says the same."""
    rng = np.random.default_rng(17)
    H, Hk, d, n, m = 6, 3, 64, 70, 9
    ref = bo.BlockCache(1, Hk, d, "int8")
    k, v = (rand_values(rng, (n + m, Hk, d), "bf16", 1.5).astype(np.float64) for _ in range(2))
    for h in range(Hk):
        ref.append(0, h, k[:n, h], v[:n, h])
    q = rand_values(rng, (m, H, d), "bf16", 1.5)
    want, weights, spread = bo.extend(ref, 0, q.astype(np.float64), k[n:], v[n:], 1 / np.sqrt(d), 4)
    from block_util import DeviceCache
    dev = DeviceCache(rng, 1, Hk, d, "int8", 2)
    shape = st3.gqa_shape(1, H, Hk, d)
    to = lambda x: torch.from_numpy(np.asarray(x, np.float32)).to(DEV).bfloat16()  # noqa: E731
    st3.st3_block_store(shape, to(k[:n]), to(v[:n]), torch.tensor([0, n], dtype=torch.int32, device=DEV), n, dev.c)
    dev.set_len([n])
    cu = torch.tensor([0, m], dtype=torch.int32, device=DEV)
    st3.st3_block_append(shape, to(k[n:]), to(v[n:]), cu, m, dev.c, n + m)
    out, score = torch.empty((m, H, d), dtype=torch.bfloat16, device=DEV), torch.zeros((1, Hk, n + m), device=DEV)
    ws = torch.empty(st3.st3_block_attend_workspace_bytes(shape, m, m, n + m), dtype=torch.uint8, device=DEV)
    st3.st3_block_attend(shape, to(q), cu, m, dev.c, n + m, out, 4, score, ws)
    dev.check(ref)
    slack = fp32_slack(float(np.abs(q).max() * np.abs(k).max()) * d / np.sqrt(d), d, n + m)
    assert np.all(np.abs(to_np64(out) - want) <= HALF * (np.abs(want) + spread) * 1.01 + slack * spread)
    assert np.all(np.abs(to_np64(score)[0] - weights) <= 2 * slack * weights + 1e-30)
