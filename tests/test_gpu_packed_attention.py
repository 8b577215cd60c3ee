"""st3_packed_attention against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from block_util import fp32_slack
from gpu_util import DEV, TORCH_DTYPE, rand_values, to_np64
from oracle import block_oracle as bo
from paper_2412_20105_amd import binding as st3

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8            # half a step of bf16, relative


def reference(q, k, v, lens, scale, window):
    """out, sum of p |v| (what a relative error of the weights is worth), scores; float64 on the device, head by head."""
    H, Hk = q.shape[1], k.shape[1]
    q, k, v = (x.double() for x in (q, k, v))
    out, spread, scores, start, worst = torch.zeros_like(q), torch.zeros_like(q), [], 0, 0.0
    for n in lens:
        score = torch.zeros((Hk, n), dtype=torch.float64, device=q.device)
        rows = slice(start, start + n)
        for h in range(H if n else 0):
            kh = h // (H // Hk)
            a = q[rows, h] @ k[rows, kh].t() * scale
            worst = max(worst, float((q[rows, h].abs() @ k[rows, kh].abs().t()).max()) * scale)
            a = torch.softmax(a.masked_fill(torch.ones_like(a, dtype=torch.bool).triu(1), -torch.inf), -1)
            out[rows, h], spread[rows, h] = a @ v[rows, kh], a @ v[rows, kh].abs()
            if window:
                score[kh] += a[max(0, n - window):].sum(0)
        scores.append(score)
        start += n
    return out, spread, scores, worst


def run(rng, lens, H, Hk, d, dtype, window, layout="fused", scale=0.0, sigma=1.5, pad=3, max_len=None, stream=None):
    """Through the binding and against the reference; returns what the library left."""
    T = sum(lens)
    dt = TORCH_DTYPE[dtype]
    rows = torch.full((T + pad, H + 2 * Hk, d), float("nan"), dtype=dt, device=DEV)
    rows[:T] = torch.from_numpy(rand_values(rng, (T, H + 2 * Hk, d), dtype, sigma)).to(DEV).to(dt)
    q, k, v = rows[:, :H], rows[:, H:H + Hk], rows[:, H + Hk:]
    out = torch.full((T + pad, H, d), 7.0, dtype=dt, device=DEV)
    if layout == "heads":       # heads outside rows
        q, k, v = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v))
        out = torch.full((H, T + pad, d), 7.0, dtype=dt, device=DEV).transpose(0, 1)
    elif layout == "wide":      # out in the columns of a wider buffer
        out = torch.full((T + pad, H + 2, d), 7.0, dtype=dt, device=DEV)[:, 1:1 + H]
    shape = st3.gqa_shape(len(lens), H, Hk, d, st3.ST3_F32 if dtype == "f32" else st3.ST3_BF16, scale)
    cu = torch.tensor([0, *np.cumsum(lens)], dtype=torch.int32, device=DEV)
    top = max(lens) if max_len is None else max_len
    score = torch.full((len(lens), Hk, top + 5), -3.0, device=DEV) if window else None
    ws = torch.empty(max(256, st3.st3_packed_workspace_bytes(shape, T + pad)), dtype=torch.uint8, device=DEV)
    st3.st3_packed_attention(shape, q, k, v, cu, top, out, window, score, ws, stream)
    torch.cuda.synchronize()
    real = scale if scale else 1.0 / np.sqrt(d)
    want, spread, scores, worst = reference(q[:T], k[:T], v[:T], lens, real, window)
    slack = fp32_slack(worst, d, top)
    got = out[:T].double()
    if dtype == "bf16":         # the output's rounding, and that of every weight
        bound = HALF * (want.abs() + spread) * 1.01 + slack * spread
    else:
        bound = 2 * slack * spread
    assert bool(torch.isfinite(got).all())
    assert bool(((got - want).abs() <= bound + 1e-30).all()), float(((got - want).abs() / (bound + 1e-30)).max())
    assert bool((out[T:] == 7.0).all())
    if window:
        for b, n in enumerate(lens):
            s = score[b, :, :n].double()
            assert bool(((s - scores[b]).abs() <= 2 * slack * scores[b] + 1e-30).all()), (b, n)
            assert bool((score[b, :, n:] == -3.0).all())
    return out, score, (shape, q, k, v, cu, top, ws)


LENS = [[1], [2, 0, 5], [33, 64, 1, 130], [127, 128, 129], [300, 31, 32, 16, 15, 17], [0, 0, 3], [7] * 70, [200, 0, 1] * 25]


@pytest.mark.parametrize("lens", LENS, ids=lambda x: "-".join(map(str, x[:6])))
@pytest.mark.parametrize("H,Hk,d", [(4, 4, 64), (8, 2, 128), (7, 1, 128), (6, 2, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_against_the_definition(lens, H, Hk, d, dtype):
    run(np.random.default_rng(sum(lens) + H + d), lens, H, Hk, d, dtype, window=5)


@pytest.mark.parametrize("H,Hk", [(32, 1), (40, 40), (20, 5), (28, 4), (33, 3)])
@pytest.mark.parametrize("window", [0, 1, 40])
def test_groups_and_windows(H, Hk, window):
    run(np.random.default_rng(H + window), [70, 3, 41], H, Hk, 128, "bf16", window)


@pytest.mark.parametrize("layout", ["fused", "heads", "wide"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides(layout, dtype):
    run(np.random.default_rng(5), [65, 20], 8, 4, 128, dtype, 3, layout)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_window_of_all_rows_and_a_scale_of_its_own(dtype):
    run(np.random.default_rng(6), [90, 150], 4, 2, 64, dtype, 1000, scale=0.3, sigma=1.0)


def test_bound_above_the_longest():
    run(np.random.default_rng(7), [50, 10], 4, 2, 64, "bf16", 4, max_len=60)


@pytest.mark.parametrize("lens,H,Hk", [([2500, 777], 8, 2), ([4100], 4, 4), ([1025] * 9, 16, 8), ([5000, 1, 64, 900], 6, 1)])
def test_long(lens, H, Hk):
    run(np.random.default_rng(sum(lens)), lens, H, Hk, 128, "bf16", 33)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens", [[130, 17], [300], [257, 255], [1100], [1025, 3], [400] * 3, [600] * 4], ids=lambda x: "-".join(map(str, x)))
def test_few_and_many_row_tiles(lens, d):
    """Short and long walks over the keys with few row tiles, more, and many: however a launch is cut."""
    run(np.random.default_rng(sum(lens) + d), lens, 32, 8, d, "bf16", 21)


@pytest.mark.parametrize("seed", range(24))
def test_random_batches(seed):
    rng = np.random.default_rng(1000 + seed)
    H, Hk = [(8, 2), (4, 4), (12, 4), (7, 1), (16, 8), (5, 5)][seed % 6]
    lens = [int(x) for x in np.exp(rng.uniform(0, np.log(700), size=rng.integers(1, 9)))]
    run(rng, lens, H, Hk, int(rng.choice([64, 128])), "f32" if seed % 4 == 3 else "bf16", int(rng.integers(0, 70)),
        ["fused", "heads", "wide"][seed % 3])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_other_sequences_do_not_leak(dtype):
    """Infinities and NaN in one sequence, and in the rows behind the last, reach no other."""
    rng = np.random.default_rng(11)
    lens, H, Hk, d = [37, 20, 45], 4, 2, 64
    dt = TORCH_DTYPE[dtype]
    x = torch.from_numpy(rand_values(rng, (sum(lens), H + 2 * Hk, d), dtype)).to(DEV).to(dt)
    shape = st3.gqa_shape(3, H, Hk, d, st3.ST3_F32 if dtype == "f32" else st3.ST3_BF16)
    cu = torch.tensor([0, 37, 57, 102], dtype=torch.int32, device=DEV)
    ws = torch.empty(st3.st3_packed_workspace_bytes(shape, 102), dtype=torch.uint8, device=DEV)
    got = []
    for bad in (0.0, float("nan"), float("inf"), -float("inf"), torch.finfo(dt).min):
        y = x.clone()
        if bad != 0.0:
            y[37:57] = bad
        out, score = torch.zeros((102, H, d), dtype=dt, device=DEV), torch.zeros((3, Hk, 45), device=DEV)
        st3.st3_packed_attention(shape, y[:, :H], y[:, H:H + Hk], y[:, H + Hk:], cu, 45, out, 4, score, ws)
        got.append((torch.cat([out[:37], out[57:]]), score[0], score[2]))
    for g in got[1:]:
        for a, b in zip(got[0], g):
            assert torch.equal(a, b)


def test_later_keys_do_not_leak():
    """A row sees no key behind it, whatever lies there."""
    rng = np.random.default_rng(12)
    n, H, Hk, d = 130, 4, 2, 128
    x = torch.from_numpy(rand_values(rng, (n, H + 2 * Hk, d), "bf16")).to(DEV).bfloat16()
    shape = st3.gqa_shape(1, H, Hk, d)
    cu = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    for at in (1, 31, 32, 33, 64, 100, 129):
        y = x.clone()
        y[at:, H + Hk:] = float("nan")      # values of the rows from `at` on
        y[at:, H:H + Hk] = float("inf")
        a, b = (torch.zeros((n, H, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        st3.st3_packed_attention(shape, x[:, :H], x[:, H:H + Hk], x[:, H + Hk:], cu, n, a)
        st3.st3_packed_attention(shape, y[:, :H], y[:, H:H + Hk], y[:, H + Hk:], cu, n, b)
        clean = at // 64 * 64 if at % 64 else at
        assert torch.equal(a[:min(clean, at)], b[:min(clean, at)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens, H, Hk, d", [([40], 4, 1, 128), ([5, 300, 33], 8, 8, 64), ([100, 31, 700], 12, 4, 128), ([300] * 9, 32, 32, 64)])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(lens, H, Hk, d, dtype):
    """Infinities and NaN in single elements of V, in a row's own tile of keys and in earlier ones: 0 times them is no part of any sum."""
    rng = np.random.default_rng(sum(lens))
    T, dt = sum(lens), TORCH_DTYPE[dtype]
    q, k, v = (torch.from_numpy(rand_values(rng, (T, h, d), dtype, 1.0)).to(DEV).to(dt) for h in (H, Hk, Hk))
    bad = []
    for j in rng.choice(T, 5, replace=False):
        at = (int(j), int(rng.integers(Hk)), int(rng.integers(d)))
        bad.append(at)
        v[at] = float(rng.choice([np.inf, -np.inf, np.nan]))
    shape = st3.gqa_shape(len(lens), H, Hk, d, st3.ST3_F32 if dtype == "f32" else st3.ST3_BF16)
    cu = torch.tensor([0, *np.cumsum(lens)], dtype=torch.int32, device=DEV)
    out = torch.empty((T, H, d), dtype=dt, device=DEV)
    st3.st3_packed_attention(shape, q, k, v, cu, max(lens), out)
    clean = torch.where(torch.isfinite(v), v, torch.zeros_like(v))
    want, spread, _, worst = reference(q, k, clean, lens, 1.0 / np.sqrt(d), 0)
    for j, kh, col in bad:
        end = next(int(e) for e in cu[1:].tolist() if j < e)
        for h in range(kh * (H // Hk), (kh + 1) * (H // Hk)):
            want[j:end, h, col] += float(v[j, kh, col])     # (every weight of these logits is above 0)
    got, odd = out.double(), ~torch.isfinite(want)
    assert bool(odd.any()) and torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(got[odd].nan_to_num(nan=0.0), want[odd].nan_to_num(nan=0.0))
    slack = fp32_slack(worst, d, max(lens))
    room = spread * (slack + (2 * HALF if dtype == "bf16" else 0)) + want.abs() * (HALF if dtype == "bf16" else 0) + 1e-30
    assert bool(((got - want).abs() <= room)[~odd].all())


def test_lengths_that_lie_are_cut():
    """cu_len past the rows that exist, or a sequence longer than the bound: what exists is attended, nothing else is touched."""
    rng = np.random.default_rng(13)
    H, Hk, d, T = 4, 2, 64, 50
    x = torch.from_numpy(rand_values(rng, (T, H + 2 * Hk, d), "bf16")).to(DEV).bfloat16()
    shape = st3.gqa_shape(2, H, Hk, d)
    good, bad = (torch.full((T, H, d), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    st3.st3_packed_attention(shape, x[:, :H], x[:, H:H + Hk], x[:, H + Hk:], torch.tensor([0, 20, 50], dtype=torch.int32, device=DEV), 30, good)
    st3.st3_packed_attention(shape, x[:, :H], x[:, H:H + Hk], x[:, H + Hk:], torch.tensor([-4, 20, 900], dtype=torch.int32, device=DEV), 25, bad)
    assert torch.equal(good[:45], bad[:45]) and bool((bad[45:] == 7.0).all())


def test_same_result_every_time_and_on_another_stream():
    rng = np.random.default_rng(14)
    out, score, (shape, q, k, v, cu, top, ws) = run(rng, [400, 3, 250], 8, 2, 128, "bf16", 16)
    side = torch.cuda.Stream()
    for s in (None, side, side.cuda_stream):
        o, c = torch.full_like(out, 7.0), torch.full_like(score, -3.0)
        torch.cuda.synchronize()
        st3.st3_packed_attention(shape, q, k, v, cu, top, o, 16, c, ws, s)
        torch.cuda.synchronize()
        assert torch.equal(o, out) and torch.equal(c, score)


def test_captured_into_a_graph():
    rng = np.random.default_rng(15)
    out, score, (shape, q, k, v, cu, top, ws) = run(rng, [130, 77], 8, 2, 128, "bf16", 8)
    graph, o, c = torch.cuda.CUDAGraph(), torch.zeros_like(out), torch.zeros_like(score)
    with torch.cuda.graph(graph):
        st3.st3_packed_attention(shape, q, k, v, cu, top, o, 8, c, ws)
    for i in range(4):
        o.fill_(7.0), c.fill_(-3.0)
        if i == 2:
            cu.copy_(torch.tensor([0, 77, 207], dtype=torch.int32))     # other lengths within the bounds
        want_o, want_c = torch.full_like(out, 7.0), torch.full_like(score, -3.0)
        st3.st3_packed_attention(shape, q, k, v, cu, top, want_o, 8, want_c, ws)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want_o) and torch.equal(c, want_c), i


def test_against_the_oracle():
    """The oracle's own row-by-row form says the same."""
    rng = np.random.default_rng(16)
    lens, H, Hk, d = [20, 1, 37], 6, 3, 64
    out, score, (shape, q, k, v, cu, top, ws) = run(rng, lens, H, Hk, d, "f32", 4)
    want, scores = bo.packed_attention(*(to_np64(x[:58]) for x in (q, k, v)), lens, 1 / np.sqrt(d), 4)
    np.testing.assert_allclose(to_np64(out[:58]), want, atol=2e-5)
    for b, n in enumerate(lens):
        np.testing.assert_allclose(to_np64(score[b, :, :n]), scores[b], atol=2e-5)
