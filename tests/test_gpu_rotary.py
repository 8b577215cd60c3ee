"""st3_rotary_table and st3_rotate_rows against their definitions."""
import numpy as np
import pytest
import torch

from gpu_util import DEV, TORCH_DTYPE, rand_values, to_np64
from oracle import block_oracle as bo
from paper_2412_20105_amd import binding as st3
from workloads.synth import bf16_bits_to_f32, bf16_round_bits

pytestmark = pytest.mark.gpu


def freqs(pairs, base=10000.0):
    return (base ** (-np.arange(pairs) / pairs)).astype(np.float32)


def table_of(positions, inv_freq, axis, width=None):
    axes, T = positions.shape
    pairs = len(inv_freq)
    out = torch.full((T, width or pairs, 2), 7.0, device=DEV)
    st3.st3_rotary_table(torch.from_numpy(positions).to(DEV), torch.from_numpy(inv_freq).to(DEV), axis, out[:, :pairs])
    torch.cuda.synchronize()
    assert bool((out[:, pairs:] == 7.0).all())
    return out[:, :pairs]


# A cosine or sine of a reduced angle r: r is rounded to float32 (half a step of at most pi/4, 2^-25), the series' last step and the result's rounding are
# half a step of 1 each (2^-25), the terms left out 2^-28.
TABLE = 2.0 ** -25 * 3 + 2.0 ** -28


@pytest.mark.parametrize("T", [1, 2, 7, 64, 1000])
@pytest.mark.parametrize("pairs", [8, 24, 32, 40, 64])
@pytest.mark.parametrize("axes", [1, 2, 3, 4])
def test_table(T, pairs, axes):
    rng = np.random.default_rng(T + pairs + axes)
    positions = rng.integers(-1000, 200000, (axes, T)).astype(np.int32)
    axis = rng.integers(0, axes, pairs).tolist()
    f = freqs(pairs, float(rng.choice([1e4, 1e6])))
    got = to_np64(table_of(positions, f, axis, pairs + 2 * int(rng.integers(0, 3))))
    assert np.abs(got - bo.rotary_table(positions, f, axis)).max() <= TABLE


def test_far_positions_and_quarter_turns():
    ends = np.array([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 2 ** 31 - 2, 2 ** 30, 12345678, -87654321, 355, 710, 103993]], np.int32)
    f = np.concatenate([freqs(56), np.float32([np.pi / 2, np.pi, np.pi / 4, 1e-30, 0.0, 400.0, 3.3, 1.5])])
    got = to_np64(table_of(ends, f, None))
    want = bo.rotary_table(ends, f, [0] * 64)
    assert np.abs(got - want).max() <= TABLE
    assert np.array_equal(got[0], np.stack([np.ones(64), np.zeros(64)], -1))
    # cos^2 + sin^2 of a rotation: each off by TABLE
    assert np.abs((got ** 2).sum(-1) - 1).max() <= 2 * 2 ** 0.5 * TABLE + 2 * TABLE ** 2
    # opposite positions turn opposite ways, bit for bit
    back = to_np64(table_of(np.array([[-5, 5, -2 ** 31 + 1, 2 ** 31 - 1]], np.int32), f, None))
    assert np.array_equal(back[0::2, :, 0], back[1::2, :, 0]) and np.array_equal(back[0::2, :, 1], -back[1::2, :, 1])


def test_frequencies_that_are_not_finite_stay_with_their_pairs():
    f = freqs(16)
    f[3], f[9], f[10] = np.nan, np.inf, -np.inf
    got = to_np64(table_of(np.arange(1, 40, dtype=np.int32)[None], f, None))
    assert np.isnan(got[:, [3, 9, 10]]).all() and np.isfinite(np.delete(got, [3, 9, 10], 1)).all()


def test_one_axis_needs_no_second_dimension_and_axes_may_lie_apart():
    f, pos = torch.from_numpy(freqs(32)).to(DEV), torch.arange(100, 150, dtype=torch.int32, device=DEV)
    a, b, c = (torch.zeros((50, 32, 2), device=DEV) for _ in range(3))
    st3.st3_rotary_table(pos, f, None, a)
    wide = torch.zeros((3, 77), dtype=torch.int32, device=DEV)
    wide[2, 9:59] = pos
    st3.st3_rotary_table(wide[:, 9:59], f, [2] * 32, b)
    st3.st3_rotary_table(wide[2:, 9:59], f, None, c)
    assert torch.equal(a, b) and torch.equal(a, c)


def rounded(x, dtype):
    return bf16_bits_to_f32(bf16_round_bits(x)) if dtype == "bf16" else x


def angles(rng, T, pairs):
    a = rng.uniform(0, 2 * np.pi, (T, pairs))
    return np.stack([np.cos(a), np.sin(a)], -1).astype(np.float32)


def lay(x, layout, dt):
    """x as rows of a wider projection, heads outside rows, or by itself."""
    y = torch.from_numpy(x).to(DEV).to(dt)
    if layout == "fused":
        wide = torch.full((x.shape[0], x.shape[1] + 3, x.shape[2]), 7.0, dtype=dt, device=DEV)
        wide[:, 2:-1] = y
        return wide[:, 2:-1]
    return y.transpose(0, 1).contiguous().transpose(0, 1) if layout == "heads" else y


@pytest.mark.parametrize("T,H", [(1, 1), (1, 40), (3, 7), (33, 12), (700, 5), (5, 1024), (2500, 40)])
@pytest.mark.parametrize("d,pairs", [(64, 32), (64, 8), (128, 64), (128, 24), (128, 40)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("adjacent", [False, True])
def test_rotate_is_the_definition_bit_for_bit(T, H, d, pairs, dtype, adjacent):
    rng = np.random.default_rng(T + H + d + pairs)
    x, cs = rand_values(rng, (T, H, d), dtype, 1.5), angles(rng, T, pairs)
    layout = ["plain", "fused", "heads"][(T + H + pairs) % 3]
    inverse = bool((H + pairs // 8) % 2)
    dev, table = lay(x, layout, TORCH_DTYPE[dtype]), torch.from_numpy(cs).to(DEV)
    turned = st3.rotary(table, st3.ST3_ROTARY_ADJACENT if adjacent else st3.ST3_ROTARY_HALVES)
    want = rounded(bo.rotate(x, cs, adjacent, inverse), dtype)
    out = lay(np.full_like(x, 3.0), "fused", TORCH_DTYPE[dtype])
    st3.st3_rotate_rows(dev, out, turned, inverse)
    assert np.array_equal(to_np64(dev), x.astype(np.float64))
    np.testing.assert_array_equal(to_np64(out), want)
    st3.st3_rotate_rows(dev, dev, turned, inverse)          # in place
    np.testing.assert_array_equal(to_np64(dev), want)
    for t in (dev, out):
        if t._base is not None and t._base.shape[1] == H + 3:
            assert bool((t._base[:, :2] == 7.0).all() and (t._base[:, -1:] == 7.0).all())


@pytest.mark.parametrize("adjacent", [False, True])
def test_the_gradient_is_the_inverse(adjacent):
    """g = R^T y against the formula and against differences of <y, R x>."""
    rng = np.random.default_rng(4)
    T, H, d, pairs = 6, 3, 64, 24
    x, y = (torch.from_numpy(rand_values(rng, (T, H, d), "f32")).to(DEV) for _ in range(2))
    cs = angles(rng, T, pairs)
    turned = st3.rotary(torch.from_numpy(cs).to(DEV), int(adjacent))
    grad = torch.empty_like(x)
    st3.st3_rotate_rows(y, grad, turned, True)
    want = bo.rotate(to_np64(y), cs, adjacent, True)
    np.testing.assert_array_equal(to_np64(grad), want)
    def value(z):
        out = torch.empty_like(z)
        st3.st3_rotate_rows(z, out, turned)
        return float((out.double() * y.double()).sum())
    # linear: a difference at any step is the derivative, up to the rounding of out (2 steps of float32 at |out| <= 2 |pair|, two columns)
    for _ in range(20):
        i = tuple(int(rng.integers(s)) for s in x.shape)
        z = x.clone()
        z[i] += 1.0
        step = float(z[i] - x[i])
        bound = 4 * 2.0 ** -23 * (float(x[i[0], i[1]].abs().max()) + 1) * 2 * float(y[i[0], i[1]].abs().max()) * 2
        assert abs((value(z) - value(x)) / step - float(grad[i])) <= bound


def test_infinities_and_nan_stay_in_their_pairs():
    rng = np.random.default_rng(5)
    x, cs = rand_values(rng, (4, 2, 64), "bf16"), angles(rng, 4, 16)
    x[1, 0, 3], x[2, 1, 20], x[3, 0, 60], x[0, 1, 9] = np.inf, np.nan, -np.inf, -np.inf
    dev = torch.from_numpy(x).to(DEV).bfloat16()
    st3.st3_rotate_rows(dev, dev, st3.rotary(torch.from_numpy(cs).to(DEV)))
    np.testing.assert_array_equal(to_np64(dev), rounded(np.where(np.isnan(y := bo.rotate(x, cs, False)), np.float32("nan"), y), "bf16"))


def test_no_rows_another_stream_and_a_graph():
    rng = np.random.default_rng(6)
    x, cs = rand_values(rng, (50, 8, 128), "bf16"), angles(rng, 50, 64)
    dev, table = torch.from_numpy(x).to(DEV).bfloat16(), torch.zeros((50, 64, 2), device=DEV)
    st3.st3_rotate_rows(dev[:0], dev[:0], st3.rotary(table[:0]))
    st3.st3_rotary_table(torch.zeros((1, 0), dtype=torch.int32, device=DEV), torch.ones(64, device=DEV), None, table[:0])
    pos, f = torch.arange(50, dtype=torch.int32, device=DEV), torch.from_numpy(freqs(64)).to(DEV)
    turned = st3.rotary(table)
    out, want = torch.zeros_like(dev), torch.zeros_like(dev)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        st3.st3_rotary_table(pos, f, None, table)
        st3.st3_rotate_rows(dev, want, turned)
    side.synchronize()
    np.testing.assert_array_equal(to_np64(want), rounded(bo.rotate(x, table.cpu().numpy(), False), "bf16"))
    st3.st3_rotate_rows(dev, out, turned, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        st3.st3_rotary_table(pos, f, None, table)
        st3.st3_rotate_rows(dev, out, turned)
    for i in range(4):
        pos.add_(1000)
        out.zero_(), table.zero_()
        graph.replay()
        torch.cuda.synchronize()
        again = torch.zeros_like(table)
        st3.st3_rotary_table(pos, f, None, again)
        st3.st3_rotate_rows(dev, want, st3.rotary(again))
        torch.cuda.synchronize()
        assert torch.equal(table, again) and torch.equal(out, want), i
