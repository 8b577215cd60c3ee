"""Positions, rotation, further rows of a cache and attention over it without a GPU: what is refused, workspaces, the oracle, the binding."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from paper_2412_20105_amd import binding as st3
from paper_2412_20105_amd.block_pipeline import BlockGeneration

FAKE, FAR = 0x10000, 0x10000 + (1 << 30)
OK, INVALID, UNSUPPORTED, SMALL = 0, 1, 2, 3


def rows(data=FAKE, st=1024, sh=128):
    return C.byref(st3.Rows(data, st, sh))


def shape(batch=2, heads=8, kv_heads=2, dim=128, dtype=st3.ST3_BF16, scale=0.0):
    return C.byref(st3.gqa_shape(batch, heads, kv_heads, dim, dtype, scale))


def cache(**more):
    f = dict(k_codes=FAKE, v_codes=FAKE, k_scale=FAKE, v_scale=FAKE, k_tail=FAKE, v_tail=FAKE, table=FAKE, table_stride=8, len=FAKE,
             table_blocks=8, n_pages=4, code=st3.ST3_BLOCK_INT8)
    f.update(more)
    return C.byref(st3.BlockCache(*f.values()))


def rotary(table=FAKE, st=128, pairs=64, layout=0):
    return C.byref(st3.Rotary(table, st, pairs, layout))


def table(axes=1, pairs=64, axis=None, freq=FAKE, pos=FAKE, ps=10, total=10, out=FAKE, st=128):
    return st3.lib().st3_rotary_table(axes, pairs, axis, freq, pos, ps, total, out, st, None)


@pytest.mark.parametrize("bad,want", [
    (dict(axes=0), INVALID), (dict(axes=5), UNSUPPORTED), (dict(pairs=0), INVALID), (dict(pairs=12), UNSUPPORTED), (dict(pairs=72, st=144), UNSUPPORTED),
    (dict(axis=bytes([0] * 63 + [1])), INVALID), (dict(axes=2, axis=bytes([2] + [0] * 63)), INVALID), (dict(freq=None), INVALID), (dict(freq=FAKE + 4), INVALID),
    (dict(pos=None), INVALID), (dict(axes=2, ps=9), INVALID), (dict(total=-1), INVALID), (dict(out=None), INVALID), (dict(out=FAKE + 8), INVALID),
    (dict(axes=2, ps=-10), INVALID), (dict(st=127), INVALID), (dict(st=126), INVALID), (dict(st=130), INVALID), (dict(total=0, pos=None, out=None), OK)], ids=str)
def test_table_refuses(bad, want):
    assert table(**bad) == want


def rotate(x=None, out=None, heads=8, total=10, dim=128, dtype=st3.ST3_BF16, r=None):
    return st3.lib().st3_rotate_rows(x or rows(), out or rows(FAR), heads, total, dim, dtype, r or rotary(FAKE + (1 << 29)), 0, None)


@pytest.mark.parametrize("bad,want", [
    (dict(heads=0), INVALID), (dict(heads=1025), UNSUPPORTED), (dict(total=-1), INVALID), (dict(dim=96), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED),
    (dict(x=rows(None)), INVALID), (dict(x=rows(FAKE + 2)), INVALID), (dict(out=rows(FAR, 1024, 64)), INVALID), (dict(out=rows(FAR, 512, 128)), INVALID),
    (dict(r=rotary(None)), INVALID), (dict(r=rotary(pairs=0)), INVALID), (dict(r=rotary(pairs=20)), UNSUPPORTED), (dict(r=rotary(layout=2)), INVALID),
    (dict(r=rotary(layout=-1)), INVALID), (dict(r=rotary(st=120)), INVALID), (dict(r=rotary(st=130)), INVALID), (dict(r=rotary(FAKE + 4)), INVALID),
    (dict(dim=64, r=rotary(pairs=40)), INVALID), (dict(total=0, x=rows(None), out=rows(None)), OK)], ids=str)
def test_rotate_refuses(bad, want):
    assert rotate(**bad) == want


def test_rotate_refuses_memory_that_is_shared():
    assert rotate(out=rows(FAKE + 1024)) == INVALID                       # half way into the rows
    assert rotate(x=rows(FAKE, 2048), out=rows(FAKE, 1024)) == INVALID    # from the same place with other strides
    assert rotate(out=rows(FAR), r=rotary(FAR)) == INVALID                # the table
    assert rotate(out=rows(FAR), r=rotary(FAR - 10 * 512 + 16)) == INVALID
    assert rotate(x=rows(FAR), out=rows(FAR), r=rotary(FAR + 10 * 2048 - 16)) == INVALID


def append(sh=None, k=None, v=None, cu=FAKE, total=100, most=50, c=None, top=100, r=None):
    return st3.lib().st3_block_append(sh or shape(), k or rows(), v or rows(), cu, total, most, c or cache(), top, r, None)


def attend(sh=None, q=None, cu=FAKE, total=100, most=50, c=None, top=100, out=None, window=1, score=FAKE, sb=200, s_h=100, ws=FAKE, wb=1 << 30):
    return st3.lib().st3_block_attend(sh or shape(), q or rows(), cu, total, most, c or cache(), top, out or rows(FAR), window, score, sb, s_h, ws, wb, None)


SHAPES = [(dict(batch=0), INVALID), (dict(heads=0), INVALID), (dict(kv_heads=0), INVALID), (dict(heads=9), INVALID), (dict(dim=80), UNSUPPORTED),
          (dict(dtype=2), UNSUPPORTED), (dict(heads=2048), UNSUPPORTED), (dict(batch=70000), UNSUPPORTED), (dict(scale=-1.0), INVALID),
          (dict(scale=float("nan")), INVALID), (dict(dtype=st3.ST3_F32), UNSUPPORTED)]


@pytest.mark.parametrize("bad,want", SHAPES)
def test_shapes_that_are_refused(bad, want):
    sh = shape(**bad)
    assert append(sh) == want and attend(sh) == want
    if bad != dict(dtype=st3.ST3_F32):
        assert st3.lib().st3_block_attend_workspace_bytes(sh, 100, 50, 100) == 0


CACHES = [dict([(n, None)]) for n in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail", "table", "len")] + \
         [dict(table_stride=7), dict(table_blocks=0), dict(n_pages=0), dict(code=2), dict(k_codes=FAKE + 8), dict(v_tail=FAKE + 2)]


@pytest.mark.parametrize("bad", CACHES, ids=str)
def test_caches_that_are_refused(bad):
    assert append(c=cache(**bad)) == INVALID and attend(c=cache(**bad)) == INVALID


@pytest.mark.parametrize("bad,want", [
    (dict(cu=None), INVALID), (dict(total=-1), INVALID), (dict(most=-1), INVALID), (dict(most=101), INVALID), (dict(top=-1), INVALID),
    (dict(top=9 * 64), INVALID), (dict(top=2 ** 30), UNSUPPORTED), (dict(k=rows(None)), INVALID), (dict(v=rows(FAKE + 2)), INVALID), (dict(k=rows(FAKE, 64)), INVALID),
    (dict(r=rotary(None)), INVALID), (dict(r=rotary(pairs=72)), UNSUPPORTED), (dict(sh=shape(dim=64), r=rotary()), INVALID), (dict(r=rotary(layout=5)), INVALID),
    (dict(total=0, most=0, k=rows(None), v=rows(None)), OK), (dict(most=0), OK),
    (dict(total=2 ** 31 - 1, most=2 ** 31 - 1, top=100), UNSUPPORTED)], ids=str)
def test_append_refuses(bad, want):
    assert append(**bad) == want


@pytest.mark.parametrize("bad,want", [
    (dict(cu=None), INVALID), (dict(total=-1), INVALID), (dict(most=-1), INVALID), (dict(most=101), INVALID), (dict(top=-1), INVALID),
    (dict(top=9 * 64, s_h=600, sb=2000), INVALID), (dict(top=2 ** 30, s_h=2 ** 30, sb=2 ** 31), UNSUPPORTED), (dict(window=-1), INVALID), (dict(window=0), INVALID),
    (dict(s_h=99), INVALID), (dict(sb=99), INVALID), (dict(ws=None), INVALID), (dict(ws=FAKE + 4), INVALID), (dict(q=rows(None)), INVALID),
    (dict(out=rows(FAR + 2)), INVALID), (dict(out=rows(FAR, 256)), INVALID), (dict(out=rows(FAKE)), INVALID), (dict(out=rows(FAKE + 2048)), INVALID),
    (dict(wb=0), SMALL), (dict(score=None, window=0, wb=0), SMALL), (dict(total=0, most=0, q=rows(None), out=rows(None)), OK), (dict(most=0), OK)], ids=str)
def test_attend_refuses(bad, want):
    assert attend(**bad) == want


def test_workspace_for_the_most_is_enough_for_less():
    for s in (st3.gqa_shape(1, 32, 8, 128), st3.gqa_shape(16, 40, 40, 128), st3.gqa_shape(4, 16, 1, 64)):
        totals, lens = [1, 2, 5, 17, 64, 65, 300, 1000, 5000, 20000], [1, 63, 64, 300, 3000, 40000, 130000]
        need = {(t, n): st3.st3_block_attend_workspace_bytes(s, t, t, n) for t in totals for n in lens}
        for (t, n), size in need.items():
            assert all(need[u, k] <= size for u in totals for k in lens if u <= t and k <= n)
            assert size >= t * s.heads * 8
        assert attend(C.byref(s), total=300, most=300, top=3000, c=cache(table_blocks=50, table_stride=50), s_h=3000, sb=2 ** 20, wb=need[300, 3000] - 1,
                      q=rows(st=8192), out=rows(FAR, 8192)) == SMALL


# ---- the oracle -------------------------------------------------------------------------------------------------------------------
def test_oracle_table():
    pos = np.array([[0, 1, 100000], [5, -3, 2 ** 31 - 1]])
    f = np.float32([1.0, 0.01])
    got = bo.rotary_table(pos, f, [0, 1])
    for t in range(3):
        for c in range(2):
            angle = float(pos[c, t]) * float(f[c])
            np.testing.assert_allclose(got[t, c], [np.cos(angle), np.sin(angle)], atol=1e-8)


@pytest.mark.parametrize("adjacent", [False, True])
def test_oracle_rotation_is_that_of_complex_numbers(adjacent):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 3, 64)).astype(np.float32)
    a = rng.uniform(0, 6.3, (5, 24))
    cs = np.stack([np.cos(a), np.sin(a)], -1).astype(np.float32)
    y = bo.rotate(x, cs, adjacent)
    z = x[..., 0:48:2] + 1j * x[..., 1:48:2] if adjacent else x[..., :24] + 1j * x[..., 24:48]
    z = z * (cs[..., 0] + 1j * cs[..., 1])[:, None]
    got = y[..., 0:48:2] + 1j * y[..., 1:48:2] if adjacent else y[..., :24] + 1j * y[..., 24:48]
    np.testing.assert_allclose(got, z, atol=1e-6)
    assert np.array_equal(y[..., 48:], x[..., 48:])
    np.testing.assert_allclose(bo.rotate(y, cs, adjacent, True), x, atol=2e-6)


def test_oracle_extend_is_decode_row_by_row_where_no_block_fills():
    rng = np.random.default_rng(2)
    one, many = (bo.BlockCache(1, 2, 8, "int8") for _ in range(2))
    k, v = rng.standard_normal((2, 90, 2, 8))
    for c in (one, many):
        for h in range(2):
            c.append(0, h, k[:70, h], v[:70, h])
    q = rng.standard_normal((20, 4, 8))
    out, weights, spread = bo.extend(one, 0, q, k[70:], v[70:], 0.3, 5)
    total = np.zeros((2, 90))
    for t in range(20):
        o, w = bo.decode(many, 0, q[t], k[70 + t], v[70 + t], 0.3)
        np.testing.assert_allclose(out[t], o, atol=1e-12)
        if t >= 15:
            total[:, :71 + t] += w
    np.testing.assert_allclose(weights, total, atol=1e-12)
    assert np.all(spread >= np.abs(out) - 1e-12)


# ---- the binding and the generation ------------------------------------------------------------------------------------------------
def test_binding_refuses_what_the_library_cannot_see():
    with pytest.raises(TypeError):
        st3.rotary(torch.zeros(3, 8, 2))                                         # not on the device
    with pytest.raises(ValueError):
        st3.rotary(torch.zeros(3, 8))
    with pytest.raises(ValueError):
        st3.rotary(torch.zeros(3, 2, 8).transpose(1, 2))                         # cosines and sines apart
    with pytest.raises(ValueError):
        st3._check_rotary(type("R", (), {"_rows": 4})(), 5)
    with pytest.raises(ValueError):
        st3.st3_rotate_rows(torch.zeros(3, 2, 64), torch.zeros(3, 2, 64), None)


def a_generation(lens):
    gen = BlockGeneration.__new__(BlockGeneration)
    gen.B, gen.lens, gen.capacity, gen.budget, gen.new, gen.device, gen.evictions = len(lens), lens, 256, 128, None, "cpu", 0
    gen.shape, gen._turn_ws = st3.gqa_shape(len(lens), 8, 2, 128), torch.empty(0, dtype=torch.uint8)
    gen.len, gen.live = torch.tensor(lens, dtype=torch.int32), torch.tensor([int(n >= 0) for n in lens], dtype=torch.int32)
    gen.evict = lambda: (setattr(gen, "evictions", gen.evictions + 1), setattr(gen, "lens", [min(n, 128) for n in gen.lens]), gen.len.clamp_(max=128))
    return gen


def test_turns_of_a_generation():
    gen = a_generation([200, -1, 30])
    for bad in ([1, 0], [1, 1, 1], [-1, 0, 0], [129, 0, 0], [0, 0, 227]):
        with pytest.raises(ValueError):
            gen.begin_turn(bad)
    for call in (gen.finish_turn, lambda: gen.extend_layer(0, None, None, None)):
        with pytest.raises(ValueError):
            call()
    gen.begin_turn([56, 0, 9])
    assert gen.evictions == 0 and gen.total == 65 and gen.cu.tolist() == [0, 56, 56, 65] and gen._turn_ws.numel() > 0
    for call in (lambda: gen.begin_turn([0, 0, 0]), gen.begin_step, lambda: gen.extend_layer(0, *(torch.zeros(64, 1, 1),) * 3)):
        with pytest.raises(ValueError):
            call()
    gen.finish_turn()
    assert gen.lens == [256, -1, 39] and gen.len.tolist() == gen.lens
    gen.begin_turn([1, 0, 100])         # one has no room left
    assert gen.evictions == 1 and gen.lens == [128, -1, 39]
    gen.lens[2], gen.live[2], gen.len[2] = -1, 0, -1            # retired before the turn's end
    gen.finish_turn()
    assert gen.lens == [129, -1, -1] and gen.len.tolist() == gen.lens


def test_nothing_else_while_a_turn_is_open():
    gen = a_generation([20, -1, 30])
    del gen.evict
    gen.begin_turn([5, 0, 9])
    rows = torch.zeros(14, 1, 1)
    for call in (gen.begin_step, gen.finish_step, gen.evict, lambda: gen.begin_turn([0, 0, 0]), lambda: gen.prefill_layer(0, rows, rows, rows),
                 lambda: gen.decode_layer(0, rows, rows, rows)):
        with pytest.raises(ValueError):
            call()
    assert gen.lens == [20, -1, 30] and gen.len.tolist() == gen.lens
    gen.finish_turn()
    assert gen.lens == [25, -1, 39]


def test_positions_that_overlap_are_refused():
    for positions in (torch.zeros(12, dtype=torch.int32).as_strided((3, 8), (2, 1)), torch.zeros(30, dtype=torch.int32).as_strided((2, 8), (1, 2))):
        with pytest.raises(ValueError, match="axes"):
            st3.st3_rotary_table(positions, torch.zeros(8), None, torch.zeros(8, 8, 2))


@pytest.mark.parametrize("seed", range(8))
def test_any_sizes_are_cut_into_a_launch(seed):
    """From one token to the largest sizes, batches with far more rows than their sequences have among them: the only thing missing is workspace.  (Parts
    of more than 2^26 rows and heads, most of them no sequence's, are no launch.)"""
    rng = np.random.default_rng(seed)
    pick = lambda most: int(np.exp(rng.uniform(0, np.log(most))))  # noqa: E731
    for _ in range(500):
        Hk, batch = pick(64), pick(300)
        H = Hk * pick(16)
        new = pick(4096)
        total = max(new, pick(200000) if rng.integers(2) else int(batch * new * rng.uniform(0.2, 1)))
        both = new + pick(2 ** 20) - 1
        blocks = both // 64 + 1
        d = int(rng.choice([64, 128]))
        s = C.byref(st3.gqa_shape(batch, H, Hk, d))
        got = st3.lib().st3_block_attend(s, rows(st=H * d, sh=d), FAKE, total, new, cache(table_blocks=blocks, table_stride=blocks), both, rows(1 << 50, H * d, d), 3,
                                         FAKE, Hk * both, both, FAKE, 0, None)
        assert got == SMALL or got == UNSUPPORTED and total * H > 2 ** 26 and batch * new < total, (batch, H, Hk, d, total, new, both, got)
        assert st3.st3_block_attend_workspace_bytes(st3.gqa_shape(batch, H, Hk, d), total, new, both) > 0


def test_the_rotation_has_the_header_s_layout(tmp_path):
    import os
    import shutil
    import subprocess

    from conftest import ROOT
    if shutil.which("gcc") is None:
        pytest.skip("no C compiler")
    names = [n for n, _ in st3.Rotary._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "st3.h"\nint main(void) {\n  printf("%zu", sizeof(st3_rotary));\n' +
                   "".join(f'  printf(" %zu", offsetof(st3_rotary, {n}));\n' for n in names) +
                   '  printf(" %d %d", ST3_ROTARY_HALVES, ST3_ROTARY_ADJACENT);\n  return 0;\n}\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [C.sizeof(st3.Rotary), *(getattr(st3.Rotary, n).offset for n in names), st3.ST3_ROTARY_HALVES, st3.ST3_ROTARY_ADJACENT]
