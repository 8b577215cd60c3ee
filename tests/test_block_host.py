"""The grouped-head calls without a GPU: what they refuse, and the oracle they are tested against."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import block_oracle as bo
from paper_2412_20105_amd import binding as st3

FAKE = 0x10000
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


def packed(sh=None, q=None, k=None, v=None, cu=FAKE, total=100, max_len=50, out=None, window=1, score=FAKE, sb=100, s_h=50, ws=FAKE, wb=1 << 20):
    far = FAKE + (1 << 30)
    return st3.lib().st3_packed_attention(sh or shape(), q or rows(), k or rows(FAKE, 256, 128), v or rows(FAKE, 256, 128), cu, total, max_len,
                                          out or rows(far), window, score, sb, s_h, ws, wb, None)


SHAPES = [(dict(batch=0), INVALID), (dict(heads=0), INVALID), (dict(kv_heads=0), INVALID), (dict(heads=9), INVALID), (dict(dim=80), UNSUPPORTED),
          (dict(dtype=2), UNSUPPORTED), (dict(heads=2048), UNSUPPORTED), (dict(batch=70000), UNSUPPORTED), (dict(scale=-1.0), INVALID),
          (dict(scale=float("nan")), INVALID)]


@pytest.mark.parametrize("bad,want", SHAPES)
def test_shapes_that_are_refused_by_every_call(bad, want):
    L, sh = st3.lib(), shape(**bad)
    assert packed(sh) == want
    assert L.st3_block_store(sh, rows(), rows(), FAKE, 100, 50, cache(), None) == want
    assert L.st3_block_decode(sh, rows(), rows(), rows(), cache(), 50, rows(), None, 0, 0, FAKE, 1 << 30, None) == want
    assert L.st3_block_evict(sh, cache(), cache(k_tail=1 << 40, v_tail=1 << 41), 50, 20, 0, 0, FAKE, 50, 50, FAKE, 50, 50, FAKE, 50, 50, None) == want
    assert L.st3_packed_workspace_bytes(sh, 100) == 0 and L.st3_block_workspace_bytes(sh, 100) == 0
    assert L.st3_packed_attention(None, rows(), rows(), rows(), FAKE, 1, 1, rows(), 0, None, 0, 0, None, 0, None) == INVALID


@pytest.mark.parametrize("bad,want", [
    (dict(cu=None), INVALID), (dict(total=-1), INVALID), (dict(max_len=-1), INVALID), (dict(max_len=101), INVALID), (dict(window=-1), INVALID),
    (dict(window=0), INVALID), (dict(s_h=49), INVALID), (dict(sb=49), INVALID), (dict(ws=None), INVALID), (dict(ws=FAKE + 4), INVALID),
    (dict(wb=100 * 8 * 8 - 1), SMALL), (dict(q=rows(None)), INVALID), (dict(q=rows(FAKE + 2)), INVALID), (dict(k=rows(FAKE, 260, 130)), INVALID),
    (dict(v=rows(FAKE, 0, 128)), INVALID), (dict(q=rows(FAKE, 1024, 64)), INVALID), (dict(k=rows(FAKE, 1 << 26, 128)), UNSUPPORTED)])
def test_packed_attention_refuses(bad, want):
    assert packed(**bad) == want


def test_packed_attention_refuses_an_output_that_shares_memory():
    base = FAKE
    assert packed(out=rows(base)) == INVALID                                    # the queries themselves
    assert packed(out=rows(base + 2 * 50 * 1024)) == INVALID                    # half way into them
    assert packed(k=rows(base + (1 << 29), 256, 128), v=rows(base + (1 << 29) + 512, 256, 128), out=rows(base + (1 << 29) + 256)) == INVALID
    # a workspace that is too small is what remains to be said about slices that alternate
    assert packed(q=rows(base, 2048, 128), out=rows(base + 2 * 1024, 2048, 128), k=rows(base + (1 << 29), 256), v=rows(base + (1 << 29), 256), wb=0) == SMALL
    assert packed(q=rows(base, 2048, 128), out=rows(base + 2 * 1023 // 16 * 16, 2048, 128), k=rows(base + (1 << 29), 256), v=rows(base + (1 << 29), 256), wb=0) == INVALID


def test_nothing_to_attend_is_fine():
    assert packed(total=0, max_len=0) == OK and packed(max_len=0) == OK
    assert st3.lib().st3_block_store(shape(), rows(), rows(), FAKE, 0, 0, cache(), None) == OK


CACHES = [dict([(n, None)]) for n in ("k_codes", "v_codes", "k_scale", "v_scale", "k_tail", "v_tail", "table", "len")] + \
         [dict(table_stride=7), dict(table_blocks=0), dict(n_pages=0), dict(code=2), dict(code=-1), dict(k_codes=FAKE + 8), dict(v_tail=FAKE + 2)]


@pytest.mark.parametrize("bad", CACHES, ids=str)
def test_caches_that_are_refused(bad):
    L, c = st3.lib(), cache(**bad)
    assert L.st3_block_store(shape(), rows(), rows(), FAKE, 100, 50, c, None) == INVALID
    assert L.st3_block_decode(shape(), rows(), rows(), rows(), c, 50, rows(), None, 0, 0, FAKE, 1 << 30, None) == INVALID
    good = cache(k_tail=1 << 40, v_tail=1 << 41)
    assert L.st3_block_evict(shape(), c, good, 50, 20, 0, 0, FAKE, 50, 50, FAKE, 50, 50, FAKE, 50, 50, None) == INVALID
    assert L.st3_block_evict(shape(), good, c, 50, 20, 0, 0, FAKE, 50, 50, FAKE, 50, 50, FAKE, 50, 50, None) == INVALID


def test_blocks_need_bf16_and_a_table_that_reaches():
    L, f32 = st3.lib(), shape(dtype=st3.ST3_F32)
    assert L.st3_block_store(f32, rows(), rows(), FAKE, 100, 50, cache(), None) == UNSUPPORTED
    assert L.st3_block_decode(f32, rows(), rows(), rows(), cache(), 50, rows(), None, 0, 0, FAKE, 1 << 30, None) == UNSUPPORTED
    assert L.st3_block_store(shape(), rows(), rows(), FAKE, 1000, 9 * 64, cache(), None) == INVALID
    assert L.st3_block_store(shape(), rows(), rows(), FAKE, 100, 101, cache(), None) == INVALID
    assert L.st3_block_store(shape(), rows(), rows(), None, 100, 50, cache(), None) == INVALID


def decode(k=True, v=True, top=50, score=None, sb=0, sh=0, ws=FAKE, wb=1 << 30, q=None, c=None):
    return st3.lib().st3_block_decode(shape(), q or rows(), rows() if k else None, rows() if v else None, c or cache(), top, rows(), score, sb, sh, ws,
                                      wb, None)


def test_decode_refuses():
    need = st3.st3_block_workspace_bytes(st3.gqa_shape(2, 8, 2, 128), 50)
    assert need > 0
    for bad, want in ((dict(v=False), INVALID), (dict(k=False), INVALID), (dict(top=-1), INVALID), (dict(ws=None), INVALID), (dict(ws=FAKE + 4), INVALID),
                      (dict(wb=need - 1), SMALL), (dict(q=rows(FAKE + 2)), INVALID), (dict(top=8 * 64 + 63), INVALID),
                      (dict(score=FAKE, sb=50, sh=51), INVALID), (dict(score=FAKE, sb=51, sh=50), INVALID)):
        assert decode(**bad) == want, bad


def test_workspaces_grow_with_what_they_hold():
    s = st3.gqa_shape(4, 8, 2, 128)
    sizes = [st3.st3_block_workspace_bytes(s, n) for n in (0, 63, 64, 1000, 100000)]
    assert sizes == sorted(sizes) and sizes[0] > 0 and sizes[0] == sizes[1]
    assert st3.st3_packed_workspace_bytes(s, 1000) >= 1000 * 8 * 8


def evict(frm=None, to=None, top=50, keep=20, sink=0, recent=0, score=FAKE, sb=50, sh=50, ts=FAKE, tb=20, th=20, kept=FAKE, ib=20, ih=20):
    return st3.lib().st3_block_evict(shape(), frm or cache(), to or cache(k_tail=1 << 40, v_tail=1 << 41), top, keep, sink, recent, score, sb, sh, ts, tb, th,
                                     kept, ib, ih, None)


@pytest.mark.parametrize("bad", [
    dict(to=cache(code=st3.ST3_BLOCK_E4M3, k_tail=1 << 40, v_tail=1 << 41)), dict(score=None), dict(ts=None), dict(kept=None), dict(top=-1), dict(keep=0),
    dict(sink=-1), dict(recent=-1), dict(sink=11, recent=10), dict(sink=2 ** 31 - 1, recent=2 ** 31 - 1), dict(sh=49), dict(sb=49), dict(th=19),
    dict(tb=19), dict(ih=19), dict(ib=19), dict(to=cache()), dict(to=cache(k_tail=1 << 40)), dict(to=cache(k_tail=FAKE + 2 * 2 * 2 * 64 * 128 - 16, v_tail=1 << 41)),
    dict(top=9 * 64 + 5), dict(top=700, keep=600, sb=700, sh=700, tb=600, th=600, ib=600, ih=600, frm=cache(table_blocks=20, table_stride=20))], ids=str)
def test_evict_refuses(bad):
    assert evict(**bad) == INVALID


# ---- the oracle -------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("H,Hk", [(4, 4), (6, 2), (3, 1)])
def test_oracle_packed_attention_is_the_library_attention_of_each_sequence(H, Hk):
    rng, lens, d = np.random.default_rng(1), [7, 0, 1, 12], 16
    q, k, v = (rng.standard_normal((20, h, d)) for h in (H, Hk, Hk))
    out, scores = bo.packed_attention(q, k, v, lens, 0.25, 3)
    start = 0
    for b, n in enumerate(lens):
        if n:
            t = [torch.from_numpy(x[start:start + n]).transpose(0, 1) for x in (q, k, v)]
            t[1], t[2] = (x.repeat_interleave(H // Hk, 0) for x in t[1:])
            want = torch.nn.functional.scaled_dot_product_attention(*(x[None] for x in t), is_causal=True, scale=0.25)[0]
            np.testing.assert_allclose(out[start:start + n], want.transpose(0, 1).numpy(), atol=1e-12)
            np.testing.assert_allclose(scores[b].sum(), H * min(3, n))          # every row's weights sum to one
        start += n


def test_oracle_quantizer():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((64, 8)).astype(np.float32)
    for code, top, step in (("int8", 127, 0.5), ("e4m3", 448, 16)):
        c, s = bo.quantize_block(x, code)
        assert np.abs(c).max() == top and s == np.float32(np.abs(x).max()) * (np.float32(1) / np.float32(top))
        assert np.all(np.abs(c * s - x) <= step * s * (1 + 1e-6))
        z, s = bo.quantize_block(np.zeros((64, 8)), code)
        assert s == 0 and not z.any()
    # hand-worked: largest value 127 makes the scale 1; halves go to even
    y = np.zeros((64, 8), np.float32)
    y[0, :6] = [127, 0.5, 1.5, -2.5, 126.5, -0.5]
    np.testing.assert_array_equal(bo.quantize_block(y, "int8")[0][0, :6], [127, 0, 2, -2, 126, 0])
    y[0, :6] = [448, 17, 19, 2.0 ** -10, 3 * 2.0 ** -10, -1000]
    y[0, 5] = -448
    np.testing.assert_array_equal(bo.quantize_block(y, "e4m3")[0][0, :6], [448, 16, 20, 0, 2.0 ** -8, -448])
    y[0, :4] = [448, np.nan, np.inf, -np.inf]
    c, s = bo.quantize_block(y, "e4m3")
    assert s == 1 and np.isnan(c[0, 1]) and c[0, 2] == 448 and c[0, 3] == -448


def test_oracle_kept_rows():
    assert list(bo.kept_rows(np.array([1., 2, 3]), 3, 0, 0)) == [0, 1, 2]
    assert list(bo.kept_rows(np.array([5., 1, 1, 1, 4]), 3, 0, 0)) == [0, 1, 4]               # a tie: the lower row
    assert list(bo.kept_rows(np.array([0., 9, 8, 0, 0]), 3, 1, 1)) == [0, 1, 4]
    assert list(bo.kept_rows(np.array([0., np.nan, -np.inf, -0.0, 0.0]), 3, 0, 0)) == [0, 3, 4]


def test_oracle_cache_appends_like_it_was_stored_at_once():
    rng = np.random.default_rng(3)
    k, v = rng.standard_normal((2, 200, 8)).astype(np.float32).astype(np.float64)
    for code in ("int8", "e4m3"):
        one, many = bo.BlockCache(1, 1, 8, code), bo.BlockCache(1, 1, 8, code)
        one.append(0, 0, k, v)
        for i in range(200):
            many.append(0, 0, k[i:i + 1], v[i:i + 1])
        assert one.length(0) == many.length(0) == 200
        for a, b in zip(one.values(0, 0), many.values(0, 0)):
            np.testing.assert_array_equal(a, b)
        assert np.abs(one.values(0, 0)[0] - k).max() < 0.3


def test_binding_refuses_what_the_library_cannot_see():
    s = st3.gqa_shape(2, 4, 2, 64)
    with pytest.raises((ValueError, TypeError)):
        st3._rows(s, torch.zeros(3, 4, 64), 4, 3)                                # not on the device
    with pytest.raises(ValueError):
        st3._rows(s, torch.zeros(3, 4, 32, dtype=torch.bfloat16), 4, 3)
    with pytest.raises(TypeError):
        st3._scores(s, torch.zeros(2, 2, 9), "score", 9)
    with pytest.raises(ValueError):
        st3.block_cache(*(torch.zeros(1, 2, 32, 64, dtype=torch.int8) for _ in range(2)), *(torch.zeros(1, 2) for _ in range(2)),
                        *(torch.zeros(2, 2, 64, 64) for _ in range(2)), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))


@pytest.mark.parametrize("batch,heads,kv_heads,dim", [(1, 32, 8, 128), (4, 32, 8, 128), (2, 40, 40, 128), (8, 16, 1, 64), (32, 32, 8, 128), (3, 48, 2, 64)])
def test_workspace_for_the_longest_is_enough_for_every_shorter_cache(batch, heads, kv_heads, dim):
    shape = st3.gqa_shape(batch, heads, kv_heads, dim)
    sizes = [st3.st3_block_workspace_bytes(shape, n) for n in [*range(0, 70000, 37), *range(63, 20000, 64)]]
    by_length = [s for _, s in sorted(zip([*range(0, 70000, 37), *range(63, 20000, 64)], sizes))]
    assert by_length == sorted(by_length)


@pytest.mark.parametrize("change", [dict(layers=0), dict(budget=0), dict(budget=256), dict(n_sink=-1), dict(n_sink=100, n_recent=29), dict(window=0), dict(code=7)])
def test_generation_refuses_before_it_allocates(change):
    from paper_2412_20105_amd.block_pipeline import BlockGeneration

    good = dict(layers=2, heads=8, kv_heads=2, head_dim=128, batch=2, capacity=256, budget=128, n_sink=4, n_recent=64, window=32)
    with pytest.raises(ValueError):
        BlockGeneration(**{**good, **change})
