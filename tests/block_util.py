"""Caches of 8-bit blocks on the device beside the oracle's, for the tests of the grouped-head calls."""
import numpy as np
import torch

from gpu_util import DEV, rand_values, to_np64
from oracle import block_oracle as bo
from paper_2412_20105_amd import binding as st3
from workloads.synth import bf16_bits_to_f32, bf16_round_bits

BLOCK = bo.BLOCK


def bf16(x):
    return bf16_bits_to_f32(bf16_round_bits(np.asarray(x, np.float32))).astype(np.float64)


def code_values(t: torch.Tensor) -> np.ndarray:
    return to_np64(t if t.dtype == torch.int8 else t.view(torch.float8_e4m3fn).float())


class DeviceCache:
    """Pools, tails and table; pages in a shuffled order, `spare` of them left for a second table."""

    def __init__(self, rng, batch, kv_heads, dim, code, blocks, pool=None, pages=None, names=None):
        self.batch, self.kv_heads, self.dim, self.code, self.blocks = batch, kv_heads, dim, code, blocks
        dt = torch.int8 if code == "int8" else torch.uint8
        pages = pages or 2 * batch * blocks + 2
        if pool is None:
            # whatever lies in pages and tails that nothing was written to
            self.k_codes = torch.randint(0, 256, (pages, kv_heads, BLOCK, dim), dtype=torch.uint8, device=DEV).view(dt)
            self.v_codes = torch.randint(0, 256, (pages, kv_heads, dim, BLOCK), dtype=torch.uint8, device=DEV).view(dt)
            self.k_scale = torch.full((pages, kv_heads), float("nan"), device=DEV)
            self.v_scale = torch.full((pages, kv_heads), float("nan"), device=DEV)
            order = rng.permutation(pages).astype(np.int32)
        else:
            self.k_codes, self.v_codes, self.k_scale, self.v_scale = pool.k_codes, pool.v_codes, pool.k_scale, pool.v_scale
            order = pool.free
        names = order[:batch * blocks] if names is None else names
        self.free = order[batch * blocks:]
        self.k_tail = torch.full((batch, kv_heads, BLOCK, dim), float("nan"), dtype=torch.bfloat16, device=DEV)
        self.v_tail = torch.full((batch, kv_heads, dim, BLOCK), float("nan"), dtype=torch.bfloat16, device=DEV)
        self.table = torch.from_numpy(np.ascontiguousarray(names.reshape(batch, blocks))).to(DEV)
        self.len = torch.zeros(batch, dtype=torch.int32, device=DEV)
        self.describe()

    def describe(self):
        self.c = st3.block_cache(self.k_codes, self.v_codes, self.k_scale, self.v_scale, self.k_tail, self.v_tail, self.table, self.len)

    def set_len(self, lens):
        self.len.copy_(torch.tensor(lens, dtype=torch.int32))

    def check(self, cache: bo.BlockCache, sequences=None):
        """Codes, scales and tails equal the oracle's, bit for bit."""
        pages = self.table.clamp(0, len(self.k_codes) - 1).long().view(-1)        # (a pool may be far larger than what is used of it)
        table = np.arange(len(pages)).reshape(self.table.shape)
        kc, vc = code_values(self.k_codes[pages]), code_values(self.v_codes[pages])
        ks, vs, kt, vt = (to_np64(x) for x in (self.k_scale[pages], self.v_scale[pages], self.k_tail, self.v_tail))
        for b in range(self.batch) if sequences is None else sequences:
            for h in range(self.kv_heads):
                for j, ((k, s), (v, z)) in enumerate(cache.blocks[b][h]):
                    page = table[b, j]
                    assert ks[page, h] == s and vs[page, h] == z, (b, h, j, ks[page, h], s)
                    np.testing.assert_array_equal(kc[page, h], k, err_msg=f"K codes {b} {h} {j}")
                    np.testing.assert_array_equal(vc[page, h].T, v, err_msg=f"V codes {b} {h} {j}")
                k, v = cache.tail[b][h]
                np.testing.assert_array_equal(kt[b, h, :len(k)], k, err_msg=f"K tail {b} {h}")
                np.testing.assert_array_equal(vt[b, h, :, :len(v)].T, v, err_msg=f"V tail {b} {h}")


def filled(rng, lens, kv_heads, dim, code, blocks, **more):
    """A device cache holding random rows of these lengths (through the store), and the oracle's."""
    batch, total = len(lens), sum(lens)
    k, v = (rand_values(rng, (total, kv_heads, dim), "bf16", 1.5) for _ in range(2))
    dev = DeviceCache(rng, batch, kv_heads, dim, code, blocks, **more)
    shape = st3.gqa_shape(batch, kv_heads, kv_heads, dim)
    cu = torch.tensor([0, *np.cumsum(lens)], dtype=torch.int32, device=DEV)
    if total:
        st3.st3_block_store(shape, torch.from_numpy(k).to(DEV).bfloat16(), torch.from_numpy(v).to(DEV).bfloat16(), cu, max(lens), dev.c)
    dev.set_len(lens)
    ref = bo.BlockCache(batch, kv_heads, dim, code)
    start = 0
    for b, n in enumerate(lens):
        for h in range(kv_heads):
            ref.append(b, h, k[start:start + n, h].astype(np.float64), v[start:start + n, h].astype(np.float64))
        start += n
    return dev, ref


def fp32_slack(q_abs_k, dim, n):
    """Relative error of a softmax weight formed in float32: a dot product of `dim` terms whose magnitudes sum to q_abs_k (scale
    included), in numerator and normaliser alike, the exponential and the scale (8 steps), and a sum of n weights."""
    step = 2.0 ** -24
    return 2 * (dim + 8) * step * float(q_abs_k) + (n + 32) * step
