"""Decode over blocks in every form that the rule on sizes can take: whole strips by four and by twelve waves, short and long, chunks of both head sizes with
and without scores, groups of more heads than a workgroup has columns.  Each case names the form that it is meant to reach."""
import numpy as np
import pytest
import torch

import decode_cut
from block_util import BLOCK, DeviceCache, code_values, fp32_slack
from gpu_util import DEV, to_np64
from oracle import block_oracle as bo
from paper_2412_20105_amd import binding as st3

pytestmark = pytest.mark.gpu

HALF, SPLIT = 2.0 ** -8, 2.0 ** -15         # half a step of bf16; a weight held as two bf16 terms


def random_cache(rng, lens, Hk, d, code):
    """Pages, scales and tails drawn on the device, as blocks of normal values have them."""
    B, g = len(lens), torch.Generator(device=DEV).manual_seed(int(rng.integers(1 << 30)))
    dev = DeviceCache(rng, B, Hk, d, code, max(lens) // BLOCK + 1)
    for x in (dev.k_codes, dev.v_codes):
        y = torch.randn(x.shape, generator=g, device=DEV)
        x.copy_((y * 31).round_().clamp_(-127, 127).to(torch.int8) if code == "int8" else (y * 112).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    for x in (dev.k_scale, dev.v_scale):
        x.copy_((0.8 + 0.4 * torch.rand(x.shape, generator=g, device=DEV)) * (1.5 / (31 if code == "int8" else 112)))
    for b, n in enumerate(lens):            # (what lies behind the rows that exist stays NaN)
        r = max(n, 0) % BLOCK
        dev.k_tail[b, :, :r] = (1.5 * torch.randn((Hk, r, d), generator=g, device=DEV)).bfloat16()
        dev.v_tail[b, :, :, :r] = (1.5 * torch.randn((Hk, d, r), generator=g, device=DEV)).bfloat16()
    dev.set_len(lens)
    return dev


def values(dev, b, n, name):
    """Rows 0 .. n - 1 of sequence b in 64 bits, [Hk, n, d]."""
    pages = dev.table[b, :n // BLOCK].long()
    x = getattr(dev, name + "_codes")[pages]
    x = (x if dev.code == "int8" else x.view(torch.float8_e4m3fn).float()).double() * getattr(dev, name + "_scale")[pages].double()[..., None, None]
    tail = getattr(dev, name + "_tail")[b].double()
    if name == "v":
        x, tail = x.transpose(-1, -2), tail.transpose(-1, -2)
    return torch.cat([x.transpose(0, 1).reshape(dev.kv_heads, -1, dev.dim), tail[:, :n % BLOCK]], 1)


SHORT, LONG = [700, 1, 64, 511, 0, 63, 1023, 128, 129, -1], [1400, 1535, 3500, 63, 0, 2111, 1300, 64, -1, 127]


def some(lens, n):
    return [lens[i % len(lens)] for i in range(n)]


# lens, heads, key heads, head size, scored, a new row; (waves, whole strips) that this is meant to reach
CASES = [
    (some(LONG, 25), 16, 8, 128, True, True, (12, True)), (some(LONG, 25), 16, 8, 64, True, True, (12, True)),
    (some(LONG, 25), 16, 8, 128, False, True, (12, True)), (some(LONG, 25), 24, 8, 64, True, False, (12, True)),
    (some(SHORT, 24), 32, 8, 128, True, True, (12, True)),
    (some(SHORT, 10), 30, 30, 128, True, True, (4, True)), (some(SHORT, 10), 30, 30, 64, True, True, (4, True)),
    (some(LONG, 10), 30, 30, 128, True, True, (4, True)), (some(LONG, 10), 30, 30, 64, True, False, (4, True)),
    (some(LONG, 10), 30, 30, 128, False, True, (4, True)), (some(LONG, 10), 60, 30, 64, False, False, (4, True)),
    (some(LONG, 10), 480, 30, 128, False, True, (4, True)),
    ([1500, 5000], 4, 1, 64, True, True, (4, False)), ([1500, 5000], 4, 1, 64, False, True, (4, False)), ([5000, 1500, 0, -1], 14, 2, 64, True, False, (4, False)),
    ([1500, 5000], 4, 1, 128, False, True, (4, False)), ([5000, 63, 1], 8, 2, 128, False, False, (4, False)), ([9000, 4095], 4, 4, 128, True, True, (4, False)),
    (some(SHORT, 8), 17, 1, 128, False, True, (12, True)), (some(SHORT, 8), 40, 1, 64, False, True, (12, True)), (some(SHORT, 40), 80, 2, 128, False, True, (12, True)),
    (some(SHORT, 44), 80, 2, 64, False, False, (4, True)), ([5000, 300], 17, 1, 64, False, True, (4, False)), ([5000, 300], 40, 1, 128, False, True, (4, False)),
    (some(SHORT, 8), 17, 1, 64, True, True, (4, False)), ([5000, 300], 40, 1, 128, True, True, (4, False)), ([2000, 300], 40, 1, 64, True, True, (4, False)),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{len(c[0])}x{c[2]}-{c[1] // c[2]}h-{max(c[0])}-d{c[3]}{'-scored' if c[4] else ''}{'' if c[5] else '-no_row'}")
@pytest.mark.parametrize("code", ["int8", "e4m3"])
def test_every_form(case, code):
    lens, H, Hk, d, scored, fresh, form = case
    B, G, top = len(lens), H // Hk, max(lens)
    waves, chunk, _ = decode_cut.cut(B, H, Hk, d, top, scored)
    assert (waves, chunk == 0) == form
    rng = np.random.default_rng(B + H + d + top)
    dev = random_cache(rng, lens, Hk, d, code)
    x = torch.from_numpy(rng.standard_normal((B, H + 2 * Hk, d)).astype(np.float32) * np.float32(1.5)).to(DEV).bfloat16()
    q, k, v = x[:, :H], x[:, H:H + Hk], x[:, H + Hk:]
    score = torch.from_numpy(rng.exponential(size=(B, Hk, top + 3)).astype(np.float32)).to(DEV)
    before, out = score.double(), torch.full((B, H, d), 7.0, dtype=torch.bfloat16, device=DEV)
    want, spread, weight, most, coded = torch.zeros((B, H, d), dtype=torch.float64, device=DEV), torch.zeros((B, H, d), dtype=torch.float64, device=DEV), {}, {}, {}
    for b, n in enumerate(lens):
        if n < 0:
            continue
        kk, vv = values(dev, b, n, "k"), values(dev, b, n, "v")
        if fresh:
            kk, vv = torch.cat([kk, k[b].double()[:, None]], 1), torch.cat([vv, v[b].double()[:, None]], 1)
        if kk.shape[1] == 0:
            continue
        qq = q[b].double().reshape(Hk, G, d)
        p = torch.softmax(torch.matmul(qq, kk.transpose(1, 2).contiguous()) / np.sqrt(d), -1)
        want[b], spread[b], weight[b] = torch.matmul(p, vv).view(H, d), torch.matmul(p, vv.abs()).view(H, d), p.sum(1)
        most[b] = float(torch.matmul(qq.abs(), kk.abs().transpose(1, 2).contiguous()).max()) / np.sqrt(d)
        if fresh and n % BLOCK == BLOCK - 1:
            coded[b] = [[bo.quantize_block(t[h, n - BLOCK + 1:].float().cpu().numpy(), code) for h in range(Hk)] for t in (kk, vv)]
    tails = dev.k_tail.clone(), dev.v_tail.clone()
    shape = st3.gqa_shape(B, H, Hk, d)
    ws = torch.full((st3.st3_block_workspace_bytes(shape, top),), 0xff, dtype=torch.uint8, device=DEV)
    st3.st3_block_decode(shape, q, k if fresh else None, v if fresh else None, dev.c, top, out, score if scored else None, ws)
    torch.cuda.synchronize()
    after = score.double()
    for b, n in enumerate(lens):
        m, slack = max(n, 0) + (1 if fresh and n >= 0 else 0), fp32_slack(max(most.get(b, 1.0), 1.0), d, max(n, 0) + 1)
        bound = HALF * 1.01 * want[b].abs() + (SPLIT + 2 * slack) * spread[b] + 1e-30
        assert bool(((out[b].double() - want[b]).abs() <= bound).all()), (b, n, float(((out[b].double() - want[b]).abs() / bound).max()))
        if scored and b in weight:
            full = weight[b].clone()
            full[:, :n] += before[b, :, :n]
            assert bool(((after[b, :, :m] - full).abs() <= 2 * slack * weight[b] + 2.0 ** -23 * full.abs() + 1e-30).all()), (b, n)
            assert torch.equal(after[b, :, m:], before[b, :, m:])
        else:
            assert torch.equal(after[b], before[b])
        if fresh and n >= 0:
            tails[0][b, :, n % BLOCK], tails[1][b, :, :, n % BLOCK] = k[b], v[b]
        if b in coded:
            page = int(dev.table[b, n // BLOCK])
            for which, (codes, scale) in enumerate(((dev.k_codes, dev.k_scale), (dev.v_codes, dev.v_scale))):
                got = code_values(codes[page])
                for h in range(Hk):
                    c, s = coded[b][which][h]
                    np.testing.assert_array_equal(got[h].T if which else got[h], c, err_msg=f"{b} {h}")
                    assert to_np64(scale)[page, h] == s
    for old, new in zip(tails, (dev.k_tail, dev.v_tail)):
        assert torch.equal(old.nan_to_num(nan=9.0), new.nan_to_num(nan=9.0))
