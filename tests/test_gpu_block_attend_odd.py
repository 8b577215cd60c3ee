"""st3_block_attend where logits are not finite and where blocks' scales are extreme, in every form of the launch."""
import numpy as np
import pytest
import torch

from block_util import BLOCK, fp32_slack
from gpu_util import DEV
from paper_2412_20105_amd import binding as st3
from test_gpu_block_attend import HALF, run

pytestmark = pytest.mark.gpu

# rows in front, new tokens, query heads, key heads, d
FORMS = {
    "few_whole_scored_at_once": (190, 3, 4, 2, 64),         # weights from logits in LDS
    "few_odd_columns": (190, 3, 10, 2, 128),                # 15 rows of a key head
    "few_two_columns": (190, 5, 8, 2, 128),                 # 20 rows
    "few_two_groups": (190, 32, 4, 2, 128),                 # 32 rows each, scores formed again
    "few_pieces": (5000, 3, 8, 2, 128),                     # and joined
    "few_pieces_of_two_groups": (5000, 22, 4, 2, 64),
    "tiles": (100, 50, 4, 2, 128),
    "tiles_of_two_columns": (60, 150, 4, 2, 64),
    "tiles_in_pieces": (3000, 50, 4, 2, 128),
    "tiles_of_two_columns_in_pieces": (3000, 150, 4, 2, 64),
}


def rows_of(dev, length, name):
    """K or V of sequence 0's rows, float64 [Hk, length, d], as the cache holds them; those of a block without a page are 0."""
    kind, blocks = torch.int8 if dev.code == "int8" else torch.float8_e4m3fn, length // BLOCK
    pages = dev.table[0, :blocks].long()
    gone = (pages < 0) | (pages >= len(dev.k_codes))
    pages = pages.masked_fill(gone, 0)
    codes = getattr(dev, name + "_codes")[pages].view(kind).float().double() * getattr(dev, name + "_scale")[pages].double()[..., None, None]
    codes[gone] = 0.0
    tail = getattr(dev, name + "_tail")[0].double()
    if name == "v":
        codes, tail = codes.transpose(2, 3), tail.transpose(1, 2)
    codes = codes.permute(1, 0, 2, 3).reshape(dev.kv_heads, blocks * BLOCK, dev.dim)
    return torch.cat([codes, tail[:, :length % BLOCK]], 1)


def check(dev, q, old, new, window, out, score, before, tiny=1e-30, weight=HALF):
    """Against the definition in 64 bits: what is NaN, and how far the rest is off (the output's rounding, and that of every weight: `weight` of it)."""
    both, H, Hk, d = old + new, q.shape[1], dev.kv_heads, dev.dim
    k, v = rows_of(dev, both, "k"), rows_of(dev, both, "v")
    see = torch.arange(both, device=DEV) <= old + torch.arange(new, device=DEV)[:, None]
    counts = torch.arange(new, device=DEV) >= new - window
    pages = dev.table[0, :both // BLOCK]
    there = torch.ones(both, dtype=torch.bool, device=DEV)
    there[:both // BLOCK * BLOCK] = ((pages >= 0) & (pages < len(dev.k_codes))).repeat_interleave(BLOCK)
    see = see & there
    for kh in range(Hk):
        given, odd_keys = torch.zeros(both, dtype=torch.float64, device=DEV), torch.zeros(both, dtype=torch.bool, device=DEV)
        slack = 0.0
        for h in range(kh * (H // Hk), (kh + 1) * (H // Hk)):
            x = q[:new, h].double()
            logits = (x @ k[kh].t() / np.sqrt(d)).masked_fill(~see, -torch.inf)     # (a product with an infinite element is infinite or NaN, as in float32)
            odd = (torch.isnan(logits) | (logits == torch.inf)).any(-1)
            p = torch.softmax(logits.masked_fill(odd[:, None], 0.0), -1).nan_to_num(nan=0.0) * see          # (nothing to see: 0)
            worst = float((x.nan_to_num(nan=0.0, posinf=0.0, neginf=0.0).abs() @ k[kh].nan_to_num(nan=0.0, posinf=0.0, neginf=0.0).abs().t()).max()) / np.sqrt(d)
            slack = max(slack, fp32_slack(worst, d, both))
            want, spread, got = p @ v[kh], p @ v[kh].abs(), out[:new, h].double()
            assert bool(torch.isnan(got[odd]).all()), (h, "a logit that is NaN or +infinity")
            bound = (HALF * want.abs() + weight * spread) * 1.01 + slack * spread + tiny
            assert bool(((got - want).abs() <= bound)[~odd].all()), (h, float(((got - want).abs() / bound)[~odd].max()))
            given += p[counts & ~odd].sum(0)
            odd_keys |= see[counts & odd].any(0)
        s, first = score[0, kh].double(), before[0, kh].double()
        assert torch.equal(s[both:], first[both:])
        assert bool(torch.isnan(s[:both][odd_keys]).all()), (kh, "scores of a row of NaN")
        full = given.clone()
        full[:old] += first[:old]
        room = 2 * slack * given + 2.0 ** -23 * full + 1e-30
        assert bool(((s[:both] - full).abs() <= room)[~odd_keys].all()), (kh, float(((s[:both] - full).abs() / room)[~odd_keys].max()))
        untouched = (~odd_keys) & (given == 0) & (torch.arange(both, device=DEV) < old)
        assert torch.equal(s[:both][untouched], first[:both][untouched])


def prepared(form, code, window, seed):
    old, new, H, Hk, d = FORMS[form]
    return run(np.random.default_rng(seed), [old], [new], H, Hk, d, code, window)[2]


def call(state, q, window):
    shape, _, at, most, dev, top, ws, before = state
    out, score = torch.full((q.shape[0], q.shape[1], dev.dim), 7.0, dtype=torch.bfloat16, device=DEV), before.clone()
    ws.fill_(255)
    st3.st3_block_attend(shape, q, at, most, dev.c, top, out, window, score, ws)
    torch.cuda.synchronize()
    return out, score


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("window", [1, 50])
def test_queries_that_are_not_finite(form, window):
    """One head of the first, of a middle and of the last token."""
    old, new, H, Hk, d = FORMS[form]
    state = prepared(form, "int8", window, 1)
    for t in sorted({0, new // 2, new - 1}):
        for value in (float("nan"), float("inf")):
            q = state[1].clone()
            q[t, 1, 5] = value                              # (times keys of either sign: logits of +infinity, -infinity and perhaps NaN)
            out, score = call(state, q, window)
            check(state[4], q, old, new, window, out, score, state[-1])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("window", [1, 50])
@pytest.mark.parametrize("where", ["first_block", "own_block", "tail"])
def test_keys_that_are_no_numbers(form, window, where):
    """A code of NaN in a block that all rows see whole, in the last whole block, which new rows may lie in, and NaN and infinities in the tail."""
    old, new, H, Hk, d = FORMS[form]
    both = old + new
    state = prepared(form, "e4m3", window, 2)
    dev, q = state[4], state[1].clone()
    q[:, :, 3] = q[:, :, 3].abs() + 0.5                     # (a key's infinity keeps its sign)
    if where == "tail":
        for value in (float("nan"), float("inf")):
            keep = dev.k_tail.clone()
            dev.k_tail[0, 0, both % BLOCK - 1, 3] = value   # the last token's own row
            out, score = call(state, q, window)
            check(dev, q, old, new, window, out, score, state[-1])
            dev.k_tail.copy_(keep)
        dev.k_tail[0, 0, both % BLOCK - 1, 3] = -float("inf")
    else:
        j = 5 if where == "first_block" else both // BLOCK * BLOCK - 1
        dev.k_codes[int(dev.table[0, j // BLOCK]), 0, j % BLOCK, 3] = 0x7f
    out, score = call(state, q, window)
    check(dev, q, old, new, window, out, score, state[-1])


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("window", [1, 50])
def test_nothing_but_minus_infinity(form, window):
    """No page but the first is there, or none, and all keys of the tail are -infinity: out = 0 where a token sees nothing else, and no weight."""
    old, new, H, Hk, d = FORMS[form]
    state = prepared(form, "e4m3", window, 3)
    dev, q = state[4], state[1].clone()
    q[:, :, 3] = q[:, :, 3].abs() + 0.5
    dev.k_tail[0, :, :, 3] = -float("inf")
    dev.table[0, 1:] = -1
    out, score = call(state, q, window)
    check(dev, q, old, new, window, out, score, state[-1])
    dev.table[0, 0] = len(dev.k_codes)
    out, score = call(state, q, window)
    check(dev, q, old, new, window, out, score, state[-1])
    assert not out[:new].any() and torch.equal(score[0, :, :old], state[-1][0, :, :old]) and not score[0, :, old:old + new].any()


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("value", ["zero", "smallest", "largest"])
def test_scales_at_either_end(form, code, value):
    """The scales of the first blocks and of the last whole one, at whose edge masked logits are -infinity."""
    old, new, H, Hk, d = FORMS[form]
    both = old + new
    state = prepared(form, code, 50, 4)
    dev, q = state[4], (state[1].float() * 0.25).bfloat16()
    most = {"zero": 0.0, "smallest": 1e-38, "largest": 0.7 * 2.0 ** 119 / both}[value]      # (what the header leaves for |v|)
    for j in {0, 1, both // BLOCK - 1}:
        page = int(dev.table[0, j])
        dev.k_scale[page] = 0.0 if value == "zero" else 1e-38
        dev.v_scale[page] = most / 448
    out, score = call(state, q, 50)
    # below the smallest normal bf16 (2^-126) a rounding of a weight or of the output is a step of 2^-133 instead, or the value is lost
    check(dev, q, old, new, 50, out, score, state[-1], tiny=both * 127 * 2.0 ** -126)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("window", [0, 50])
def test_values_that_are_no_numbers(form, window):
    """Codes of NaN among V in blocks that new rows lie in, several in a column, and NaN in the tail: NaN for the rows that see one, in its column alone."""
    old, new, H, Hk, d = FORMS[form]
    both, rng = old + new, np.random.default_rng(5)
    state = prepared(form, "e4m3", window, 6)
    dev, q, last = state[4], state[1], both // BLOCK * BLOCK
    nan = torch.zeros((Hk, both, d), dtype=torch.bool, device=DEV)
    for j in [old, old + 1, last - 1, last - 2, last - 40, last - 64, both - 1, both - 2, *rng.integers(max(0, last - 64), both, 8).tolist()]:
        h, col = int(rng.integers(Hk)), int(rng.integers(d))
        for c in {col, 7}:
            nan[h, j, c] = True
            if j >= last:
                dev.v_tail[0, h, c, j - last] = float("nan")
            else:
                dev.v_codes[int(dev.table[0, j // BLOCK]), h, c, j % BLOCK] = int(rng.choice([0x7f, 0xff]))
    out, score = call(state, q, window) if window else (call_unscored(state, q), None)
    k, v = rows_of(dev, both, "k"), rows_of(dev, both, "v")
    assert torch.equal(torch.isnan(v), nan)
    see = torch.arange(both, device=DEV) <= old + torch.arange(new, device=DEV)[:, None]
    for h in range(H):
        kh = h // (H // Hk)
        x = q[:new, h].double()
        p = torch.softmax((x @ k[kh].t() / np.sqrt(d)).masked_fill(~see, -torch.inf), -1)
        slack = fp32_slack(float((x.abs() @ k[kh].abs().t()).max()) / np.sqrt(d), d, both)
        odd, clean, got = (see.double() @ nan[kh].double()) > 0, v[kh].nan_to_num(nan=0.0), out[:new, h].double()
        assert torch.equal(torch.isnan(got), odd), h
        want, spread = p @ clean, p @ clean.abs()
        assert bool(((got - want).abs() <= HALF * (want.abs() + spread) * 1.01 + slack * spread)[~odd].all())
    if window:                                              # (weights have nothing to do with values)
        assert bool(torch.isfinite(score).all())


def call_unscored(state, q):
    shape, _, at, most, dev, top, ws, _ = state
    out = torch.full((q.shape[0], q.shape[1], dev.dim), 7.0, dtype=torch.bfloat16, device=DEV)
    st3.st3_block_attend(shape, q, at, most, dev.c, top, out, 0, None, ws)
    torch.cuda.synchronize()
    return out
