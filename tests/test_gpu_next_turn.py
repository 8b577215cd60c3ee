"""The calls of a further turn together, as BlockGeneration makes them: tables, prompts, decode steps, turns and evictions, against the oracle."""
import numpy as np
import pytest
import torch

from block_util import bf16, code_values, fp32_slack
from gpu_util import DEV, rand_values, to_np64
from oracle import block_oracle as bo
from paper_2412_20105_amd import binding as st3
from paper_2412_20105_amd.block_pipeline import BlockGeneration
from test_gpu_block_pipeline import check_cache, close

pytestmark = pytest.mark.gpu

CODES = {"int8": st3.ST3_BLOCK_INT8, "e4m3": st3.ST3_BLOCK_E4M3}


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("lens,H,Hk,d,pairs,adjacent", [([70, 3, 129, 0], 4, 2, 64, 24, False), ([100, -1, 60], 6, 1, 128, 64, True)])
def test_prompts_turns_steps_and_evictions(lens, H, Hk, d, pairs, adjacent, code):
    rng = np.random.default_rng(sum(lens) + d)
    L, B, G, W, sinks, recent, capacity, budget = 2, len(lens), H // Hk, 5, 1, 1, 200, 110
    gen = BlockGeneration(L, H, Hk, d, B, capacity, budget, sinks, recent, W, CODES[code])
    scale, layout = 1.0 / np.sqrt(d), st3.ST3_ROTARY_ADJACENT if adjacent else st3.ST3_ROTARY_HALVES
    inv_freq = (10000.0 ** (-np.arange(pairs) / pairs)).astype(np.float32)
    freq_dev, axis = torch.from_numpy(inv_freq).to(DEV), [c % 3 for c in range(pairs)]
    gen.begin(lens)
    T = sum(max(n, 0) for n in lens)
    refs = [bo.BlockCache(B, Hk, d, code) for _ in range(L)]
    scores = [[np.zeros((Hk, 0)) for _ in range(B)] for _ in range(L)]
    worst = 0.0
    for l in range(L):
        qkv = rand_values(rng, (T, H + 2 * Hk, d), "bf16", 1.2)
        dev = torch.from_numpy(qkv).to(DEV).bfloat16()
        q, k, v = (np.asarray(x, np.float64) for x in (qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]))
        gen.prefill_layer(l, dev[:, :H], dev[:, H:H + Hk], dev[:, H + Hk:])
        worst = max(worst, 2 * float(np.abs(q).max() * np.abs(k).max()) * d * scale)       # (turned columns: up to sqrt 2 of each)
        first, start = bo.packed_attention(q, k, v, [max(n, 0) for n in lens], scale, W)[1], 0
        for b, n in enumerate(lens):
            for h in range(Hk):
                refs[l].append(b, h, k[start:start + max(n, 0), h], v[start:start + max(n, 0), h])
            scores[l][b] = first[b]
            start += max(n, 0)
    live = [n >= 0 for n in lens]
    for turn in range(4):
        new = [[5, 30, 1, 64], [60, 0, 70, 65], [1, 1, 0, 2], [40, 90, 80, 70]][turn][:B]
        new = [m if a else 0 for m, a in zip(new, live)]
        before, had = list(gen.lens), gen.evictions
        gen.begin_turn(new)
        assert (gen.evictions > had) == any(n + m > capacity for n, m in zip(before, new))
        if gen.evictions > had:
            for l in range(L):
                kept = gen.kept[l].cpu().numpy()
                for b, n in enumerate(before):
                    if n < 0:
                        continue
                    chosen = np.zeros((Hk, n))
                    for h in range(Hk):
                        chosen[h, kept[b, h, :min(n, budget)]] = 1.0       # (what is kept is tested elsewhere)
                    state, rows = bo.evict(refs[l], b, chosen, budget, sinks, recent, bf16)
                    for h in range(Hk):
                        refs[l].blocks[b][h], refs[l].tail[b][h] = state[h]
                    scores[l][b] = np.stack([scores[l][b][h][rows[h]] for h in range(Hk)])
        T = sum(new)
        positions = rng.integers(0, 5000, (3, T)).astype(np.int32)
        table = torch.zeros((T, pairs, 2), device=DEV)
        st3.st3_rotary_table(torch.from_numpy(positions).to(DEV), freq_dev, axis, table)
        turned, cs = st3.rotary(table, layout), table.cpu().numpy()
        assert np.abs(cs - bo.rotary_table(positions, inv_freq, axis)).max() < 2.0 ** -23
        for l in range(L):
            qkv = rand_values(rng, (T, H + 2 * Hk, d), "bf16", 1.2)
            dev = torch.from_numpy(qkv).to(DEV).bfloat16()
            out = to_np64(gen.extend_layer(l, dev[:, :H], dev[:, H:H + Hk], dev[:, H + Hk:], turned if turn != 2 else None))
            q, k = ((bf16(bo.rotate(x, cs, adjacent)) if turn != 2 else x.astype(np.float64)) for x in (qkv[:, :H], qkv[:, H:H + Hk]))
            v, start = qkv[:, H + Hk:].astype(np.float64), 0
            worst = max(worst, float(np.abs(q).max() * np.abs(k).max(initial=4.0)) * d * scale * 1.5)
            for b, m in enumerate(new):
                if not m:
                    continue
                at = slice(start, start + m)
                want, weights, spread = bo.extend(refs[l], b, q[at], k[at], v[at], scale, W)
                close(out[at], want, spread, fp32_slack(worst, d, capacity), 1)
                n = scores[l][b].shape[1]
                weights[:, :n] += scores[l][b]
                scores[l][b] = weights
                start += m
        gen.finish_turn()
        for step in range(3):
            gen.begin_step()
            for l in range(L):
                qkv = rand_values(rng, (B, H + 2 * Hk, d), "bf16", 1.2)
                dev = torch.from_numpy(qkv).to(DEV).bfloat16()
                gen.decode_layer(l, dev[:, :H], dev[:, H:H + Hk], dev[:, H + Hk:])
                for b in range(B):
                    if gen.lens[b] >= 0:
                        x = qkv[b].astype(np.float64)
                        _, weights = bo.decode(refs[l], b, x[:H], x[H:H + Hk], x[H + Hk:], scale)
                        scores[l][b] = np.pad(scores[l][b], ((0, 0), (0, 1))) + weights
            gen.finish_step()
        for l in range(L):
            check_cache(gen, l, refs[l])
            for b, n in enumerate(gen.lens):
                if n > 0:
                    got, s = to_np64(gen.score[l, b, :, :n]), scores[l][b]
                    assert np.all(np.abs(got - s) <= 2 * fp32_slack(worst, d, capacity) * s + 40 * 2.0 ** -24 * s + 1e-30)
    assert gen.evictions > 0


def test_a_prompt_in_pieces_is_the_prompt_at_once():
    """Chunked prefill: the same cache, bit for bit, and outputs that differ by what the cache's codes differ from their rows."""
    rng = np.random.default_rng(3)
    H, Hk, d, n = 8, 2, 128, 300
    x = torch.from_numpy(rand_values(rng, (n, H + 2 * Hk, d), "bf16", 1.0)).to(DEV).bfloat16()
    whole, pieces = (BlockGeneration(1, H, Hk, d, 1, 512, 256) for _ in range(2))
    whole.begin([n])
    want = whole.prefill_layer(0, x[:, :H], x[:, H:H + Hk], x[:, H + Hk:])
    pieces.begin([0])
    outs, at = [], 0
    for m in (100, 1, 63, 128, 8):
        pieces.begin_turn([m])
        y = x[at:at + m]
        outs.append(pieces.extend_layer(0, y[:, :H], y[:, H:H + Hk], y[:, H + Hk:]))
        pieces.finish_turn()
        at += m
    torch.cuda.synchronize()
    blocks = n // 64
    a, b = whole.table(0)[0, :blocks].long(), pieces.table(0)[0, :blocks].long()
    assert torch.equal(whole.k_codes[a], pieces.k_codes[b]) and torch.equal(whole.v_codes[a], pieces.v_codes[b])
    assert torch.equal(whole.k_scale[a], pieces.k_scale[b]) and torch.equal(whole.v_scale[a], pieces.v_scale[b])
    assert all(torch.equal(s[0, :, :n % 64] if i == 0 else s[0, ..., :n % 64], t[0, :, :n % 64] if i == 0 else t[0, ..., :n % 64])
               for i, (s, t) in enumerate(zip(whole.tails(0), pieces.tails(0))))
    # K is off by half a code at most (1/254 of a block's largest): a logit by that times the sum of |q|, V by its own half code
    kmax, vmax, qsum = float(x[:, H:H + Hk].abs().max()), float(x[:, H + Hk:].abs().max()), float(x[:, :H].float().abs().sum(-1).max())
    off = kmax / 254 * qsum / np.sqrt(d)
    bound = (np.expm1(2 * off) + 2.0 ** -8) * vmax + vmax / 254 + 2 * 2.0 ** -8 * vmax
    assert float((torch.cat(outs).float() - want.float()).abs().max()) <= bound


def test_turns_on_another_stream_give_the_same():
    rng = np.random.default_rng(5)
    L, H, Hk, d, lens = 3, 8, 2, 128, [150, 64, 20]
    prompt = torch.from_numpy(rand_values(rng, (L, sum(lens), H + 2 * Hk, d), "bf16", 1.5)).to(DEV).bfloat16()
    turns = [torch.from_numpy(rand_values(rng, (L, T, H + 2 * Hk, d), "bf16", 1.5)).to(DEV).bfloat16() for T in (60, 9)]
    positions = [torch.arange(T, dtype=torch.int32, device=DEV) + 200 for T in (60, 9)]
    inv_freq = torch.from_numpy((10000.0 ** (-np.arange(64) / 64)).astype(np.float32)).to(DEV)
    torch.cuda.synchronize()

    def go():
        gen = BlockGeneration(L, H, Hk, d, 3, 192, 90, 4, 16)
        gen.begin(lens)
        outs = [gen.prefill_layer(l, prompt[l, :, :H], prompt[l, :, H:H + Hk], prompt[l, :, H + Hk:]) for l in range(L)]
        for x, p, new in zip(turns, positions, ([50, 3, 7], [3, 3, 3])):
            gen.begin_turn(new)
            table = torch.empty((len(p), 64, 2), device=DEV)
            st3.st3_rotary_table(p, inv_freq, None, table)
            outs += [gen.extend_layer(l, x[l, :, :H], x[l, :, H:H + Hk], x[l, :, H + Hk:], st3.rotary(table)) for l in range(L)]
            gen.finish_turn()
        torch.cuda.current_stream().synchronize()
        assert gen.evictions == 1 and gen.lens == [143, 70, 30] and gen.len.tolist() == gen.lens
        return outs

    first = go()
    with torch.cuda.stream(torch.cuda.Stream()):
        second = go()
    assert all(torch.equal(a, b) for a, b in zip(first, second))
