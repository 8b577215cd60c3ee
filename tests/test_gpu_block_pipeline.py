"""BlockGeneration: prompts, decode steps and evictions in their order, against the oracle's cache row by row."""
import numpy as np
import pytest
import torch

from block_util import bf16, code_values, fp32_slack
from gpu_util import DEV, rand_values, to_np64
from oracle import block_oracle as bo
from paper_2412_20105_amd import binding as st3
from paper_2412_20105_amd.block_pipeline import BlockGeneration

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8
CODES = {"int8": st3.ST3_BLOCK_INT8, "e4m3": st3.ST3_BLOCK_E4M3}


def close(got, want, spread, slack, halves):
    bound = halves * HALF * spread + HALF * np.abs(want) + 2 * slack * spread + 1e-30
    assert np.all(np.abs(got - want) <= bound), float(np.max(np.abs(got - want) / bound))


def check_cache(gen, l, caches):
    """Codes, scales and tails of layer l, bit for bit."""
    kc, vc = code_values(gen.k_codes), code_values(gen.v_codes)
    ks, vs, table = to_np64(gen.k_scale), to_np64(gen.v_scale), gen.table(l).cpu().numpy()
    kt, vt = (to_np64(x) for x in gen.tails(l))
    for b, n in enumerate(gen.lens):
        if n < 0:
            continue
        assert caches.length(b) == n
        for h in range(gen.Hk):
            for j, ((k, s), (v, z)) in enumerate(caches.blocks[b][h]):
                page = table[b, j]
                assert ks[page, h] == s and vs[page, h] == z, (b, h, j)
                np.testing.assert_array_equal(kc[page, h], k)
                np.testing.assert_array_equal(vc[page, h].T, v)
            k, v = caches.tail[b][h]
            np.testing.assert_array_equal(kt[b, h, :len(k)], k)
            np.testing.assert_array_equal(vt[b, h, :, :len(v)].T, v)


@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("lens,H,Hk,d,capacity,budget", [([70, 3, 129, 0], 4, 2, 64, 131, 70), ([100, -1, 60], 6, 1, 128, 104, 64),
                                                         ([1], 8, 8, 64, 4, 2)])
def test_prompts_steps_and_evictions(lens, H, Hk, d, capacity, budget, code):
    rng = np.random.default_rng(sum(lens) + d)
    L, B, G, W, sinks, recent = 2, len(lens), H // Hk, 5, 1, 1
    gen = BlockGeneration(L, H, Hk, d, B, capacity, budget, sinks, recent, W, CODES[code])
    scale = 1.0 / np.sqrt(d)
    for answer in range(2):         # the second one over what the first left
        gen.begin(lens)
        T = sum(max(n, 0) for n in lens)
        refs = [bo.BlockCache(B, Hk, d, code) for _ in range(L)]
        scores = [[np.zeros((Hk, 0)) for _ in range(B)] for _ in range(L)]
        worst = 0.0
        for l in range(L):
            qkv = rand_values(rng, (T, H + 2 * Hk, d), "bf16", 1.2)
            dev = torch.from_numpy(qkv).to(DEV).bfloat16()
            q, k, v = (np.asarray(x, np.float64) for x in (qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]))
            out = to_np64(gen.prefill_layer(l, dev[:, :H], dev[:, H:H + Hk], dev[:, H + Hk:]))
            want, first = bo.packed_attention(q, k, v, [max(n, 0) for n in lens], scale, W)
            spread = bo.packed_attention(q, k, np.abs(v), [max(n, 0) for n in lens], scale, 0)[0]
            # the largest sum of magnitudes of a logit that any row can have
            worst = max(worst, float(np.abs(q).max() * np.abs(k).max()) * d * scale)
            close(out, want, spread, fp32_slack(worst, d, capacity), 1)
            start = 0
            for b, n in enumerate(lens):
                for h in range(Hk):
                    refs[l].append(b, h, k[start:start + max(n, 0), h], v[start:start + max(n, 0), h])
                scores[l][b] = first[b]
                start += max(n, 0)
            check_cache(gen, l, refs[l])
        for step in range(9):
            if gen.longest >= capacity:
                before = list(gen.lens)
                gen.begin_step()
                assert gen.lens == [min(n, budget) for n in before]
                for l in range(L):
                    kept, slack = gen.kept[l].cpu().numpy(), 2 * fp32_slack(worst, d, capacity)
                    for b, n in enumerate(before):
                        if n < 0:
                            continue
                        m, chosen = min(n, budget), np.zeros((Hk, n))
                        for h in range(Hk):
                            rows, s = kept[b, h, :m], scores[l][b][h]
                            assert np.all(np.diff(rows) > 0) and set(range(min(sinks, m))) <= set(rows) and (m == 0 or n - 1 in rows)
                            chosen[h, rows] = 1.0
                            left = np.setdiff1d(np.arange(n), rows)
                            between = [r for r in rows if sinks <= r < n - recent]
                            if len(left) and between:       # no row left behind has a weight above that of one that was kept
                                assert s[left].max() <= s[between].min() * (1 + slack) + slack * s[left].max()
                        state, rows = bo.evict(refs[l], b, chosen, budget, sinks, recent, bf16)
                        for h in range(Hk):
                            refs[l].blocks[b][h], refs[l].tail[b][h] = state[h]
                        scores[l][b] = np.stack([scores[l][b][h][rows[h]] for h in range(Hk)])
                    check_cache(gen, l, refs[l])
            else:
                gen.begin_step()
            if step == 6 and B > 2:
                gen.retire(2)
            for l in range(L):
                qkv = rand_values(rng, (B, H + 2 * Hk, d), "bf16", 1.2)
                dev = torch.from_numpy(qkv).to(DEV).bfloat16()
                out = to_np64(gen.decode_layer(l, dev[:, :H], dev[:, H:H + Hk], dev[:, H + Hk:]))
                for b in range(B):
                    if gen.lens[b] < 0:
                        assert not out[b].any()
                        continue
                    q, k, v = (np.asarray(x, np.float64) for x in (qkv[b, :H], qkv[b, H:H + Hk], qkv[b, H + Hk:]))
                    held = [refs[l].values(b, h) for h in range(Hk)]
                    spread = np.zeros((H, d))
                    for h in range(H):
                        kk = np.concatenate([held[h // G][0], k[h // G][None]])
                        vv = np.concatenate([held[h // G][1], v[h // G][None]])
                        worst = max(worst, float((np.abs(q[h]) @ np.abs(kk).T).max()) * scale)
                        spread[h] = bo.softmax_rows(q[h] @ kk.T * scale) @ np.abs(vv)
                    want, weights = bo.decode(refs[l], b, q, k, v, scale)
                    # (a weight is two bf16 terms: off by the second one's half step)
                    close(out[b], want, spread, fp32_slack(worst, d, capacity) + 2.0 ** -16, 0)
                    scores[l][b] = np.pad(scores[l][b], ((0, 0), (0, 1))) + weights
            gen.finish_step()
            for l in range(L):
                check_cache(gen, l, refs[l])
                for b, n in enumerate(gen.lens):
                    if n > 0:
                        got, s = to_np64(gen.score[l, b, :, :n]), scores[l][b]
                        assert np.all(np.abs(got - s) <= 2 * fp32_slack(worst, d, capacity) * s + 20 * 2.0 ** -24 * s + 1e-30)
        assert gen.evictions > 0
    assert gen.kv_bytes() > 0


def test_a_batch_on_another_stream_gives_the_same():
    rng = np.random.default_rng(5)
    L, H, Hk, d, lens = 3, 8, 2, 128, [150, 64, 20]
    prompt = torch.from_numpy(rand_values(rng, (L, sum(lens), H + 2 * Hk, d), "bf16", 1.5)).to(DEV).bfloat16()
    steps = torch.from_numpy(rand_values(rng, (12, L, 3, H + 2 * Hk, d), "bf16", 1.5)).to(DEV).bfloat16()
    torch.cuda.synchronize()

    def go():
        gen = BlockGeneration(L, H, Hk, d, 3, 160, 90, 4, 16)
        gen.begin(lens)
        outs = [gen.prefill_layer(l, prompt[l, :, :H], prompt[l, :, H:H + Hk], prompt[l, :, H + Hk:]) for l in range(L)]
        for x in steps:
            gen.begin_step()
            outs += [gen.decode_layer(l, x[l, :, :H], x[l, :, H:H + Hk], x[l, :, H + Hk:]).clone() for l in range(L)]
            gen.finish_step()
        torch.cuda.current_stream().synchronize()
        assert gen.evictions == 1 and gen.lens == [92, 76, 32] and gen.len.tolist() == gen.lens
        return outs

    first = go()
    with torch.cuda.stream(torch.cuda.Stream()):
        second = go()
    assert all(torch.equal(a, b) for a, b in zip(first, second))
