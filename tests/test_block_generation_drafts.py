"""Turns that do not stay: drafted tokens are checked, and the sequences are as they were."""
import numpy as np
import pytest
import torch

from paper_2412_20105_amd import binding as st3
from paper_2412_20105_amd.block_pipeline import BlockGeneration


def test_a_turn_that_does_not_stay_adds_no_rows():
    gen = BlockGeneration.__new__(BlockGeneration)          # (no GPU: up to the library's first call)
    gen.B, gen.capacity, gen.budget, gen.device = 3, 256, 128, "cpu"
    gen.lens, gen.shape, gen._turn_ws = [60, -1, 30], st3.gqa_shape(3, 8, 2, 128), torch.empty(0, dtype=torch.uint8)
    gen.len, gen.live = torch.tensor(gen.lens, dtype=torch.int32), torch.tensor([1, 0, 1], dtype=torch.int32)
    gen.begin_turn([8, 0, 5], stays=False)
    assert gen.total == 13 and not gen.counts
    for call in (gen.begin_step, lambda: gen.begin_turn([1, 0, 1])):
        with pytest.raises(ValueError, match="open"):
            call()
    gen.finish_turn()
    assert gen.lens == [60, -1, 30] and gen.len.tolist() == gen.lens
    gen.begin_turn([2, 0, 5])
    assert gen.counts
    gen.finish_turn()
    assert gen.lens == [62, -1, 35] and gen.len.tolist() == gen.lens


@pytest.mark.gpu
@pytest.mark.parametrize("code", ["int8", "e4m3"])
@pytest.mark.parametrize("lens,new", [([60, 30, 128], [8, 5, 3]), ([0, 64, 63], [4, 70, 2]), ([150, -1, 10], [130, 0, 64])])
def test_drafts_leave_nothing_behind(lens, new, code):
    """Outputs are those of a turn that stays; codes, scales, tails, scores and lengths are what they are without it, also where drafts fill blocks; and steps,
    turns and evictions go on the same."""
    from gpu_util import DEV, rand_values
    rng = np.random.default_rng(sum(new))
    L, H, Hk, d, kind = 2, 8, 2, 128, {"int8": st3.ST3_BLOCK_INT8, "e4m3": st3.ST3_BLOCK_E4M3}[code]
    draw = lambda n: [torch.from_numpy(rand_values(rng, (n, H + 2 * Hk, d), "bf16", 1.2)).to(DEV).bfloat16() for _ in range(L)]  # noqa: E731
    split = lambda x: (x[:, :H], x[:, H:H + Hk], x[:, H + Hk:])  # noqa: E731
    prompt, drafts, step = draw(sum(max(n, 0) for n in lens)), draw(sum(new)), draw(3)
    accepted = [m // 3 for m in new]
    pick = torch.tensor([sum(new[:b]) + t for b in range(3) for t in range(accepted[b])], device=DEV)
    table = torch.empty((sum(new), 64, 2), device=DEV)
    st3.st3_rotary_table(torch.arange(sum(new), dtype=torch.int32, device=DEV), torch.rand(64, device=DEV), None, table)
    gens, outs = {}, {}
    for name in ("without", "with", "stays"):
        gen = gens[name] = BlockGeneration(L, H, Hk, d, 3, 384, 90, 2, 8, 4, kind)
        gen.begin(lens)
        for l in range(L):
            gen.prefill_layer(l, *split(prompt[l]))
        if name != "without":
            gen.begin_turn(new, stays=name == "stays")
            outs[name] = [gen.extend_layer(l, *split(drafts[l]), st3.rotary(table)) for l in range(L)]
            gen.finish_turn()
    assert all(torch.equal(a, b) for a, b in zip(outs["with"], outs["stays"]))
    assert gens["stays"].lens == [n + m for n, m in zip(lens, new)]

    def same():
        a, b = gens["without"], gens["with"]
        torch.cuda.synchronize()
        assert a.lens == b.lens and torch.equal(a.len, b.len) and a._of == b._of
        for l in range(L):
            for s, n in enumerate(a.lens):
                blocks, rest = max(n, 0) // 64, max(n, 0) % 64
                pages = a.table(l)[s, :blocks].long()
                for x in ("k_codes", "v_codes", "k_scale", "v_scale"):
                    assert torch.equal(getattr(a, x)[pages], getattr(b, x)[pages]), (x, s)
                (ka, va), (kb, vb) = a.tails(l), b.tails(l)
                assert torch.equal(ka[s, :, :rest], kb[s, :, :rest]) and torch.equal(va[s, ..., :rest], vb[s, ..., :rest]), s
                assert torch.equal(a.score[l, s, :, :max(n, 0)], b.score[l, s, :, :max(n, 0)])

    same()
    results = []
    for gen in (gens["without"], gens["with"]):
        got = []
        gen.begin_step()
        got += [gen.decode_layer(l, *split(step[l])).clone() for l in range(L)]
        gen.finish_step()
        gen.begin_turn(accepted)
        if len(pick):
            got += [gen.extend_layer(l, *split(drafts[l][pick]), st3.rotary(table[pick])) for l in range(L)]
        gen.finish_turn()
        gen.evict()
        results.append(got)
    assert all(torch.equal(x, y) for x, y in zip(*results))
    same()
