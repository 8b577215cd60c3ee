"""The next turn of a dialogue over an 8-bit cache: what is measured.

A sequence whose cache is filled gets several new tokens at once: the next question, a piece of a long prompt, tokens that were drafted and
are to be checked.  Four calls work together.  The tokens' positions, one axis for text or three (time, height, width) for images and video,
become cosines and sines, once a step for all layers (`table`); queries are rotated by them (`rotate`); keys, rotated on the way, and values are
appended to the cache of 8-bit blocks (`append`); and the new tokens attend to everything before them, themselves included (`attend`), with the
weight that each cached token receives added up.

Layouts.  Packed rows: q [T, H, d], k and v [T, Hk, d]; sequence b owns rows cu[b] .. cu[b + 1].  Table: float32 [T, pairs, 2].  Cache: pages
`k_codes` [pages, Hk, 64, d] and `v_codes` [pages, Hk, d, 64] (values of a column side by side), `k_scale`, `v_scale` [pages, Hk]; the rows of a
sequence that do not fill a block yet stay in 16 bits in `k_tail` [B, Hk, 64, d] and `v_tail` [B, Hk, d, 64]; `table` [B, blocks] names the page of
each block.  `len` says the rows in front of the new ones.  Scores: [B, Hk, capacity].

Sizes are those of this repository's workloads (32 and 40 heads of 128, small float32 models of 64, prompts of 35 to 3136 tokens) with 1 to 40 key
heads, and generic long contexts.  Values are what those workloads draw: N(0, sigma^2), sigma = 0.02 sqrt(heads * dim).
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
BLOCK = 64


# ---------------------------------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------------------------------
def _table(tokens, pairs=64, axes=1, alternate=False, base=10000.0, far=0, **more):
    return {"op": "table", "tokens": tokens, "pairs": pairs, "axes": axes, "alternate": alternate, "base": base, "far": far, **more}


def _rotate(tokens, heads, dim=128, pairs=64, dtype="bf16", adjacent=False, inverse=False, in_place=True, **more):
    return {"op": "rotate", "tokens": tokens, "heads": heads, "dim": dim, "pairs": pairs, "dtype": dtype, "adjacent": adjacent, "inverse": inverse,
            "in_place": in_place, **more}


def _cache(op, batch, old_lo, old_hi, new_lo, new_hi, heads=32, kv_heads=8, dim=128, code="int8", lens_seed=1, **more):
    return {"op": op, "batch": batch, "old_lo": old_lo, "old_hi": old_hi, "new_lo": new_lo, "new_hi": new_hi, "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "code": code, "lens_seed": lens_seed, **more}


def listed():
    return [
        # one decode step of eight users: all latency
        _table(8, name="table_step"),
        # a batch of tiled images among text: three axes that alternate over the columns, positions behind a long history
        _table(50176, axes=3, alternate=True, base=1000000.0, far=120000, name="table_images"),
        # small float32 models that checks are run with: the gradient of rows half of whose columns turn
        _rotate(320, 12, dim=64, pairs=16, dtype="f32", adjacent=True, inverse=True, in_place=False, name="rotate_back_f32"),
        # queries and keys of a batch of prompts, in place in the projection's output
        _rotate(16000, 40, name="rotate_prompts"),
        # eight users, one token each
        _cache("append", 8, 611, 1251, 1, 1, pairs=64, adjacent=False, name="append_step"),
        # sixteen users ask their next question
        _cache("append", 16, 611, 3136, 20, 300, code="e4m3", pairs=64, adjacent=False, name="append_turn"),
        # two long documents are read on, a piece at a time; keys come rotated already
        _cache("append", 2, 20000, 70000, 2000, 4100, pairs=0, adjacent=False, name="append_piece"),
        # one user: five drafted tokens are checked
        _cache("attend", 1, 739, 739, 5, 5, window=5, name="attend_draft"),
        # a serving batch: four drafted tokens each, the weights not wanted
        _cache("attend", 32, 611, 3136, 4, 4, code="e4m3", window=0, name="attend_drafts"),
        # sixteen users ask their next question
        _cache("attend", 16, 611, 3136, 20, 300, code="e4m3", window=32, name="attend_turn"),
        # a piece of a long document
        _cache("attend", 1, 30000, 30000, 2048, 2048, window=64, name="attend_piece"),
        # a short question about two long documents
        _cache("attend", 2, 70000, 131072, 9, 33, window=16, name="attend_long"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["table", "rotate", "rotate", "append", "append", "append", "attend", "attend", "attend", "attend", "attend"])
    if op == "table":
        return _table(_log(rng, 1, 50000), rng.choice([64, 64, 32, 16, 48, 8]), rng.choice([1, 1, 2, 3, 3, 4]), rng.random() < 0.5,
                      rng.choice([10000.0, 500000.0, 1000000.0]), rng.choice([0, 0, 5000, 1000000]))
    heads, kv_heads = rng.choice([(32, 8), (32, 8), (32, 32), (40, 40), (40, 10), (40, 8), (28, 4), (14, 2), (24, 8), (16, 1), (20, 5)])
    dim = rng.choice([128, 128, 128, 64])
    pairs = rng.choice([dim // 2, dim // 2, dim // 4, 24, 8])
    adjacent = rng.random() < 0.4
    if op == "rotate":
        return _rotate(_log(rng, 1, 16000), heads + rng.choice([0, kv_heads]), dim, pairs, rng.choice(["bf16", "bf16", "f32"]), adjacent, rng.random() < 0.3,
                       rng.random() < 0.5)
    seed, code = rng.randrange(1 << 30), rng.choice(["int8", "e4m3"])
    if op == "append":
        new = _log(rng, 1, 4100)
        batch = _log(rng, 1, max(1.0, min(64.0, 16000 / new)))
        old = _log(rng, 1, max(2.0, min(70000.0, 1.2e6 / (batch * kv_heads))))
        return _cache(op, batch, rng.randint(0, old), old, max(1, int(new * rng.uniform(0.05, 1.0))), new, heads, kv_heads, dim, code, seed,
                      pairs=rng.choice([0, pairs, pairs]), adjacent=adjacent)
    new = _log(rng, 1, 2048)
    # no more logits than the piece of a long document has, nor a larger cache than the long documents'
    old = _log(rng, 1, max(2.0, min(130000.0, 6.0e7 * 32 / (new * heads), 2.0e6 / kv_heads)))
    most = min(64.0, 6.0e7 * 32 / (new * (old + new) * heads), 2.0e6 / ((old + new) * kv_heads))
    return _cache(op, _log(rng, 1, max(1.0, most)), rng.randint(0, old), old, max(1, int(new * rng.uniform(0.1, 1.0))), new, heads, kv_heads, dim, code, seed,
                  window=rng.choice([0, 1, 8, 32, 64]))


def _lens(c, what):
    """Lengths of the batch, spread over their logarithm, the longest among them."""
    r, lo, hi = random.Random(c["lens_seed"] * 31 + c["batch"] + (7 if what == "new" else 0)), c[what + "_lo"], c[what + "_hi"]
    lens = [_log(r, lo + 1, hi + 1) - 1 for _ in range(c["batch"])]
    lens[r.randrange(c["batch"])] = hi
    return lens


def work(c):
    if c["op"] == "table":
        return {"bytes": 4 * c["axes"] * c["tokens"] + 4 * c["pairs"] + 8 * c["tokens"] * c["pairs"], "flops": 20 * c["tokens"] * c["pairs"]}
    if c["op"] == "rotate":
        T, e = c["tokens"], 4 if c["dtype"] == "f32" else 2
        cols = 2 * c["pairs"] if c["in_place"] else c["dim"]
        return {"bytes": 2 * e * T * c["heads"] * cols + 8 * T * c["pairs"], "flops": 6 * T * c["heads"] * c["pairs"]}
    H, Hk, d, B, old, new = c["heads"], c["kv_heads"], c["dim"], c["batch"], _lens(c, "old"), _lens(c, "new")
    both, M = [n + m for n, m in zip(old, new)], sum(new)
    if c["op"] == "append":
        filled = sum(s // BLOCK - n // BLOCK for s, n in zip(both, old))
        before = sum(n % BLOCK for s, n in zip(both, old) if s // BLOCK > n // BLOCK)
        behind = sum(s % BLOCK if s // BLOCK > n // BLOCK else m for s, n, m in zip(both, old, new))
        return {"bytes": 2 * Hk * (2 * d * (M + before + behind) + filled * (BLOCK * d + 4)) + 8 * c["pairs"] * M + 4 * (filled + 2 * B + 1),
                "flops": 4 * Hk * d * M + 6 * Hk * c["pairs"] * M}
    W = c["window"]
    pairs = sum(n * m + m * (m + 1) // 2 for n, m in zip(old, new))
    seen = sum(sum(s - i for i in range(min(W, m))) for s, m in zip(both, new))
    b = 2 * Hk * sum(s // BLOCK * (BLOCK * d + 4) + 2 * d * (s % BLOCK) for s in both) + 4 * d * H * M + 4 * sum(s // BLOCK + 2 for s in both)
    return {"bytes": b + (4 * Hk * sum(n + s for n, s in zip(old, both)) if W else 0), "flops": 4 * d * H * pairs + 2 * d * H * seen}


# ---------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed) * 7919 + 31)


def _randn(g, shape, sigma, dtype):
    return (torch.randn(shape, generator=g, device=DEV) * sigma).to(dtype)


def _codes(g, shape, code):
    """Codes as a block of normal values has them: the largest of a block's values, about four sigma, takes the largest code."""
    x = torch.randn(shape, generator=g, device=DEV)
    if code == "int8":
        return (x * 31).round_().clamp_(-127, 127).to(torch.int8)
    return (x * 112).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _angles(c, g):
    """Cosines and sines of tokens behind one another, as a program has them in hand."""
    T, pairs = sum(_lens(c, "new")), c["pairs"]
    start = int(torch.randint(0, 100000, (1,), generator=g, device=DEV))
    freq = (10000.0 ** (-torch.arange(pairs, device=DEV, dtype=torch.float64) / pairs))
    angle = (start + torch.arange(T, device=DEV, dtype=torch.float64))[:, None] * freq
    return torch.stack([angle.cos(), angle.sin()], -1).float()


def prepare(c, seed):
    g = _gen(seed)
    s = {"case": dict(c)}
    if c["op"] == "table":
        T, A = c["tokens"], c["axes"]
        i = torch.arange(T, device=DEV)
        start = c["far"] + torch.randint(0, 1000, (1,), generator=g, device=DEV)
        # images of 24 x 24 patches: an axis for the image, its rows, its columns (and one for the tile it belongs to)
        grid = torch.stack([i // 576, i % 576 // 24, i % 24, i // 2880])[:A] if A > 1 else i[None]
        s["positions"] = (start + grid).to(torch.int32).contiguous()
        s["inv_freq"] = (c["base"] ** (-torch.arange(c["pairs"], device=DEV, dtype=torch.float64) / c["pairs"])).float()
        s["axis"] = [p % A if c["alternate"] else p * A // c["pairs"] for p in range(c["pairs"])]
        s["axis_of"] = torch.tensor(s["axis"], device=DEV)
        s["out"] = torch.zeros((T, c["pairs"], 2), device=DEV)
        return s
    if c["op"] == "rotate":
        T, H, d = c["tokens"], c["heads"], c["dim"]
        dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        s["x"] = _randn(g, (T, H + 8, d), 0.02 * math.sqrt(H * d), dt)[:, :H]               # rows of a projection that gives values too
        s["out"] = torch.zeros((T, H, d), dtype=dt, device=DEV)
        angle = torch.rand((T, c["pairs"]), generator=g, device=DEV, dtype=torch.float64) * (2 * math.pi)
        s["angles"] = torch.stack([angle.cos(), angle.sin()], -1).float()
        return s
    H, Hk, d, B, old, new = c["heads"], c["kv_heads"], c["dim"], c["batch"], _lens(c, "old"), _lens(c, "new")
    sigma, M = 0.02 * math.sqrt(H * d), sum(new)
    # a layer's cache as a serving program holds it: pages in no order, a few of them free
    both = [n + m for n, m in zip(old, new)]
    blocks, want = max(both) // BLOCK + 1, sum(n // BLOCK + 1 for n in both)
    pages = want + 3
    names = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    rows = torch.tensor([n // BLOCK + 1 for n in both], device=DEV)
    at = torch.arange(blocks, device=DEV)
    place = (rows.cumsum(0) - rows)[:, None] + at
    s["table"] = torch.where(at < rows[:, None], names[place.clamp_(max=pages - 1)], torch.zeros_like(names[:1])).contiguous()
    s["free"] = names[want:]
    s["k_codes"], s["v_codes"] = _codes(g, (pages, Hk, BLOCK, d), c["code"]), _codes(g, (pages, Hk, d, BLOCK), c["code"])
    for name in ("k_scale", "v_scale"):
        s[name] = (0.8 + 0.4 * torch.rand((pages, Hk), generator=g, device=DEV)) * (sigma / (31 if c["code"] == "int8" else 112))
    s["k_tail"] = _randn(g, (B, Hk, BLOCK, d), sigma, torch.bfloat16)
    s["v_tail"] = _randn(g, (B, Hk, d, BLOCK), sigma, torch.bfloat16)
    s["len"] = torch.tensor(old, dtype=torch.int32, device=DEV)
    s["cu"] = torch.tensor([0] + new, device=DEV).cumsum(0).to(torch.int32)
    s["new_top"], s["top"], s["scale"] = max(new), max(both), 1.0 / math.sqrt(d)
    # one matrix product gives a token's queries, keys and values: rows of one tensor
    qkv = _randn(g, (M, H + 2 * Hk, d), sigma, torch.bfloat16)
    if c["op"] == "append":
        s["k"], s["v"] = qkv[:, H:H + Hk], qkv[:, H + Hk:]
        s["angles"] = _angles(c, g) if c["pairs"] else None
        return s
    s["q"] = qkv[:, :H]
    s["out"] = torch.zeros((M, H, d), dtype=torch.bfloat16, device=DEV)
    s["score"] = torch.randn((B, Hk, s["top"] + BLOCK), generator=g, device=DEV).mul_(1.5).exp_() if c["window"] else None
    return s


# ---------------------------------------------------------------------------------------------------
# the calls
# ---------------------------------------------------------------------------------------------------
def run(s):
    op = s["case"]["op"]
    if own:
        {"table": _own_table, "rotate": _own_rotate, "append": _own_append, "attend": _own_attend}[op](s)
    else:
        {"table": _plain_table, "rotate": _plain_rotate, "append": _plain_append, "attend": _plain_attend}[op](s)
    if op == "append":
        kind = torch.int8 if s["case"]["code"] == "int8" else torch.float8_e4m3fn
        return {"k_codes": s["k_codes"].view(kind), "v_codes": s["v_codes"].view(kind), "k_scale": s["k_scale"], "v_scale": s["v_scale"],
                "k_tail": s["k_tail"], "v_tail": s["v_tail"]}
    if op == "attend":
        return {"out": s["out"], **({} if s["score"] is None else {"score": s["score"]})}
    return {"out": s["x"] if op == "rotate" and s["case"]["in_place"] else s["out"]}


# -- through the framework: shape, descriptions and workspace are made once, as a program keeps them --------------------------------
def _handle(s):
    from paper_2412_20105_amd import binding as st3
    c = s["case"]
    h = s["handle"] = {"st3": st3}
    layout = st3.ST3_ROTARY_ADJACENT if c.get("adjacent") else st3.ST3_ROTARY_HALVES
    h["rotary"] = None if s.get("angles") is None else st3.rotary(s["angles"], layout)
    if c["op"] in ("append", "attend"):
        h["shape"] = st3.gqa_shape(c["batch"], c["heads"], c["kv_heads"], c["dim"])
        h["cache"] = st3.block_cache(s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"], s["k_tail"], s["v_tail"], s["table"], s["len"])
    if c["op"] == "attend":
        need = st3.st3_block_attend_workspace_bytes(h["shape"], s["q"].shape[0], s["new_top"], s["top"])
        h["ws"] = torch.empty(need, dtype=torch.uint8, device=DEV)
    return h


def _own_table(s):
    h = s.get("handle") or _handle(s)
    h["st3"].st3_rotary_table(s["positions"], s["inv_freq"], s["axis"], s["out"])


def _own_rotate(s):
    h = s.get("handle") or _handle(s)
    h["st3"].st3_rotate_rows(s["x"], s["x"] if s["case"]["in_place"] else s["out"], h["rotary"], s["case"]["inverse"])


def _own_append(s):
    h = s.get("handle") or _handle(s)
    h["st3"].st3_block_append(h["shape"], s["k"], s["v"], s["cu"], s["new_top"], h["cache"], s["top"], h["rotary"])


def _own_attend(s):
    h = s.get("handle") or _handle(s)
    h["st3"].st3_block_attend(h["shape"], s["q"], s["cu"], s["new_top"], h["cache"], s["top"], s["out"], s["case"]["window"], s["score"], h["ws"])


# -- plain forms --------------------------------------------------------------------------------------------------------------------
def _plain_table(s):
    angle = s["positions"].double()[s["axis_of"]].t() * s["inv_freq"].double()
    s["out"].copy_(torch.stack([angle.cos(), angle.sin()], -1))


def _turned(x, angles, adjacent, inverse=False):
    """Rows x [T, H, d] in 32 bits, rotated."""
    pairs = angles.shape[1]
    cos, sin = angles[:, None, :, 0], angles[:, None, :, 1]
    if inverse:
        sin = -sin
    y = x.clone()
    a, b = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if adjacent else (slice(0, pairs), slice(pairs, 2 * pairs))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y


def _plain_rotate(s):
    c = s["case"]
    (s["x"] if c["in_place"] else s["out"]).copy_(_turned(s["x"].float(), s["angles"], c["adjacent"], c["inverse"]))


def _value(s, name, pages):
    """Blocks of the cache in 32 bits: [..., Hk, 64, d] of `k`, [..., Hk, d, 64] of `v`."""
    x = s[name + "_codes"][pages]
    x = x.float() if s["case"]["code"] == "int8" else x.view(torch.float8_e4m3fn).float()
    return x * s[name + "_scale"][pages][..., None, None]


def _coded(s, x):
    """(codes, scale) of blocks [..., 64 * d values]: the largest magnitude takes the largest code."""
    top = 127.0 if s["case"]["code"] == "int8" else 448.0
    scale = x.abs().amax((-1, -2)) * torch.tensor(1.0 / top, device=DEV)
    y = torch.where(scale[..., None, None] > 0, x / scale[..., None, None], torch.zeros_like(x)).clamp_(-top, top)
    return (y.round_().to(torch.int8) if top == 127.0 else y.to(torch.float8_e4m3fn).view(torch.uint8)), scale


def _plain_append(s):
    c, cu, n = s["case"], s["cu"].long(), s["len"].long()
    B, M, blocks = c["batch"], s["k"].shape[0], (s["new_top"] + BLOCK - 1) // BLOCK + 1
    m, b = cu[1:] - cu[:-1], torch.arange(c["batch"], device=DEV)
    first, total = n // BLOCK, n + m
    # rows of the blocks that the new rows lie in, from the first of them on: of the tail, new, or none yet
    at = (first * BLOCK)[:, None] + torch.arange(blocks * BLOCK, device=DEV)
    fresh = ((at >= n[:, None]) & (at < total[:, None])).view(B, blocks, 1, BLOCK, 1)
    row = (cu[:-1, None] + at - n[:, None]).clamp_(0, M - 1)
    whole = ((at[:, BLOCK - 1::BLOCK] < total[:, None])).view(-1)
    where = (first[:, None] + torch.arange(blocks, device=DEV)).clamp_(max=s["table"].shape[1] - 1)
    # a block that is not whole writes to a page that no sequence has what it holds
    pages = torch.where(whole, s["table"].gather(1, where).long().view(-1), s["free"][0].long())
    last = total // BLOCK - first
    fill = (torch.arange(BLOCK, device=DEV) < (total % BLOCK)[:, None])[:, None, :, None]
    for name in ("k", "v"):
        x = s[name].float()
        if name == "k" and s["angles"] is not None:
            x = _turned(x, s["angles"], c["adjacent"]).to(torch.bfloat16).float()
        tail = s[name + "_tail"] if name == "k" else s["v_tail"].transpose(-1, -2)
        x = torch.where(fresh, x[row.view(B, blocks, BLOCK)].transpose(2, 3), torch.nn.functional.pad(tail.float()[:, None], (0, 0, 0, 0, 0, 0, 0, blocks - 1)))
        tail.copy_(torch.where(fill, x[b, last], tail.float()))
        codes, scale = _coded(s, (x if name == "k" else x.transpose(-1, -2)).flatten(0, 1))
        s[name + "_codes"][pages] = torch.where(whole[:, None, None, None], codes, s[name + "_codes"][pages])
        s[name + "_scale"][pages] = torch.where(whole[:, None], scale, s[name + "_scale"][pages])


def _plain_attend(s):
    c, cu, n = s["case"], s["cu"].long(), s["len"].long()
    H, Hk, d, B, M, W, m_top = c["heads"], c["kv_heads"], c["dim"], c["batch"], s["q"].shape[0], c["window"], s["new_top"]
    m, b, G = cu[1:] - cu[:-1], torch.arange(c["batch"], device=DEV), H // Hk
    total, blocks = n + m, s["top"] // BLOCK + 1
    N = blocks * BLOCK
    pages, at, i = s["table"].long(), torch.arange(N, device=DEV), torch.arange(m_top, device=DEV)
    dead = (torch.arange(BLOCK, device=DEV) >= (total % BLOCK)[:, None])[:, None, :, None]  # rows of the tail that hold nothing
    k = _value(s, "k", pages)
    k[b, total // BLOCK] = s["k_tail"].float().masked_fill(dead, 0)
    k = k.permute(0, 2, 1, 3, 4).reshape(B, Hk, N, d)
    v = _value(s, "v", pages).transpose(-1, -2)
    v[b, total // BLOCK] = s["v_tail"].float().transpose(-1, -2).masked_fill(dead, 0)
    v = v.permute(0, 2, 1, 3, 4).reshape(B, Hk, N, d)
    row = (cu[:-1, None] + i).clamp_(max=M - 1)                                             # padded to the longest
    q = s["q"].float()[row].permute(0, 2, 1, 3).reshape(B, Hk, G * m_top, d)
    p = torch.matmul(q, k.transpose(-1, -2)).mul_(s["scale"]).view(B, Hk, G, m_top, N)
    p.masked_fill_((at > (n[:, None] + i)[..., None])[:, None, None], -math.inf)
    p.sub_(p.amax(-1, keepdim=True)).exp_()
    part = p.sum(-1)
    p = p.view(B, Hk, G * m_top, N)
    out = torch.matmul(p, v).view(B, Hk, G, m_top, d) / part[..., None]
    t = torch.arange(M, device=DEV)
    of = torch.bucketize(t, cu[1:], right=True)
    s["out"].copy_(out.permute(0, 3, 1, 2, 4).reshape(B, m_top, H, d)[of, t - cu[of]])
    if W:
        seen = (i >= m[:, None] - W) & (i < m[:, None])                                     # the rows whose weights count
        w = (seen[:, None, None, :] / part).reshape(B, Hk, 1, G * m_top)
        got, old = torch.matmul(w, p).view(B, Hk, N), s["score"][:, :, :N]
        here, there = (at < n[:, None])[:, None], ((at >= n[:, None]) & (at < total[:, None]))[:, None]
        got = torch.where(here, old + got, torch.where(there, got, old))
        s["score"][:, :, :N] = torch.where((m > 0)[:, None, None], got, old)


# ---------------------------------------------------------------------------------------------------
# the definition, in 64 bits
# ---------------------------------------------------------------------------------------------------
def exact(c, seed):
    s = prepare(c, seed)
    return {"table": _exact_table, "rotate": _exact_rotate, "append": _exact_append, "attend": _exact_attend}[c["op"]](c, s)


def _exact_table(c, s):
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    for p in range(c["pairs"]):
        z = torch.polar(torch.ones(c["tokens"], dtype=torch.float64, device=DEV), s["positions"][s["axis"][p]].double() * float(s["inv_freq"][p]))
        out[:, p, 0], out[:, p, 1] = z.real, z.imag
    return {"out": out}


def _exact_turned(x, angles, adjacent):
    """x as complex numbers times the angles' own."""
    pairs = angles.shape[1]
    z = torch.view_as_complex(angles.double().contiguous())[:, None]
    lead = x[..., :2 * pairs].double()
    if adjacent:
        y = torch.view_as_real(torch.view_as_complex(lead.reshape(*lead.shape[:-1], pairs, 2).contiguous()) * z).flatten(-2)
    else:
        w = torch.complex(lead[..., :pairs].contiguous(), lead[..., pairs:].contiguous()) * z
        y = torch.cat([w.real, w.imag], -1)
    return torch.cat([y, x[..., 2 * pairs:].double()], -1)


def _exact_rotate(c, s):
    angles = s["angles"] * torch.tensor([1.0, -1.0], device=DEV) if c["inverse"] else s["angles"]
    return {"out": _exact_turned(s["x"], angles, c["adjacent"])}


def _exact_append(c, s):
    kind, top = (torch.int8, 127.0) if c["code"] == "int8" else (torch.float8_e4m3fn, 448.0)
    got = {name: s[name].view(kind).double() for name in ("k_codes", "v_codes")}
    got.update({name: s[name].double() for name in ("k_scale", "v_scale", "k_tail", "v_tail")})
    start, table = 0, s["table"].tolist()
    k = s["k"] if s["angles"] is None else _exact_turned(s["k"], s["angles"], c["adjacent"])
    for b, (n, m) in enumerate(zip(_lens(c, "old"), _lens(c, "new"))):
        for name, new in (("k", k), ("v", s["v"])):
            tail = s[name + "_tail"][b].double()
            tail = tail if name == "k" else tail.transpose(1, 2)
            x = torch.cat([tail[:, :n % BLOCK], new[start:start + m].double().transpose(0, 1)], 1)
            whole = x.shape[1] // BLOCK
            for j in range(whole):
                y, page = x[:, j * BLOCK:(j + 1) * BLOCK], table[b][n // BLOCK + j]
                scale = y.abs().flatten(1).amax(-1) / top
                got[name + "_scale"][page] = scale
                got[name + "_codes"][page] = (y if name == "k" else y.transpose(1, 2)) / scale[:, None, None]
            rest = x[:, whole * BLOCK:]
            if name == "k":
                got["k_tail"][b, :, :rest.shape[1]] = rest
            else:
                got["v_tail"][b, :, :, :rest.shape[1]] = rest.transpose(1, 2)
        start += m
    if s["angles"] is not None:
        got["k_scale"] = None       # a rotated key has 16 bits before it is coded: the scale hangs on how one value was rounded
    return got


def _exact_attend(c, s):
    H, Hk, d, W = c["heads"], c["kv_heads"], c["dim"], c["window"]
    kind, G = torch.int8 if c["code"] == "int8" else torch.float8_e4m3fn, c["heads"] // c["kv_heads"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    score = None if s["score"] is None else s["score"].double()
    start = 0
    for b, (n, m) in enumerate(zip(_lens(c, "old"), _lens(c, "new"))):
        total = n + m
        pages = s["table"][b, :total // BLOCK].long()
        j, i = torch.arange(total, device=DEV), torch.arange(m, device=DEV)[:, None]
        for kh in range(Hk):
            rows = []
            for name in ("k", "v"):
                x = s[name + "_codes"][pages, kh].view(kind).double() * s[name + "_scale"][pages, kh].double()[:, None, None]
                x = x if name == "k" else x.transpose(1, 2)
                tail = s[name + "_tail"][b, kh].double()
                tail = tail if name == "k" else tail.t()
                rows.append(torch.cat([x.reshape(-1, d), tail[:total % BLOCK]]))
            got = torch.zeros(total, dtype=torch.float64, device=DEV)
            for h in range(kh * G, (kh + 1) * G if m else 0):
                a = s["q"][start:start + m, h].double() @ rows[0].t() / math.sqrt(d)
                a = torch.softmax(torch.where(j <= n + i, a, -math.inf), -1)
                out[start:start + m, h] = a @ rows[1]
                got += a[max(0, m - W):].sum(0)
            if score is not None and m:
                score[b, kh, :n] += got[:n]
                score[b, kh, n:total] = got[n:]
        start += m
    return {"out": out, **({} if score is None else {"score": score})}
