"""CPU oracle (float64 NumPy) of the calls for grouped heads: packed prompts, caches of 8-bit blocks, further turns, eviction by accumulated weight.

Written from the definitions in include/st3.h, row by row and head by head, sharing no code with the library.  A cache is
kept as a list of rows for each (sequence, key head): whole blocks hold codes and a scale, the rows behind them plain values.
Whatever a rounding decides (a code, a kept row) is decided in float32, as the format is defined.
"""
from __future__ import annotations

import numpy as np

from oracle.st3_oracle import e4m3_decode, e4m3_quantize

BLOCK = 64


def softmax_rows(logits: np.ndarray) -> np.ndarray:
    e = np.exp(logits - logits.max(axis=-1, keepdims=True))
    return e / e.sum(axis=-1, keepdims=True)


def packed_attention(q, k, v, lens, scale, window=0):
    """q [T,H,d], k, v [T,Hk,d] -> out [T,H,d] and, for each sequence, the weight [Hk, n] that its last `window` rows give."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    H, Hk = q.shape[1], k.shape[1]
    out, scores, start = np.zeros_like(q), [], 0
    for n in lens:
        score = np.zeros((Hk, n))
        for h in range(H):
            kh = h // (H // Hk)
            rows = slice(start, start + n)
            for i in range(n):
                p = softmax_rows(q[start + i, h] @ k[rows, kh][:i + 1].T * scale)
                out[start + i, h] = p @ v[rows, kh][:i + 1]
                if i >= n - window:
                    score[kh, :i + 1] += p
        scores.append(score)
        start += n
    return out, scores


def quantize_block(x: np.ndarray, code: str):
    """Codes (as their values in units of the scale) and scale of one block, x [64, d] float32."""
    x = np.asarray(x, np.float32)
    top = np.float32(127.0 if code == "int8" else 448.0)
    finite = np.where(np.isfinite(x), np.abs(x), np.float32(0))
    scale = np.float32(finite.max()) * (np.float32(1) / top)
    if scale > 0:
        with np.errstate(invalid="ignore", over="ignore"):
            y = x / scale
    else:
        y = np.where(np.isnan(x), x, np.float32(0)) if code == "e4m3" else np.zeros_like(x)
    if code == "int8":
        return np.rint(np.clip(np.where(np.isnan(y), 0, y), -top, top)), scale
    return np.asarray(e4m3_decode(e4m3_quantize(y, np.float32(1))), np.float64).reshape(x.shape), scale


class BlockCache:
    """Rows of every (sequence, key head)."""

    def __init__(self, batch: int, kv_heads: int, dim: int, code: str):
        self.B, self.Hk, self.d, self.code = batch, kv_heads, dim, code
        self.blocks = [[[] for _ in range(kv_heads)] for _ in range(batch)]     # ((K codes, scale), (V codes, scale)) each
        self.tail = [[[np.zeros((0, dim)), np.zeros((0, dim))] for _ in range(kv_heads)] for _ in range(batch)]

    def length(self, b: int) -> int:
        return BLOCK * len(self.blocks[b][0]) + len(self.tail[b][0][0])

    def values(self, b: int, kh: int):
        """K and V [len, d] as the cache stands for them: float32 products in blocks, plain values behind."""
        parts = [[], []]
        for block in self.blocks[b][kh]:
            for w in range(2):
                codes, scale = block[w]
                parts[w].append((codes.astype(np.float32) * scale).astype(np.float64))
        return tuple(np.concatenate(parts[w] + [self.tail[b][kh][w]], axis=0) for w in range(2))

    def append(self, b: int, kh: int, k: np.ndarray, v: np.ndarray):
        """Rows k, v [m, d] behind those that are there; blocks that become whole are coded."""
        t = [np.concatenate([self.tail[b][kh][w], x]) for w, x in enumerate((k, v))]
        while len(t[0]) >= BLOCK:
            self.blocks[b][kh].append(tuple(quantize_block(x[:BLOCK], self.code) for x in t))
            t = [x[BLOCK:] for x in t]
        self.tail[b][kh] = t


def decode(cache: BlockCache, b: int, q, k_new, v_new, scale):
    """One token of sequence b: out [H,d], weights [Hk, len + 1]; the rows are appended.  k_new None: nothing is."""
    H, G = q.shape[0], q.shape[0] // cache.Hk
    n = cache.length(b)
    out, weights = np.zeros((H, cache.d)), np.zeros((cache.Hk, n + (k_new is not None)))
    for kh in range(cache.Hk):
        k, v = cache.values(b, kh)
        if k_new is not None:
            k, v = np.concatenate([k, k_new[kh][None]]), np.concatenate([v, v_new[kh][None]])
            cache.append(b, kh, k_new[kh][None], v_new[kh][None])
        if not len(k):
            continue
        for h in range(kh * G, (kh + 1) * G):
            p = softmax_rows(q[h] @ k.T * scale)
            out[h] = p @ v
            weights[kh] += p
    return out, weights


def kept_rows(score: np.ndarray, keep: int, n_sink: int, n_recent: int):
    """Rows kept of len(score), ascending: (score desc, row asc) between the first and the last ones."""
    n = len(score)
    if n <= keep:
        return np.arange(n)
    mid = range(n_sink, n - n_recent)
    key = [(-np.inf if np.isnan(s) else float(s)) for s in score]
    nan = [bool(np.isnan(s)) for s in score]
    best = sorted(mid, key=lambda i: (nan[i], -key[i], i))[:keep - n_sink - n_recent]
    return np.array(sorted([*range(n_sink), *best, *range(n - n_recent, n)]), dtype=np.int64)


def evict(cache: BlockCache, b: int, score, keep: int, n_sink: int, n_recent: int, round_row) -> "tuple[list, list]":
    """New (blocks, tail) of sequence b and the rows kept, for each key head; round_row: values to the tail's type."""
    state, rows = [], []
    for kh in range(cache.Hk):
        idx = kept_rows(np.asarray(score[kh]), keep, n_sink, n_recent)
        k, v = cache.values(b, kh)
        whole = len(cache.blocks[b][kh])
        blocks = []
        for j in range(len(idx) // BLOCK):
            at = idx[j * BLOCK:(j + 1) * BLOCK]
            first = at[0] // BLOCK
            if at[0] % BLOCK == 0 and at[-1] == at[0] + BLOCK - 1 and first < whole:
                blocks.append(cache.blocks[b][kh][first])
            else:
                blocks.append(tuple(quantize_block(x[at].astype(np.float32), cache.code) for x in (k, v)))
        rest = idx[len(idx) // BLOCK * BLOCK:]
        state.append((blocks, [round_row(k[rest]), round_row(v[rest])]))
        rows.append(idx)
    return state, rows


def rotary_table(positions, inv_freq, axis):
    """[T, pairs, 2] cosines and sines (80-bit arithmetic: a position of 31 bits times a float32 has 55) of positions [axes, T]."""
    angle = np.asarray(positions)[list(axis)].T.astype(np.longdouble) * np.asarray(inv_freq, np.float32).astype(np.longdouble)
    two_pi = 8 * np.arctan(np.longdouble(1))
    angle = angle - np.rint(angle / two_pi) * two_pi
    return np.stack([np.cos(angle), np.sin(angle)], -1).astype(np.float64)


def rotate(x, table, adjacent: bool, inverse: bool = False) -> np.ndarray:
    """Rows x [T, H, d] turned, float32 with every product rounded by itself."""
    x, table = np.asarray(x, np.float32), np.asarray(table, np.float32)
    pairs = table.shape[1]
    c, s = table[:, None, :, 0], table[:, None, :, 1] * np.float32(-1 if inverse else 1)
    lead = slice(0, 2 * pairs, 2) if adjacent else slice(0, pairs)
    rear = slice(1, 2 * pairs, 2) if adjacent else slice(pairs, 2 * pairs)
    y, a, b = x.copy(), x[..., lead], x[..., rear]
    with np.errstate(invalid="ignore", over="ignore"):
        y[..., lead], y[..., rear] = a * c - b * s, b * c + a * s
    return y


def extend(cache: BlockCache, b: int, q, k_new, v_new, scale, window=0):
    """New rows of sequence b (k_new, v_new [m, Hk, d], as the tail holds them): appended, then attended: out [m, H, d], the weights
    [Hk, n + m] of the last `window` rows, and sums of p |v|."""
    m, H = q.shape[:2]
    n, G = cache.length(b), H // cache.Hk
    out, spread, weights = np.zeros((m, H, cache.d)), np.zeros((m, H, cache.d)), np.zeros((cache.Hk, n + m))
    for kh in range(cache.Hk):
        cache.append(b, kh, k_new[:, kh], v_new[:, kh])
        k, v = cache.values(b, kh)
        for t in range(m):
            for h in range(kh * G, (kh + 1) * G):
                p = softmax_rows(q[t, h] @ k[:n + t + 1].T * scale)
                out[t, h], spread[t, h] = p @ v[:n + t + 1], p @ np.abs(v[:n + t + 1])
                if t >= m - window:
                    weights[kh, :n + t + 1] += p
    return out, weights, spread
