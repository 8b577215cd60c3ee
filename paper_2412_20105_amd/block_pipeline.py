"""Call sequencing for decoders with grouped heads: packed prompts, caches of 8-bit blocks, eviction by accumulated weight.

Beside `pipeline` (one prompt length, visual segments, Alg. 3), for batches of sequences of different lengths.  This module owns the page
pool, tails, tables, scores and lengths and issues the library's calls; the only torch operations are allocations and the
lengths' own arithmetic, once a step for all layers.
"""
from __future__ import annotations

from typing import List, Optional, Sequence

import torch

from . import binding as st3


class BlockGeneration:
    """One batch of sequences through prompts, decode steps and evictions.

        gen = BlockGeneration(layers, heads, kv_heads, head_dim, batch, capacity=4096, budget=2048)
        gen.begin(prompt_lens)
        for l in range(layers):
            out = gen.prefill_layer(l, q, k, v)             # [T, heads or kv_heads, d], prompts one behind the other
        for each token:
            gen.begin_step()
            for l in range(layers):
                out = gen.decode_layer(l, q, k_new, v_new)  # [batch, heads or kv_heads, d]
            gen.finish_step()

    capacity: rows that a sequence may hold; when the longest has come to it, begin_step() has every key head of every layer keep
    `budget` rows of each longer sequence: the first n_sink, the last n_recent, and of the others those that have received the most
    attention weight so far, counted from the prompt's last `window` rows on.
    Pages: a set of them for each layer and one to spare.  An eviction writes a layer's rows into the spare set, and the
    set that the layer leaves becomes the next one to spare.
    """

    def __init__(self, layers: int, heads: int, kv_heads: int, head_dim: int, batch: int, capacity: int, budget: int, n_sink: int = 4,
                 n_recent: int = 64, window: int = 32, code: int = st3.ST3_BLOCK_INT8, softmax_scale: float = 0.0, device: str = "cuda:0"):
        if layers < 1 or not 1 <= budget < capacity:
            raise ValueError(f"{layers} layers, {budget} rows to keep of {capacity}: one layer, and less than the capacity, expected")
        if n_sink < 0 or n_recent < 0 or n_sink + n_recent > budget:
            raise ValueError(f"{n_sink} first and {n_recent} last rows do not fit into {budget}")
        if window < 1:
            raise ValueError("the scores begin with one row of the prompt at least")
        if code not in (st3.ST3_BLOCK_INT8, st3.ST3_BLOCK_E4M3):
            raise ValueError(f"no code of blocks: {code}")
        self.L, self.H, self.Hk, self.d, self.B = layers, heads, kv_heads, head_dim, batch
        self.capacity, self.budget, self.n_sink, self.n_recent, self.window = capacity, budget, n_sink, n_recent, window
        self.device = device
        self.shape = st3.gqa_shape(batch, heads, kv_heads, head_dim, st3.ST3_BF16, softmax_scale)
        blk, sets = st3.ST3_BLOCK_TOKENS, layers + 1
        self.blocks = -(-capacity // blk)
        pages = sets * batch * self.blocks
        byte = dict(dtype=torch.int8 if code == st3.ST3_BLOCK_INT8 else torch.uint8, device=device)
        half, single, count = (dict(dtype=t, device=device) for t in (torch.bfloat16, torch.float32, torch.int32))
        self.k_codes = torch.empty((pages, kv_heads, blk, head_dim), **byte)
        self.v_codes = torch.empty((pages, kv_heads, head_dim, blk), **byte)
        self.k_scale, self.v_scale = (torch.empty((pages, kv_heads), **single) for _ in range(2))
        self.k_tail = torch.empty((sets, batch, kv_heads, blk, head_dim), **half)
        self.v_tail = torch.empty((sets, batch, kv_heads, head_dim, blk), **half)
        self.tables = torch.arange(pages, **count).view(sets, batch, self.blocks)
        self.len = torch.full((batch,), -1, **count)
        self.live = torch.zeros((batch,), **count)
        self.score = torch.zeros((layers, batch, kv_heads, capacity), **single)
        self.kept = torch.full((layers, batch, kv_heads, budget), -1, **count)
        self._sets = [st3.block_cache(self.k_codes, self.v_codes, self.k_scale, self.v_scale, self.k_tail[i], self.v_tail[i], self.tables[i],
                                      self.len) for i in range(sets)]
        self._of = list(range(layers))          # the set that holds a layer
        self._spare = layers
        self._ws = torch.empty((max(256, st3.st3_block_workspace_bytes(self.shape, capacity - 1)),), dtype=torch.uint8, device=device)
        self._prompt_ws = torch.empty((0,), dtype=torch.uint8, device=device)
        self._out = torch.empty((layers, batch, heads, head_dim), **half)
        self.lens: List[int] = [-1] * batch     # host copies; negative: an empty place
        self.evictions = 0

    # ------------------------------------------------------------------------------------
    def begin(self, prompt_lens: Sequence[int]) -> None:
        """A new batch; 0 tokens are a sequence that has none yet, -1 an empty place."""
        lens = [int(n) for n in prompt_lens]
        if len(lens) != self.B or min(lens) < -1 or max(lens) > self.capacity:
            raise ValueError(f"{self.B} lengths, up to {self.capacity}, expected; {lens} given")
        self.lens, self.evictions = lens, 0
        starts = [0]
        for n in lens:
            starts.append(starts[-1] + max(n, 0))
        image = torch.tensor(lens + [int(n >= 0) for n in lens] + starts, dtype=torch.int32).to(self.device)
        self.len.copy_(image[:self.B])
        self.live.copy_(image[self.B:2 * self.B])
        self.cu = image[2 * self.B:]
        self.total = starts[-1]
        need = st3.st3_packed_workspace_bytes(self.shape, self.total)
        if need > self._prompt_ws.numel():
            self._prompt_ws = torch.empty((need,), dtype=torch.uint8, device=self.device)

    @property
    def longest(self) -> int:
        return max(0, max(self.lens))

    def prefill_layer(self, l: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Packed prompts (slices of a fused projection's output are fine) of layer l: attended, and stored.  As many rows
        as the lengths that begin() was told have together."""
        if not q.shape[0] == k.shape[0] == v.shape[0] == self.total:
            raise ValueError(f"{q.shape[0]}, {k.shape[0]} and {v.shape[0]} rows of q, k and v: {self.total} expected, the lengths' sum")
        if out is None:
            out = torch.empty((q.shape[0], self.H, self.d), dtype=q.dtype, device=q.device)
        if self.total == 0:
            return out
        st3.st3_packed_attention(self.shape, q, k, v, self.cu, self.longest, out, self.window, self.score[l], self._prompt_ws)
        st3.st3_block_store(self.shape, k, v, self.cu, self.longest, self._sets[self._of[l]])
        return out

    def begin_step(self) -> None:
        """Makes room where a sequence has none left for the step's row."""
        if self.longest >= self.capacity:
            self.evict()

    def decode_layer(self, l: int, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor) -> torch.Tensor:
        """The step's token of every sequence in layer l; empty places get 0.  The result is valid until this layer's next step."""
        st3.st3_block_decode(self.shape, q, k_new, v_new, self._sets[self._of[l]], self.longest, self._out[l], self.score[l], self._ws)
        return self._out[l]

    def finish_step(self) -> None:
        self.len.add_(self.live)
        self.lens = [n + 1 if n >= 0 else n for n in self.lens]

    def retire(self, b: int) -> None:
        """Sequence b has ended: its place stays empty until the next begin()."""
        self.len[b] = -1
        self.live[b] = 0
        self.lens[b] = -1

    def evict(self) -> None:
        """Every layer keeps `budget` rows of each longer sequence; `kept[l]` names them by the rows they had."""
        if self.longest == 0:
            return
        for l in range(self.L):
            st3.st3_block_evict(self.shape, self._sets[self._of[l]], self._sets[self._spare], self.longest, self.budget, self.n_sink, self.n_recent,
                                self.score[l], self.score[l], self.kept[l])
            self._of[l], self._spare = self._spare, self._of[l]
        self.len.clamp_(max=self.budget)
        self.lens = [min(n, self.budget) for n in self.lens]
        self.evictions += 1

    # ------------------------------------------------------------------------------------
    def cache(self, l: int) -> st3.BlockCache:
        """Layer l's cache as the library's calls take it."""
        return self._sets[self._of[l]]

    def table(self, l: int) -> torch.Tensor:
        return self.tables[self._of[l]]

    def tails(self, l: int):
        return self.k_tail[self._of[l]], self.v_tail[self._of[l]]

    def kv_bytes(self) -> int:
        """Bytes of K and V that a decode step reads: codes and scales of whole blocks, 16-bit rows behind them."""
        blk, total = st3.ST3_BLOCK_TOKENS, 0
        for n in self.lens:
            if n > 0:
                total += n // blk * (blk * self.d + 4) + n % blk * 2 * self.d
        return 2 * total * self.Hk * self.L
