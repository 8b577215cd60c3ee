"""Call sequencing for decoders with grouped heads: packed prompts, caches of 8-bit blocks, further turns, eviction by accumulated weight.

Beside `pipeline` (one prompt length, visual segments, Alg. 3), for batches of sequences of different lengths.  This module owns the page
pool, tails, tables, scores and lengths and issues the library's calls; the only torch operations are allocations and the
lengths' own arithmetic, once a step for all layers.
"""
from __future__ import annotations

from typing import List, Optional, Sequence

import torch

from . import binding as st3


class BlockGeneration:
    """One batch of sequences through prompts, decode steps, further turns and evictions.

        gen = BlockGeneration(layers, heads, kv_heads, head_dim, batch, capacity=4096, budget=2048)
        gen.begin(prompt_lens)
        for l in range(layers):
            out = gen.prefill_layer(l, q, k, v)             # [T, heads or kv_heads, d], prompts one behind the other
        for each token:
            gen.begin_step()
            for l in range(layers):
                out = gen.decode_layer(l, q, k_new, v_new)  # [batch, heads or kv_heads, d]
            gen.finish_step()
        gen.begin_turn(new_lens)                            # several new tokens at once: the next question, a piece of a long prompt
        for l in range(layers):
            out = gen.extend_layer(l, q, k, v, rotary)      # [T, heads or kv_heads, d], packed like prompts
        gen.finish_turn()

    rotary (binding.rotary, of a table that st3_rotary_table made once for the turn) turns queries and keys on the way; without it they come
    turned, as those of prefill_layer and decode_layer do.
    capacity: rows that a sequence may hold; when the longest has come to it, begin_step() has every key head of every layer keep
    `budget` rows of each longer sequence: the first n_sink, the last n_recent, and of the others those that have received the most
    attention weight so far: from the prompt's last `window` rows, from every step's row, and from the last `window` rows of every turn that counts.
    A prompt may come in pieces, as turns behind begin() with lengths of 0; where only the last of them counts, and has `window` rows, weights are those
    of the prompt's last ones, wherever it was cut.
    Drafted tokens are checked in a turn that does not stay: it attends like any other and leaves the sequences as they were (but for an eviction that
    makes room).  Those that are accepted then come in a turn of their own, with the same rows of q, k and v.
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
        self._turn_ws = torch.empty((0,), dtype=torch.uint8, device=device)
        self._copies: List[st3.BlockCache] = []
        self.evictions = 0

    new: Optional[List[int]] = None             # rows that the turn adds, while one is open
    prompts: bool = True                        # the rows are the prompts' and nothing has come behind them

    def _no_turn(self) -> None:
        if self.new is not None:
            raise ValueError("a turn is open: finish_turn() comes first")

    # ------------------------------------------------------------------------------------
    def begin(self, prompt_lens: Sequence[int]) -> None:
        """A new batch; 0 tokens are a sequence that has none yet, -1 an empty place."""
        lens = [int(n) for n in prompt_lens]
        if len(lens) != self.B or min(lens) < -1 or max(lens) > self.capacity:
            raise ValueError(f"{self.B} lengths, up to {self.capacity}, expected; {lens} given")
        self.lens, self.evictions, self.new, self.prompts = lens, 0, None, True
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
        as the lengths that begin() was told have together, and before the first step's end, turn or eviction."""
        self._no_turn()
        if not self.prompts:
            raise ValueError("rows have come behind the prompts, or left them: begin() comes first")
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
        self._no_turn()
        if self.longest >= self.capacity:
            self.evict()

    def decode_layer(self, l: int, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor) -> torch.Tensor:
        """The step's token of every sequence in layer l; empty places get 0.  The result is valid until this layer's next step."""
        self._no_turn()
        st3.st3_block_decode(self.shape, q, k_new, v_new, self._sets[self._of[l]], self.longest, self._out[l], self.score[l], self._ws)
        return self._out[l]

    def finish_step(self) -> None:
        self._no_turn()
        self.prompts = False
        self.len.add_(self.live)
        self.lens = [n + 1 if n >= 0 else n for n in self.lens]

    # ------------------------------------------------------------------------------------
    def begin_turn(self, new_lens: Sequence[int], counts: bool = True, stays: bool = True) -> None:
        """A turn of so many new tokens of each sequence (an empty place has none); makes room where a sequence has too little.  counts: whether what
        the turn attends to counts as weight; where it does not, its own rows begin with none.  stays: whether the sequences have its rows behind
        finish_turn(); where they do not, nothing of it counts either."""
        self._no_turn()
        new = [int(m) for m in new_lens]
        if len(new) != self.B or min(new) < 0 or any(m and n < 0 for n, m in zip(self.lens, new)):
            raise ValueError(f"{self.B} numbers of new tokens, none for an empty place, expected; {new} given")
        if any(min(n, self.budget) + m > self.capacity for n, m in zip(self.lens, new)):
            raise ValueError(f"{new} new tokens do not fit behind {self.budget} rows into {self.capacity}")
        if any(n + m > self.capacity for n, m in zip(self.lens, new)):
            self.evict()
        starts = [0]
        for m in new:
            starts.append(starts[-1] + m)
        image = torch.tensor(new + starts, dtype=torch.int32).to(self.device)
        self.prompts, self.counts, self.stays = False, counts and stays, stays
        self.new, self.total, self._added, self.cu = new, starts[-1], image[:self.B], image[self.B:]
        self._top = max(0, max(n + m for n, m in zip(self.lens, new)))
        need = st3.st3_block_attend_workspace_bytes(self.shape, self.total, max(new), self._top)
        if need > self._turn_ws.numel():
            self._turn_ws = torch.empty((need,), dtype=torch.uint8, device=self.device)
        if stays and not counts and self.total > 0:
            rows = torch.arange(self._top, dtype=torch.int32, device=self.device) - self.len[:, None]
            self.score[..., :self._top].masked_fill_(((rows >= 0) & (rows < self._added[:, None]))[:, None], 0.0)

    def extend_layer(self, l: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, rotary: Optional[st3.Rotary] = None,
                     out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The turn's packed rows in layer l: queries and keys turned, keys and values appended, queries attended; the scores go on where the turn counts."""
        if self.new is None:
            raise ValueError("no turn is open: begin_turn() comes first")
        if not q.shape[0] == k.shape[0] == v.shape[0] == self.total:
            raise ValueError(f"{q.shape[0]}, {k.shape[0]} and {v.shape[0]} rows of q, k and v: {self.total} expected, the new tokens' sum")
        if out is None:
            out = torch.empty((q.shape[0], self.H, self.d), dtype=q.dtype, device=q.device)
        if self.total == 0:
            return out
        most, cache = max(self.new), self._sets[self._of[l]] if self.stays else self._copied_tails(self._of[l])
        st3.st3_block_append(self.shape, k, v, self.cu, most, cache, self._top, rotary)
        if rotary is not None:
            turned = torch.empty((q.shape[0], self.H, self.d), dtype=q.dtype, device=q.device)
            st3.st3_rotate_rows(q, turned, rotary)
            q = turned
        st3.st3_block_attend(self.shape, q, self.cu, most, cache, self._top, out, self.window, self.score[l] if self.counts else None, self._turn_ws)
        return out

    def _copied_tails(self, i: int) -> st3.BlockCache:
        """Set i's cache with copies of its tails.  Rows appended to it leave the set as it is: blocks that they fill go into pages that none of its
        lengths reach, but a tail that overflows is lost (so a lower length alone would not bring it back)."""
        if not self._copies:
            self._copied = torch.empty_like(self.k_tail[0]), torch.empty_like(self.v_tail[0])
            self._copies = [st3.block_cache(self.k_codes, self.v_codes, self.k_scale, self.v_scale, *self._copied, t, self.len) for t in self.tables]
        self._copied[0].copy_(self.k_tail[i])
        self._copied[1].copy_(self.v_tail[i])
        return self._copies[i]

    def finish_turn(self) -> None:
        if self.new is None:
            raise ValueError("no turn is open: begin_turn() comes first")
        if self.stays:
            self.len.add_(self._added * self.live)
            self.lens = [n + m if n >= 0 else n for n, m in zip(self.lens, self.new)]
        self.new = None

    def retire(self, b: int) -> None:
        """Sequence b has ended: its place stays empty until the next begin()."""
        self.len[b] = -1
        self.live[b] = 0
        self.lens[b] = -1

    def evict(self) -> None:
        """Every layer keeps `budget` rows of each longer sequence; `kept[l]` names them by the rows they had."""
        self._no_turn()
        if self.longest == 0:
            return
        self.prompts = False
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
