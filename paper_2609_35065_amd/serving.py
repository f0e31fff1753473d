"""Serving over a paged cache: new tokens through the operators of one GPU.

``ServedCache`` takes the paged tensors that a retrieve filled (or empty ones)
and runs, for each step of a ragged batch, every layer's
    kv_rope_append        the new tokens' rotated keys, and values, into the blocks
    kv_paged_attention    their attention over all that the cache holds
    kv_attention_weights  what each cached token received, accumulated
and between steps, to hold fewer bytes, kv_evict_select and kv_evict_compact.
A token's cache index changes when others are evicted, its rotary position
does not, so both are counted.  A sliding window reaches back over positions,
the operators' over cache indices: an eviction therefore has to leave the
tokens that a window still reaches.

This module only sequences the calls and owns their buffers; it computes
nothing itself and never waits for the GPU: what a step uploads lies in pinned
memory, so that the host may be steps ahead.
"""
from __future__ import annotations

from typing import List, Optional, Sequence

import numpy as np
import torch

from . import (KvLayout, kv_attention_weights, kv_evict_compact, kv_evict_select, kv_paged_attention,
               kv_paged_attention_workspace, kv_rope_append, make_batch)


class ServedCache:
    """The cache of ``len(lengths)`` requests, which hold ``lengths`` tokens at positions 0, 1, ... at the start.

    ``layers`` and ``block_tables`` (int32 [requests, n]) are the paged tensors and tables of the copies;
    ``freqs`` (float64, on the device) and ``magnitude`` come from kv_rope_frequencies.  ``decay`` is the factor on
    weights accumulated in earlier steps (None: weights are not kept, and nothing can be evicted); ``k_scale`` and
    ``v_scale`` are float32 [layers, kv_heads] for an 8-bit cache.

    The layers of a step share buffers, so that calls follow one another on the GPU: one that comes on another stream
    than the last waits for that one's work.  (Not in a graph capture: its replays are the program's to order.)"""

    def __init__(self, layout: KvLayout, layers: Sequence[torch.Tensor], block_tables: torch.Tensor, lengths,
                 q_heads: int, freqs: torch.Tensor, *, magnitude: float = 1.0, interleaved: bool = False,
                 scale: Optional[float] = None, window: int = 0, decay: Optional[float] = 1.0,
                 k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None):
        self.layout, self.layers, self.block_tables = layout, list(layers), block_tables
        self.q_heads, self.freqs, self.magnitude, self.interleaved = q_heads, freqs, magnitude, interleaved
        self.scale = layout.head_dim ** -0.5 if scale is None else scale
        self.window, self.decay, self.k_scale, self.v_scale = window, decay, k_scale, v_scale
        self.dev = block_tables.device
        self.capacity = block_tables.shape[1] * layout.block_size
        self.lengths = np.asarray(lengths, np.int64).copy()     # tokens that the cache holds
        self.positions = self.lengths.copy()                    # position of each request's next token
        if self.lengths.shape != (block_tables.shape[0],) or (self.lengths < 0).any() \
                or (self.lengths > self.capacity).any():
            raise ValueError("lengths must hold one length per request, within its block table")
        self.weights = None
        if decay is not None:
            self.weights = torch.zeros((layout.num_layers, len(self.lengths), layout.kv_heads, self.capacity),
                                       dtype=torch.float32, device=self.dev)
        self.batch, self._workspace, self._lse, self._positions = None, None, None, None
        self._stream = torch.cuda.current_stream(self.dev) if self.dev.type == "cuda" else None

    def _follow(self) -> None:
        """Put the current stream behind the one of the last call, and keep the buffers for it."""
        now = torch.cuda.current_stream(self.dev)
        if now == self._stream or torch.cuda.is_current_stream_capturing():
            return
        now.wait_stream(self._stream)
        self._stream = now
        held = [self.weights, self._workspace, self._lse, self._positions]
        for t in held + list(self.batch.tensors if self.batch else ()):
            if t is not None:
                t.record_stream(now)

    def _upload(self, *arrays: np.ndarray) -> List[torch.Tensor]:
        """Copies on the device, by one upload from pinned memory that the allocator keeps until it is done.  64-bit
        arrays come first, so that all are aligned."""
        ends = np.cumsum([0] + [x.nbytes for x in arrays])
        host = torch.empty(int(ends[-1]), dtype=torch.uint8, pin_memory=self.dev.type == "cuda")
        for x, a, b in zip(arrays, ends, ends[1:]):
            host.numpy()[a:b] = x.view(np.uint8)
        there = host.to(self.dev, non_blocking=True)
        return [there[a:b].view(torch.from_numpy(x).dtype) for x, a, b in zip(arrays, ends, ends[1:])]

    def begin(self, new) -> None:
        """Start a step: ``new`` tokens of each request (0, 1 or many)."""
        new = np.asarray(new, np.int64)
        if new.shape != self.lengths.shape or (new < 0).any() or (self.lengths + new > self.capacity).any():
            raise ValueError("new must hold one count per request, and leave every request within its block table")
        self._follow()
        # (the counts change last: a step that is refused leaves them as they were)
        lengths = self.lengths + new
        off = np.concatenate([[0], np.cumsum(new)])
        pos = np.concatenate([np.arange(p, p + n) for p, n in zip(self.positions, new)]).astype(np.int32)
        d_off, d_len, d_pos = self._upload(off, lengths.astype(np.int32), pos)
        batch = make_batch(d_off, d_len, self.block_tables, int(off[-1]), int(new.max(initial=0)),
                           int(lengths.max(initial=0)))
        size = kv_paged_attention_workspace(self.layout, batch, self.q_heads, self.window)
        if size and (self._workspace is None or self._workspace.numel() < size):
            self._workspace = torch.empty(size, dtype=torch.uint8, device=self.dev)
        lse = torch.empty((batch.num_q, self.q_heads), dtype=torch.float32, device=self.dev)
        self.batch, self._lse, self._positions = batch, lse, d_pos
        self.lengths, self.positions = lengths, self.positions + new

    def attend(self, layer: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor) -> None:
        """One layer of the step: q [rows, q_heads, head_dim] is rotated in place, k and v go into the cache, and
        ``out`` gets the attention of q over the cache."""
        if self.batch is None:
            raise ValueError("no step: begin one first, and after an eviction")
        self._follow()
        ks = None if self.k_scale is None else self.k_scale[layer]
        vs = None if self.v_scale is None else self.v_scale[layer]
        pool = self.layers[layer]
        kv_rope_append(self.layout, pool, self.batch, q, k, v, self.freqs, interleaved=self.interleaved,
                       magnitude=self.magnitude, positions=self._positions, k_scale=ks, v_scale=vs)
        kv_paged_attention(self.layout, pool, self.batch, q, out, self.scale, window=self.window, lse=self._lse,
                           k_scale=ks, v_scale=vs, workspace=self._workspace)
        if self.weights is not None:
            kv_attention_weights(self.layout, pool, self.batch, q, self._lse, self.weights[layer], self.scale,
                                 window=self.window, decay=self.decay, k_scale=ks)

    def evict(self, budget: int, sink: int = 0, recent: int = 0) -> List[int]:
        """Cut every request to ``budget`` tokens per head and layer: the first ``sink``, the last ``recent``, and the
        most attended of the rest.  Returns how many blocks of each request's table are still in use.  With a window,
        ``recent`` must be at least ``window - 1`` where a request is cut: those tokens then lie next to one another
        in the cache as in the text, and a window over indices is one over positions.  (Where no position will reach
        the window, a cache without one gives the same results.)"""
        if self.weights is None:
            raise ValueError("nothing to choose by: this cache keeps no weights")
        # (the operators take 2^30 and more as no window)
        if 0 < self.window < 1 << 30 and recent < self.window - 1 and (self.lengths > budget).any():
            raise ValueError(f"an eviction has to leave the last {self.window - 1} tokens, which the window reaches, "
                             f"not {recent}")
        self._follow()
        L, R, h, _ = self.weights.shape
        keep = torch.empty((L, R, h, budget), dtype=torch.int32, device=self.dev)
        left = torch.empty(R, dtype=torch.int32, device=self.dev)
        size, = self._upload(self.lengths.astype(np.int32))
        kv_evict_select(self.weights, size, budget, sink, recent, keep, left)
        kv_evict_compact(self.layout, self.layers, self.block_tables, keep, left, weights=self.weights)
        # what lies behind the kept tokens belongs to none: new tokens start from 0
        gone = torch.arange(self.capacity, device=self.dev) >= left[:, None]
        self.weights.masked_fill_(gone[None, :, None], 0.0)
        self.lengths, self.batch = np.minimum(self.lengths, budget), None       # the step's lengths are gone
        return [int(-(-n // self.layout.block_size)) for n in self.lengths]
