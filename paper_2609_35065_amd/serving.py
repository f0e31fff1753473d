"""Serving over a paged cache: new tokens through the operators of one GPU.

``ServedCache`` takes the paged tensors that a retrieve filled (or empty ones)
and runs, for each step of a ragged batch, every layer's
    kv_rope_append        the new tokens' rotated keys, and values, into the blocks
    kv_paged_attention    their attention over all that the cache holds
    kv_attention_weights  what each cached token received, accumulated
and between steps, to hold fewer bytes, kv_evict_select and kv_evict_compact.
With several axes of positions the first is kv_rope_append_axes, with a
sliding window and sinks the others are kv_sink_attention and kv_sink_weights.
A token's cache index changes when others are evicted, its rotary position
does not, so both are counted.  A sliding window reaches back over positions,
the operators' over cache indices: an eviction therefore has to leave the
tokens that a window still reaches, and the sinks.  Or evictions renumber:
kv_rope_shift then turns the kept keys to the positions that their cache
indices are, so that a stream's positions stay below what its cache holds.

This module only sequences the calls and owns their buffers; it computes
nothing itself and never waits for the GPU: what a step uploads lies in pinned
memory, so that the host may be steps ahead.
"""
from __future__ import annotations

from typing import List, Optional, Sequence

import numpy as np
import torch

from . import (KV_MAX_AXES, KvLayout, kv_attention_weights, kv_evict_compact, kv_evict_select, kv_paged_attention,
               kv_rope_append, kv_rope_append_axes, kv_rope_shift, kv_sink_attention, kv_sink_attention_workspace,
               kv_sink_weights, kv_sink_weights_workspace, make_batch)


class ServedCache:
    """The cache of ``len(lengths)`` requests, which hold ``lengths`` tokens at positions 0, 1, ... at the start.

    ``layers`` and ``block_tables`` (int32 [requests, n]) are the paged tensors and tables of the copies;
    ``freqs`` (float64, on the device) and ``magnitude`` come from kv_rope_frequencies.  ``decay`` is the factor on
    weights accumulated in earlier steps (None: weights are not kept, and nothing can be evicted); ``k_scale`` and
    ``v_scale`` are float32 [layers, kv_heads] for an 8-bit cache.

    With a ``window`` the first ``sink`` tokens of each request stay visible.  ``axes`` (kv_rope_axes) makes positions
    have several axes, which ``begin`` takes.  ``renumber`` makes every eviction give the kept tokens the positions
    0, 1, ... in the cache's order, head by head (only with one axis: the tokens of several have no such order).  Each
    such eviction rounds the keys that it moves to the cache's type once more, and these roundings add up: evict many
    tokens at a time rather than one a step, above all from an 8-bit cache.

    The layers of a step share buffers, so that calls follow one another on the GPU: one that comes on another stream
    than the last waits for that one's work.  (Not in a graph capture: its replays are the program's to order.)"""

    def __init__(self, layout: KvLayout, layers: Sequence[torch.Tensor], block_tables: torch.Tensor, lengths,
                 q_heads: int, freqs: torch.Tensor, *, magnitude: float = 1.0, interleaved: bool = False,
                 scale: Optional[float] = None, window: int = 0, sink: int = 0, axes: Optional[np.ndarray] = None,
                 renumber: bool = False, decay: Optional[float] = 1.0, k_scale: Optional[torch.Tensor] = None,
                 v_scale: Optional[torch.Tensor] = None):
        self.layout, self.layers, self.block_tables = layout, list(layers), block_tables
        self.q_heads, self.freqs, self.magnitude, self.interleaved = q_heads, freqs, magnitude, interleaved
        self.scale = layout.head_dim ** -0.5 if scale is None else scale
        self.window, self.sink, self.decay, self.k_scale, self.v_scale = window, sink, decay, k_scale, v_scale
        if sink < 0:
            raise ValueError("sink must not be negative")
        if renumber and axes is not None:
            raise ValueError("evictions renumber positions of one axis only")
        self.axes, self.renumber = None if axes is None else np.ascontiguousarray(axes, np.uint8), renumber
        self.num_axes = 1 if axes is None else int(self.axes.max(initial=0)) + 1
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
        self._dtype = None                                      # of 16-bit keys, once a layer has been attended
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

    def begin(self, new, positions=None) -> None:
        """Start a step: ``new`` tokens of each request (0, 1 or many).  With several axes, ``positions`` [axes, rows]
        are those of the new tokens (text, the same on all axes: None); a request goes on after its largest, of this
        step and of those before.  Tokens held at the start have positions 0, 1, ...; where they have others, set the
        request's next one, ``positions[r]``, first."""
        new = np.asarray(new, np.int64)
        if new.shape != self.lengths.shape or (new < 0).any() or (self.lengths + new > self.capacity).any():
            raise ValueError("new must hold one count per request, and leave every request within its block table")
        # (the counts change last: a step that is refused leaves them as they were)
        lengths = self.lengths + new
        off = np.concatenate([[0], np.cumsum(new)])
        pos = np.concatenate([np.arange(p, p + n) for p, n in zip(self.positions, new)])
        after = self.positions + new
        if positions is not None:
            given = np.asarray(positions)
            # (there may be axes that no pair takes)
            if self.axes is None or given.ndim != 2 or not self.num_axes <= given.shape[0] <= KV_MAX_AXES \
                    or given.shape[1] != pos.size or given.dtype.kind not in "iu" \
                    or (given.size and (given.min() < -1 << 31 or given.max() >= 1 << 31)):
                raise ValueError(f"positions must be [axes, {pos.size}] whole numbers of 32 bits, of {self.num_axes} to "
                                 f"{KV_MAX_AXES} axes, for a cache with axes")
            pos = given
            if pos.size:
                largest = np.maximum.reduceat(pos.max(0).astype(np.int64), off[:-1][new > 0])
                after[new > 0] = np.maximum(self.positions[new > 0], largest + 1)
        else:
            if (after[new > 0] > 1 << 31).any():
                raise ValueError("positions must stay below 2^31")
            if self.axes is not None:
                pos = np.tile(pos, (self.num_axes, 1))
        self._follow()
        d_off, d_len, d_pos = self._upload(off, lengths.astype(np.int32), np.ascontiguousarray(pos, np.int32).ravel())
        if self.axes is not None:
            d_pos = d_pos.view(pos.shape)
        batch = make_batch(d_off, d_len, self.block_tables, int(off[-1]), int(new.max(initial=0)),
                           int(lengths.max(initial=0)))
        size = kv_sink_attention_workspace(self.layout, batch, self.q_heads, self.window, self.sink)
        if self.sink and self.weights is not None:
            size = max(size, kv_sink_weights_workspace(self.layout, batch, self.q_heads, self.window, self.sink))
        if size and (self._workspace is None or self._workspace.numel() < size):
            self._workspace = torch.empty(size, dtype=torch.uint8, device=self.dev)
        lse = torch.empty((batch.num_q, self.q_heads), dtype=torch.float32, device=self.dev)
        self.batch, self._lse, self._positions = batch, lse, d_pos
        self.lengths, self.positions = lengths, after

    def attend(self, layer: int, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor) -> None:
        """One layer of the step: q [rows, q_heads, head_dim] is rotated in place, k and v go into the cache, and
        ``out`` gets the attention of q over the cache."""
        if self.batch is None:
            raise ValueError("no step: begin one first, and after an eviction")
        self._follow()
        ks = None if self.k_scale is None else self.k_scale[layer]
        vs = None if self.v_scale is None else self.v_scale[layer]
        pool = self.layers[layer]
        self._dtype = q.dtype
        turn = dict(interleaved=self.interleaved, magnitude=self.magnitude, k_scale=ks, v_scale=vs)
        if self.axes is None:
            kv_rope_append(self.layout, pool, self.batch, q, k, v, self.freqs, positions=self._positions, **turn)
        else:
            kv_rope_append_axes(self.layout, pool, self.batch, q, k, v, self.freqs, self.axes, self._positions, **turn)
        if self.sink:
            kv_sink_attention(self.layout, pool, self.batch, q, out, self.scale, self.window, self.sink, lse=self._lse,
                              k_scale=ks, v_scale=vs, workspace=self._workspace)
            if self.weights is not None:
                kv_sink_weights(self.layout, pool, self.batch, q, self._lse, self.weights[layer], self.scale, self.window,
                                self.sink, decay=self.decay, k_scale=ks, workspace=self._workspace)
            return
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
        the window, a cache without one gives the same results.)  A cache that renumbers needs no such tokens: its
        window is one over the new positions.  A cache with sinks keeps at least those first tokens."""
        if self.weights is None:
            raise ValueError("nothing to choose by: this cache keeps no weights")
        # (the operators take 2^30 and more as no window)
        windowed, cut = 0 < self.window < 1 << 30, bool((self.lengths > budget).any())
        if windowed and cut and sink < self.sink:
            raise ValueError(f"an eviction has to leave the first {self.sink} tokens, which stay visible, not {sink}")
        if windowed and cut and recent < self.window - 1 and not self.renumber:
            raise ValueError(f"an eviction has to leave the last {self.window - 1} tokens, which the window reaches, "
                             f"not {recent}")
        held = [t.dtype for t in self.layers if isinstance(t, torch.Tensor) and t.is_floating_point()]
        dtype = held[0] if held else self._dtype
        if self.renumber and self.layout.elem_bytes == 2 and dtype is None:
            raise ValueError("the type of the keys is not known before a layer is attended")
        self._follow()
        L, R, h, _ = self.weights.shape
        keep = torch.empty((L, R, h, budget), dtype=torch.int32, device=self.dev)
        left = torch.empty(R, dtype=torch.int32, device=self.dev)
        size, = self._upload(self.lengths.astype(np.int32))
        kv_evict_select(self.weights, size, budget, sink, recent, keep, left)
        kv_evict_compact(self.layout, self.layers, self.block_tables, keep, left, weights=self.weights)
        if self.renumber:
            # a kept token's position was its index before, and is its index now
            now = torch.arange(budget, dtype=torch.int32, device=self.dev)
            kv_rope_shift(self.layout, self.layers, self.block_tables, left, min(budget, int(self.lengths.max(initial=0))),
                          torch.where(keep >= 0, now - keep, 0), self.freqs, interleaved=self.interleaved,
                          cache_dtype=dtype if self.layout.elem_bytes == 2 else None)
            self.positions = np.minimum(self.lengths, budget)
        # what lies behind the kept tokens belongs to none: new tokens start from 0
        gone = torch.arange(self.capacity, device=self.dev) >= left[:, None]
        self.weights.masked_fill_(gone[None, :, None], 0.0)
        self.lengths, self.batch = np.minimum(self.lengths, budget), None       # the step's lengths are gone
        return [int(-(-n // self.layout.block_size)) for n in self.lengths]
