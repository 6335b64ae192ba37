"""Attention of a multi-view denoiser over a slice of the views (Sec. 3.2,
batch-sliced anchor forward).

A cached step runs the denoiser on the anchor views only, and every token
keeps the structural index and the rotary slot it has among all views.  Only
foreground tokens take part: an asset's foreground tokens of the listed views
form one sequence, the assets' sequences lie end to end without padding, and a
token's rotary position is its (view, row, column) in the full set of views.

What follows from the views alone (token indexes, positions, the attention
plan) is built on first use and kept by the list of views for a layer's later
steps, as the runner keeps its correspondence operators.  A layer keeps the
lists used last, as many as a rotation of the most views has distinct sets:
an adaptive choice of anchors seldom repeats one.
"""
from __future__ import annotations

import math
from collections import OrderedDict
from dataclasses import dataclass, field
from typing import List, Optional, Sequence, Set, Tuple

import torch

from . import (GC_MAX_VIEWS, GC_ROPE_HALF, AttentionPlan, gc_attention, gc_attention_plan, gc_qk_norm_rope,
               gc_rope_table)


@dataclass
class TokenSlice:
    """Foreground tokens of a list of views: rows of the flattened
    [B, len(views), H, W] grid (int64), asset by asset; each asset's number of
    them; their (view, row, column) (int32 [T, 3]); the plan of attention
    among each asset's own."""
    index: torch.Tensor
    lens: List[int]
    positions: torch.Tensor
    plan: AttentionPlan
    # handles of the streams after whose work torch's allocator reuses the tensors' memory
    known_streams: Set[int] = field(default_factory=set)

    def used_here(self) -> None:
        """Work on the current stream reads the slice: its memory stays its
        own until that is done, also where the slice is dropped before."""
        stream = torch.cuda.current_stream(self.index.device)
        if stream.cuda_stream not in self.known_streams:
            self.index.record_stream(stream)
            self.positions.record_stream(stream)
            self.known_streams.add(stream.cuda_stream)

    def __getstate__(self):   # a copy's memory is another, known on no stream
        return {**self.__dict__, "known_streams": set()}


class MultiViewAttention:
    """softmax(q k) v of each asset's foreground tokens, with per-head RMS
    norms of queries and keys and rotary positions, between a fused input
    projection and an output projection.  The forward pass only: a call that
    torch would record for a gradient is refused.  One layer may be called
    under several streams and from several threads at the same time."""

    MOST_SLICES = GC_MAX_VIEWS + 1   # a rotation's distinct sets, and all views

    def __init__(self, pos: torch.Tensor, width: int, heads: int, kv_heads: int, dim: int,
                 dtype: torch.dtype = torch.bfloat16, sections: Optional[Sequence[int]] = None, base: float = 10000.0,
                 generator: Optional[torch.Generator] = None):
        """pos: device float32 [B, N, H, W, 3] position maps (NaN: background).
        sections: columns of the rotation for the view, row and column axes
        (default: the whole head, a quarter of it for the view).  The weights
        are drawn from the generator; load others into w_qkv [width, (heads +
        2 kv_heads) dim], w_out [heads dim, width], q_gain and k_gain [dim]."""
        self.B, self.N, self.H, self.W = pos.shape[:4]
        self.width, self.heads, self.kv_heads, self.dim, self.dtype = width, heads, kv_heads, dim, dtype
        if sections is None:
            view = dim // 8
            sections = (view, (dim // 2 - view) // 2, dim // 2 - view - (dim // 2 - view) // 2)
        self.sections = tuple(int(n) for n in sections)
        dev = pos.device
        self.foreground = torch.isfinite(pos).all(-1)                     # [B, N, H, W]
        self.table = gc_rope_table(max(self.N, self.H, self.W), self.sections, base, device=dev)
        rand = lambda *shape: torch.randn(shape, generator=generator, device=dev)
        self.w_qkv = (rand(width, (heads + 2 * kv_heads) * dim) / math.sqrt(width)).to(dtype)
        self.w_out = (rand(heads * dim, width) / math.sqrt(heads * dim)).to(dtype)
        self.q_gain = torch.ones(dim, dtype=torch.float32, device=dev)
        self.k_gain = torch.ones(dim, dtype=torch.float32, device=dev)
        self._slices: OrderedDict[Tuple[int, ...], TokenSlice] = OrderedDict()   # the one used last at the end

    def slice(self, views: Sequence[int]) -> TokenSlice:
        """The tokens of a list of views, built where it is not among the
        MOST_SLICES lists used last (one read-back of the assets' token
        counts)."""
        key = tuple(int(v) for v in views)
        if any(not 0 <= v < self.N for v in key):
            raise ValueError(f"views must lie in [0, {self.N}) (got {list(key)})")
        got = self._slices.pop(key, None)   # (each dict operation is whole under threads; at worst a list is built twice)
        if got is None:
            fg = self.foreground[:, list(key)]                            # [B, n, H, W]
            at = fg.nonzero()                                             # asset, place in the list, row, column
            lens = [int(n) for n in fg.flatten(1).sum(1).tolist()]
            index = ((at[:, 0] * len(key) + at[:, 1]) * self.H + at[:, 2]) * self.W + at[:, 3]
            view = torch.tensor(key, dtype=torch.int64, device=fg.device)[at[:, 1]]
            positions = torch.stack([view, at[:, 2], at[:, 3]], 1).to(torch.int32)
            # (last: its copy of the items waits for the stream, so any stream may read all of the slice)
            plan = gc_attention_plan(lens, lens, self.heads, self.kv_heads, self.dim, self.dtype, device=fg.device)
            got = TokenSlice(index, lens, positions, plan, {torch.cuda.current_stream(fg.device).cuda_stream})
        self._slices[key] = got
        while len(self._slices) > self.MOST_SLICES:
            self._slices.popitem(last=False)
        return got

    def __call__(self, x: torch.Tensor, views: Sequence[int]) -> torch.Tensor:
        """x [B, len(views), H, W, width] of the layer's type -> the layer's
        output on foreground tokens, zeros on the background."""
        shape = (self.B, len(views), self.H, self.W, self.width)
        if x.shape != shape or x.dtype != self.dtype or x.device != self.foreground.device:
            raise ValueError(f"x must be {self.dtype} {list(shape)} on {self.foreground.device} (got {x.dtype} "
                             f"{list(x.shape)} on {x.device})")
        if torch.is_grad_enabled() and any(t.requires_grad for t in (x, self.w_qkv, self.w_out, self.q_gain, self.k_gain)):
            raise ValueError("the layer has no gradient: call it under torch.no_grad(), or on tensors that require none")
        s = self.slice(views)
        s.used_here()
        H, Hk, D = self.heads, self.kv_heads, self.dim
        tokens = x.reshape(-1, self.width)[s.index]
        qkv = (tokens @ self.w_qkv).view(-1, H + 2 * Hk, D)
        q, k, v = qkv.split([H, Hk, Hk], dim=1)
        gc_qk_norm_rope(q, k, self.q_gain, self.k_gain, s.positions, self.table, sections=self.sections,
                        layout=GC_ROPE_HALF, q_out=q, k_out=k)            # where the projection left them
        out, _ = gc_attention(q, k, v, s.plan)
        y = torch.zeros(x.shape, dtype=x.dtype, device=x.device)          # (zeros_like keeps a permuted x's order)
        y.view(-1, self.width)[s.index] = out.view(-1, H * D) @ self.w_out
        return y
