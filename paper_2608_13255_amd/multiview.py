"""Attention, and whole blocks, of a multi-view denoiser over a slice of the
views (Sec. 3.2, batch-sliced anchor forward).

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
from typing import Dict, List, Optional, Sequence, Set, Tuple

import torch
from torch.autograd import forward_ad

from . import (GC_ACT_SILU, GC_MAX_VIEWS, GC_ROPE_HALF, AttentionPlan, gc_add_rms_norm, gc_attention, gc_attention_plan,
               gc_linear, gc_qk_norm_rope, gc_quantize_rows, gc_rope_table)


def _has_tangent(tensors: Sequence[Optional[torch.Tensor]]) -> bool:
    """Whether torch carries a forward-mode derivative of one of them along."""
    if getattr(forward_ad, "_current_level", 0) < 0 or torch.is_inference_mode_enabled():   # (no dual_level() is open)
        return False
    return any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors)


class _Shared:
    """Tensors that calls on several streams read.  known_streams: handles of
    the streams after whose work torch's allocator reuses their memory."""

    def _tensors(self) -> Sequence[torch.Tensor]:
        raise NotImplementedError

    def used_here(self) -> None:
        """Work on the current stream reads the tensors: their memory stays
        theirs until that is done, also where they are dropped before."""
        tensors = self._tensors()
        stream = torch.cuda.current_stream(tensors[0].device)
        if stream.cuda_stream not in self.known_streams:
            for t in tensors:
                t.record_stream(stream)
            self.known_streams.add(stream.cuda_stream)

    def __getstate__(self):   # a copy's memory is another, known on no stream
        return {**self.__dict__, "known_streams": set()}


@dataclass
class TokenSlice(_Shared):
    """Foreground tokens of a list of views: rows of the flattened
    [B, len(views), H, W] grid (int64), asset by asset; each asset's number of
    them; their (view, row, column) (int32 [T, 3]); the plan of attention
    among each asset's own."""
    index: torch.Tensor
    lens: List[int]
    positions: torch.Tensor
    plan: AttentionPlan
    known_streams: Set[int] = field(default_factory=set)

    def _tensors(self) -> Sequence[torch.Tensor]:
        return self.index, self.positions


class EightBitWeights(_Shared, Dict[str, Tuple[torch.Tensor, torch.Tensor]]):
    """(8-bit rows, their scales) of a block's weights by name."""

    def __init__(self, *args, **kwargs):
        super().__init__(*args, **kwargs)
        self.known_streams: Set[int] = set()

    def _tensors(self) -> Sequence[torch.Tensor]:
        return [t for pair in self.values() for t in pair]


class _SlicedAttention:
    """What follows from the position maps and the views at hand, and
    attention between its projections."""

    MOST_SLICES = GC_MAX_VIEWS + 1   # a rotation's distinct sets, and all views

    def __init__(self, pos: torch.Tensor, width: int, heads: int, kv_heads: int, dim: int, dtype: torch.dtype,
                 sections: Optional[Sequence[int]], base: float):
        self.B, self.N, self.H, self.W = pos.shape[:4]
        self.width, self.heads, self.kv_heads, self.dim, self.dtype = width, heads, kv_heads, dim, dtype
        if sections is None:
            view = dim // 8
            sections = (view, (dim // 2 - view) // 2, dim // 2 - view - (dim // 2 - view) // 2)
        self.sections = tuple(int(n) for n in sections)
        dev = pos.device
        self.foreground = torch.isfinite(pos).all(-1)                     # [B, N, H, W]
        self.table = gc_rope_table(max(self.N, self.H, self.W), self.sections, base, device=dev)
        self.q_gain = torch.ones(dim, dtype=torch.float32, device=dev)
        self.k_gain = torch.ones(dim, dtype=torch.float32, device=dev)
        self._slices: OrderedDict[Tuple[int, ...], TokenSlice] = OrderedDict()   # the one used last at the end
        self._captured: Dict[int, _Shared] = {}                           # what graphs read at their replays

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

    def _uses(self, shared: _Shared) -> None:
        """Work on the current stream reads `shared`; where that is captured
        into a graph, each of its replays does, for as long as the layer lives."""
        shared.used_here()
        if torch.cuda.is_current_stream_capturing():
            self._captured[id(shared)] = shared

    def _tokens(self, x: torch.Tensor, views: Sequence[int], weights: Sequence[Optional[torch.Tensor]]):
        """(slice, its tokens of x), after the checks of a call."""
        shape = (self.B, len(views), self.H, self.W, self.width)
        if x.shape != shape or x.dtype != self.dtype or x.device != self.foreground.device:
            raise ValueError(f"x must be {self.dtype} {list(shape)} on {self.foreground.device} (got {x.dtype} "
                             f"{list(x.shape)} on {x.device})")
        if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, *weights)):
            raise ValueError("the layer has no gradient: call it under torch.no_grad(), or on tensors that require none")
        if _has_tangent((x, *weights)):
            raise ValueError("the layer has no gradient, of forward mode either: call it under torch.inference_mode(), or on "
                             "tensors without tangents")
        s = self.slice(views)
        self._uses(s)
        return s, x.reshape(-1, self.width)[s.index]

    def _attend(self, qkv: torch.Tensor, s: TokenSlice) -> torch.Tensor:
        """Attention [tokens, heads, dim] of the fused projection's rows, whose queries and keys are normed in place."""
        H, Hk, D = self.heads, self.kv_heads, self.dim
        q, k, v = qkv.view(-1, H + 2 * Hk, D).split([H, Hk, Hk], dim=1)
        gc_qk_norm_rope(q, k, self.q_gain, self.k_gain, s.positions, self.table, sections=self.sections,
                        layout=GC_ROPE_HALF, q_out=q, k_out=k)            # where the projection left them
        return gc_attention(q, k, v, s.plan)[0]

    def _spread(self, y: torch.Tensor, x: torch.Tensor, s: TokenSlice) -> torch.Tensor:
        """Tokens in x's shape, zeros on the background."""
        out = torch.zeros(x.shape, dtype=x.dtype, device=x.device)        # (zeros_like keeps a permuted x's order)
        out.view(-1, self.width)[s.index] = y
        return out


class MultiViewAttention(_SlicedAttention):
    """softmax(q k) v of each asset's foreground tokens, with per-head RMS
    norms of queries and keys and rotary positions, between a fused input
    projection and an output projection.  The forward pass only: a call that
    torch would record for a gradient is refused.  One layer may be called
    under several streams and from several threads at the same time.  A call
    on views whose slice is known may be captured into a graph, which may be
    replayed while the layer lives."""

    def __init__(self, pos: torch.Tensor, width: int, heads: int, kv_heads: int, dim: int,
                 dtype: torch.dtype = torch.bfloat16, sections: Optional[Sequence[int]] = None, base: float = 10000.0,
                 generator: Optional[torch.Generator] = None):
        """pos: device float32 [B, N, H, W, 3] position maps (NaN: background).
        sections: columns of the rotation for the view, row and column axes
        (default: the whole head, a quarter of it for the view).  The weights
        are drawn from the generator; load others into w_qkv [width, (heads +
        2 kv_heads) dim], w_out [heads dim, width], q_gain and k_gain [dim]."""
        super().__init__(pos, width, heads, kv_heads, dim, dtype, sections, base)
        rand = lambda *shape: torch.randn(shape, generator=generator, device=pos.device)
        self.w_qkv = (rand(width, (heads + 2 * kv_heads) * dim) / math.sqrt(width)).to(dtype)
        self.w_out = (rand(heads * dim, width) / math.sqrt(heads * dim)).to(dtype)

    def __call__(self, x: torch.Tensor, views: Sequence[int]) -> torch.Tensor:
        """x [B, len(views), H, W, width] of the layer's type -> the layer's
        output on foreground tokens, zeros on the background."""
        s, tokens = self._tokens(x, views, (self.w_qkv, self.w_out, self.q_gain, self.k_gain))
        out = self._attend(tokens @ self.w_qkv, s)
        return self._spread(out.view(-1, self.heads * self.dim) @ self.w_out, x, s)


class MultiViewBlock(_SlicedAttention):
    """A whole block on each asset's foreground tokens x:

      h = x + attention(norm(x)),  y = h + down(act(in(norm(h))))

    with RMS norms, the attention of MultiViewAttention and a feed-forward
    part, gated (act(gate) * value) or not.  With lay_out_in_8_bits() the
    products' operands are 8-bit rows with a scale each.  The forward pass only: a call that
    torch would record for a gradient is refused.  One block may be called under several streams and from several
    threads at the same time.  A call on views whose slice is known may be captured into a graph, which may be replayed
    while the block lives; it goes on with the 8-bit rows that it was captured with."""

    def __init__(self, pos: torch.Tensor, width: int, heads: int, kv_heads: int, dim: int, hidden: int,
                 act: int = GC_ACT_SILU, gated: bool = True, dtype: torch.dtype = torch.bfloat16,
                 sections: Optional[Sequence[int]] = None, base: float = 10000.0, eps: float = 1e-6,
                 generator: Optional[torch.Generator] = None):
        """pos, sections, base: as MultiViewAttention's.  The weights, rows of
        outputs, are drawn from the generator; load others into w_qkv [(heads +
        2 kv_heads) dim, width], w_out [width, heads dim], w_in [hidden, or 2
        hidden: gates and values, width], w_down [width, hidden], the biases
        b_qkv, b_out, b_in, b_down (float32, None: none) and the gains
        attention_gain, feed_gain [width], q_gain, k_gain [dim] (float32)."""
        super().__init__(pos, width, heads, kv_heads, dim, dtype, sections, base)
        self.hidden, self.act, self.gated, self.eps = hidden, act, gated, eps
        dev = pos.device
        rand = lambda n, m: (torch.randn((n, m), generator=generator, device=dev) / math.sqrt(m)).to(dtype)
        self.w_qkv = rand((heads + 2 * kv_heads) * dim, width)
        self.w_out = rand(width, heads * dim)
        self.w_in = rand(2 * hidden if gated else hidden, width)
        self.w_down = rand(width, hidden)
        self.b_qkv = self.b_out = self.b_in = self.b_down = None
        self.attention_gain = torch.ones(width, dtype=torch.float32, device=dev)
        self.feed_gain = torch.ones(width, dtype=torch.float32, device=dev)
        self.eight_bits: Optional[EightBitWeights] = None

    def lay_out_in_8_bits(self) -> None:
        """The products' weights as they are now in 8 bits with a scale a row:
        calls from here on use those, whatever is loaded into w_... later
        (call again after that; calls that have begun go on with the rows that they began
        with).  width, heads * dim and hidden are multiples of 16."""
        for n in (self.width, self.heads * self.dim, self.hidden):
            if n % 16:
                raise ValueError(f"8-bit products need a width, heads * dim and hidden of whole 16 (got {n})")
        stream = torch.cuda.current_stream(self.foreground.device)
        rows = EightBitWeights({name: gc_quantize_rows(getattr(self, name)) for name in ("w_qkv", "w_out", "w_in", "w_down")})
        rows.known_streams.add(stream.cuda_stream)
        stream.synchronize()                                              # any stream may read them from here on
        self.eight_bits = rows

    def _product(self, name: str, rows: Optional[EightBitWeights], x: torch.Tensor, scale: Optional[torch.Tensor] = None,
                 **more) -> torch.Tensor:
        """x (of the layer's type, or 8-bit rows with their scales) times a weight, that of `rows` where there are some."""
        bias = getattr(self, "b" + name[1:])
        if rows is None:
            return gc_linear(x, getattr(self, name), bias, out_dtype=self.dtype, **more)
        if scale is None:
            x, scale = gc_quantize_rows(x)
        w, w_scale = rows[name]
        return gc_linear(x, w, bias, x_scale=scale, w_scale=w_scale, out_dtype=self.dtype, **more)

    def __call__(self, x: torch.Tensor, views: Sequence[int]) -> torch.Tensor:
        """x [B, len(views), H, W, width] of the layer's type -> the block's
        output on foreground tokens, zeros on the background."""
        s, tokens = self._tokens(x, views, (self.w_qkv, self.w_out, self.w_in, self.w_down, self.b_qkv, self.b_out, self.b_in,
                                            self.b_down, self.q_gain, self.k_gain, self.attention_gain, self.feed_gain))
        rows = self.eight_bits                                            # (another thread may lay them out again)
        if rows is not None:
            self._uses(rows)
        normed = torch.float8_e4m3fn if rows is not None else self.dtype
        n, scale, _ = gc_add_rms_norm(tokens, gain=self.attention_gain, eps=self.eps, out_dtype=normed)
        out = self._attend(self._product("w_qkv", rows, n, scale), s)
        out = self._product("w_out", rows, out.view(-1, self.heads * self.dim))
        n, scale, h = gc_add_rms_norm(out, residual=tokens, gain=self.feed_gain, eps=self.eps, out_dtype=normed, total=out)
        m = self._product("w_in", rows, n, scale, act=self.act, gated=self.gated)
        return self._spread(self._product("w_down", rows, m, residual=h, out=h), x, s)
