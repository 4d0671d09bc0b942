"""Rotary positions with a time, a height and a width axis.

Argument marshalling for fademem_rope_apply (include/fademem.h): the rotation
of a chunk's queries and keys, and its inverse, which is its gradient.
"""
from __future__ import annotations

import contextlib
import functools
from typing import Optional, Sequence

from . import fademem as fm


def rows_of(t, name: str, dtype, device, heads: int, head_dim: int, rows: int) -> int:
    """Checks a [rows][heads][head_dim] tensor whose heads and elements are
    contiguous (rows may be apart) and returns its elements between rows."""
    if t.dtype != dtype or t.device != device or t.shape != (rows, heads, head_dim):
        raise ValueError(f"{name}: expected a [{rows}][{heads}][{head_dim}] {dtype} tensor on {device}")
    if t.is_contiguous():
        return heads * head_dim
    pitch, head, one = t.stride()
    if (one != 1 and head_dim > 1) or (head != head_dim and heads > 1):
        raise ValueError(f"{name}: heads and elements must be contiguous")
    return pitch if rows > 1 else heads * head_dim


def empty_rows(shape, dtype, device, stream):
    """Memory for the result of a call on `stream` (None: the current one),
    taken from that stream's: what the current stream has let go it may still
    be working on."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


@functools.lru_cache(maxsize=None)
def _turn():
    """Rotary.apply as a step of torch's autograd (made on first use: the package imports torch only in calls)."""
    import torch

    class Turn(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, pos, rotary, inverse):
            pos = pos.clone()  # a step's positions are written over by the next plan
            ctx.save_for_backward(pos)
            ctx.rotary, ctx.inverse = rotary, inverse
            return rotary.apply(x, pos, inverse=inverse)

        @staticmethod
        def backward(ctx, g):
            pos, = ctx.saved_tensors
            g = g.contiguous()
            g = g if g.data_ptr() % 16 == 0 else g.clone()
            return ctx.rotary.apply(g, pos, inverse=not ctx.inverse), None, None, None

    return Turn


class Rotary:
    """A rotation: `pairs` = (time, height, width) pairs of a head, in this
    order from its first pair on (the rest is copied); pair k of an axis with
    P pairs turns by theta^(-k/P) per position.  layout: "interleaved" (pair p
    is elements 2p, 2p+1) or "halves" (p, p + head_dim/2).  `freq`, if given,
    replaces the frequencies (one per pair)."""

    def __init__(self, head_dim: int, pairs: Sequence[int], theta: float = 10000.0, layout: str = "interleaved",
                 freq: Optional[Sequence[float]] = None):
        if layout not in fm.ROPE_LAYOUTS:
            raise ValueError(f"layout must be one of {sorted(fm.ROPE_LAYOUTS)}")
        if len(pairs) != 3:
            raise ValueError("pairs: expected three numbers (time, height, width)")
        self.head_dim, self.pairs, self.layout = int(head_dim), tuple(int(p) for p in pairs), layout
        self.rope = fm.fademem_rope_init(self.head_dim, fm.ROPE_LAYOUTS[layout], *self.pairs, theta)
        if freq is not None:
            if len(freq) != sum(self.pairs):
                raise ValueError(f"freq: expected {sum(self.pairs)} frequencies")
            for i, f in enumerate(freq):
                self.rope.freq[i] = float(f)

    def apply(self, x, pos, out=None, inverse: bool = False, stream=None):
        """x [rows][heads][head_dim] (float32 or bfloat16; rows may be apart,
        as in a joint projection's output) turned to the positions pos, a
        contiguous int32 [rows][3] tensor of (time, height, width).  out may be
        x.  inverse=True turns back: the gradient of apply, which autograd takes
        by itself where x wants one (not into a given `out`)."""
        import torch
        dtype, device = x.dtype, x.device
        if (dtype != torch.bfloat16 and dtype != torch.float32) or x.dim() != 3 or not x.is_cuda:
            raise ValueError("x: expected a [rows][heads][head_dim] float32 or bfloat16 CUDA tensor")
        rows, heads, _ = x.shape
        x_stride = rows_of(x, "x", dtype, device, heads, self.head_dim, rows)
        if pos.dtype != torch.int32 or pos.shape != (rows, 3) or not pos.is_contiguous() or pos.device != device:
            raise ValueError(f"pos: expected a contiguous int32 [{rows}][3] tensor on {device}")
        if torch.is_grad_enabled() and (x.requires_grad or (out is not None and out.requires_grad)):
            if out is not None:
                raise ValueError("out: a result that takes part in autograd cannot be written into given memory")
            with contextlib.nullcontext() if stream is None else torch.cuda.stream(stream):  # the gradient's stream too
                return _turn().apply(x, pos, self, inverse)
        if out is None:
            out, y_stride = empty_rows((rows, heads, self.head_dim), dtype, device, stream), heads * self.head_dim
        else:
            y_stride = rows_of(out, "out", dtype, device, heads, self.head_dim, rows)
        with fm.on_device(device.index):
            fm.fademem_rope_apply(self.rope, fm.FADEMEM_BF16 if dtype == torch.bfloat16 else fm.FADEMEM_F32,
                                  pos.data_ptr(), rows, heads, x.data_ptr(), x_stride, out.data_ptr(), y_stride,
                                  1 if inverse else 0, fm.current_stream() if stream is None else int(stream.cuda_stream))
        return out
