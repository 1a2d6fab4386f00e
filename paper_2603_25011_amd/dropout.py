"""Dropout whose mask is never stored: forward and backward draw it from a counter.

Argument checks and marshalling only: the arithmetic runs in the HIP library, on the current stream, and there is no CPU path.
"""
from __future__ import annotations

import torch

from . import binding as lsr
from .distill import _KIND, _kind, _on_gpu


def _draw(x: torch.Tensor, p: float, seed: int, offset: int, state) -> torch.Tensor:
    # (the backward runs in a thread where every call costs more than the kernel: few of them)
    if not x.is_contiguous():
        x = x.contiguous()
    y = torch.empty_like(x)
    n = x.numel()
    if n:
        dev = x.get_device()
        if dev == torch._C._cuda_getDevice():
            lsr.lsr_dropout(n, _KIND[x.dtype], x, y, p, seed, offset, state, torch._C._cuda_getCurrentRawStream(dev))
        else:
            with torch.cuda.device(dev):
                lsr.lsr_dropout(n, _KIND[x.dtype], x, y, p, seed, offset, state)
    return y


class _Dropout(torch.autograd.Function):
    """The same linear map forward and backward, so that its gradients have gradients too."""

    @staticmethod
    def forward(ctx, x, p, seed, offset, state):
        ctx.draw = (p, seed, offset)
        if state is not None:
            ctx.save_for_backward(state)
        return _draw(x, p, seed, offset, state)

    @staticmethod
    def backward(ctx, dy):
        state = ctx.saved_tensors
        f = _Dropout.apply if torch.is_grad_enabled() else _draw
        return f(dy, *ctx.draw, state[0] if state else None), None, None, None, None


def dropout(x: torch.Tensor, p: float, seed: int = 0, offset: int = 0, state: torch.Tensor | None = None) -> torch.Tensor:
    """x (float32 or bfloat16, any shape) times 65536 / (65536 - t) where the element's 16-bit random number is at least t = round(65536 p), else 0.

    The number of element i (in row-major order, whatever the strides) is the (i % 8)-th half word of the Philox4x32-10 block at counter (i // 8,
    offset) with key `seed`: calls with other seeds or offsets draw other masks, the same call draws the same one.  `state`, an int64 tensor
    of two on the same GPU, is added to (seed, offset) when the work runs: a program that captures a step into a graph advances it between replays, and between steps only
    (the backward reads it again; where it was changed before, autograd says so).  While a step is captured no result of an eager call on the same
    tensor may still hold its own autograd graph (autograd would run part of the captured backward on the eager call's stream)."""
    _on_gpu("dropout", x, state)
    _kind(x, "dropout", "x")
    if not 0.0 <= p <= 1.0:
        raise ValueError(f"dropout: p is a probability, not {p}")
    if state is not None and (state.dtype != torch.int64 or state.shape != (2,) or not state.is_contiguous()):
        raise ValueError("dropout: state must be a contiguous int64 tensor of two")
    return _Dropout.apply(x, float(p), int(seed) % (1 << 64), int(offset) % (1 << 64), state)
