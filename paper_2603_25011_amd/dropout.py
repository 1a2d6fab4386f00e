"""Dropout whose mask is never stored: forward and backward draw it from a counter.

Argument checks and marshalling only: the arithmetic runs in the HIP library, on the current stream, and there is no CPU path.
"""
from __future__ import annotations

import torch

from . import binding as lsr
from .distill import _kind, _on, _on_gpu


class _Dropout(torch.autograd.Function):
    """The same linear map forward and backward, so that its gradients have gradients too."""

    @staticmethod
    def forward(ctx, x, p, seed, offset, state):
        ctx.draw = (p, seed, offset)
        ctx.save_for_backward(state)
        y = torch.empty_like(x, memory_format=torch.contiguous_format)
        if x.numel():
            x = x.contiguous()
            with _on(x.device):
                lsr.lsr_dropout(x.numel(), _kind(x, "dropout", "x"), x, y, p, seed, offset, state)
        return y

    @staticmethod
    def backward(ctx, dy):
        return _Dropout.apply(dy, *ctx.draw, *ctx.saved_tensors), None, None, None, None


def dropout(x: torch.Tensor, p: float, seed: int = 0, offset: int = 0, state: torch.Tensor | None = None) -> torch.Tensor:
    """x (float32 or bfloat16, any shape) times 65536 / (65536 - t) where the element's 16-bit random number is at least t = round(65536 p), else 0.

    The number of element i (in row-major order, whatever the strides) is the (i % 8)-th half word of the Philox4x32-10 block at counter (i // 8,
    offset) with key `seed`: calls with other seeds or offsets draw other masks, the same call draws the same one.  `state`, an int64 tensor
    of two on the same GPU, is added to (seed, offset) when the work runs: a program that captures a step into a graph advances it between replays, and between steps only
    (the backward reads it again; where it was changed before, autograd says so)."""
    _on_gpu("dropout", x, state)
    _kind(x, "dropout", "x")
    if not 0.0 <= p <= 1.0:
        raise ValueError(f"dropout: p is a probability, not {p}")
    if state is not None and (state.dtype != torch.int64 or state.shape != (2,) or not state.is_contiguous()):
        raise ValueError("dropout: state must be a contiguous int64 tensor of two")
    return _Dropout.apply(x, float(p), int(seed), int(offset), state)
