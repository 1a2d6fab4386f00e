"""The head's dense logits in 8-bit floating point (e4m3 times a power of two for each block of 128), served and trained.

    head = Fp8Head(W, bias)                       # a matrix held in 8 bits
    logits = head.logits(H)
    logits = fp8_logits(H, W, bias)               # a matrix that is a parameter: differentiable in H, W and bias

Argument checks and marshalling only: all arithmetic runs in the HIP library, on the current stream, and there is no CPU path.
"""
from __future__ import annotations

import functools

import torch

from . import binding as lsr
from .autograd import first_order_only
from .distill import _KIND, Int8Head, _as, _kind, _ld, _on, _on_gpu, _rows, _scratch


def quantize_blocks(X: torch.Tensor, square: bool = False, transposed: bool = False):
    """X [rows, cols] (float32 or bfloat16) in e4m3 blocks with a power of two each: (Q uint8 [rows, cols up to a multiple of 128],
    exps uint8 [blocks of 512 columns, rows, 4]), X[r, c] close to Q[r, c] as e4m3 times 2^(exps[c // 512, r, c // 128 % 4] - 127), Q zero behind cols.
    A block is 1 x 128 of a row, or with `square` 128 x 128.  `transposed`: the same of X transposed (a copy is not made first)."""
    _on_gpu("quantize_blocks", X)
    kind = _kind(X, "quantize_blocks", "X")
    if X.dim() != 2 or X.shape[1] < 1:
        raise ValueError("quantize_blocks: X must be a matrix with at least one column")
    rows, cols = X.shape
    n, m = (cols, rows) if transposed else (rows, cols)
    Q = torch.empty((n, _up(m, 128)), dtype=torch.uint8, device=X.device)
    exps = torch.zeros((_up(m, 512) // 512, n, 4), dtype=torch.uint8, device=X.device)
    if rows:
        X = _rows(X.detach())
        with _on(X.device):
            q, qt = ((None, 0, None), (Q, Q.shape[1], exps))[::1 if transposed else -1]
            lsr.lsr_fp8_quantize(rows, cols, kind, X, _ld(X), square, *q, *qt)
    return Q, exps


@functools.lru_cache(maxsize=256)
def _forward_bytes(N: int, V: int, D: int):
    """(of the workspace, of the matrix transposed by slab, of its exponents)"""
    return lsr.lsr_fp8_forward_workspace_bytes(N, V, D), lsr.lsr_fp8_slab_bytes(D, V), lsr.lsr_fp8_exp_bytes(D, V)


@functools.lru_cache(maxsize=256)
def _backward_bytes(N: int, V: int, D: int, need_h: bool, need_w: bool, need_b: bool) -> int:
    return lsr.lsr_fp8_backward_workspace_bytes(N, V, D, need_h, need_w, need_b)


def _up(n: int, m: int) -> int:
    return (n + m - 1) // m * m


def _bias(who: str, bias, V: int):
    if bias is not None and bias.shape != (V,):
        raise ValueError(f"{who}: bias must have one value for each row of W")
    return None if bias is None else bias.float().contiguous()


def _matmul(H: torch.Tensor, kind: int, D: int, W8: torch.Tensor, exps: torch.Tensor, bias, dtype: torch.dtype) -> torch.Tensor:
    """Logits of rows H [N, D], with the tensors' device current."""
    N, V = H.shape[0], W8.shape[0]
    out = torch.empty((N, V), dtype=dtype, device=H.device)
    ws = _scratch(lsr.lsr_fp8_matmul_workspace_bytes(N, V, D, kind), H.device)
    lsr.lsr_fp8_matmul(N, V, D, kind, _KIND[dtype], H, _ld(H), None, W8, W8.shape[1], exps, bias, out, V, ws)
    return out


class Fp8Head:
    """A head whose matrix is held in e4m3, one power of two for each 128 x 128 of it: half the bytes of bfloat16, products at twice its rate, and
    rows whose values differ much in magnitude keep their small ones (Int8Head has one scale for a whole row)."""

    def __init__(self, W: torch.Tensor, bias: torch.Tensor | None = None):
        self.W8, self.exps = quantize_blocks(W, square=True)
        self.V, self.D = W.shape
        if bias is not None:
            _on_gpu("Fp8Head", W, bias)
            bias = _bias("Fp8Head", bias.detach(), self.V)
        self.bias = bias

    def logits(self, H: torch.Tensor, dtype: torch.dtype = torch.float32) -> torch.Tensor:
        """[..., V] logits of hidden states H [..., D] (float32 or bfloat16), which are held in blocks of 128 within the call.  A row's float32 logits do not depend on
        the rows beside it; bfloat16 ones of few rows (up to 24) are those rounded, of more rows sums of the matrix cores' 8-bit instruction (2e-5 of their norm, then rounded), so that a row's may
        be a rounding apart in a call of few rows and in one of many."""
        _on_gpu("Fp8Head.logits", H, self.W8)
        kind = _kind(H, "Fp8Head.logits", "H")
        if dtype not in _KIND:
            raise TypeError(f"Fp8Head.logits: logits are float32 or bfloat16, not {dtype}")
        if H.shape[-1] != self.D:
            raise ValueError(f"Fp8Head.logits: H has {H.shape[-1]} columns, the matrix {self.D}")
        A = H.detach().reshape(-1, self.D)
        if not A.shape[0]:
            return torch.empty((*H.shape[:-1], self.V), dtype=dtype, device=H.device)
        with _on(H.device):
            return _matmul(_rows(A), kind, self.D, self.W8, self.exps, self.bias, dtype).reshape(*H.shape[:-1], self.V)

    top_logits = Int8Head.top_logits


class _Fp8Logits(torch.autograd.Function):
    """Tensors as the library takes them: H [N, D] and W [V, D] with contiguous rows, bias [V] float32 or None."""

    @staticmethod
    def forward(ctx, H, W, bias, dtype):
        N, D = H.shape
        V = W.shape[0]
        kind = _KIND[H.dtype]
        need_t = ctx.needs_input_grad[0] and N > 0      # dH takes the matrix transposed, exponents behind it: written beside the other from one read
        out = torch.empty((N, V), dtype=dtype, device=H.device)
        Wt = None
        if N:
            ws_bytes, slab_bytes, exp_bytes = _forward_bytes(N, V, D)
            with _on(H.device):
                ws = torch.empty(ws_bytes, dtype=torch.uint8, device=H.device)
                if need_t:
                    Wt = torch.empty(slab_bytes + exp_bytes, dtype=torch.uint8, device=H.device)
                    at = Wt.data_ptr()
                lsr.lsr_fp8_forward(N, V, D, kind, _KIND[dtype], H, _ld(H), W, _ld(W), bias, out, V, *((at, 0, at + slab_bytes) if need_t else (None, 0, None)), ws)
        ctx.shape = (N, V, D, _KIND[dtype], kind)
        ctx.has_bias = bias is not None
        ctx.save_for_backward(H, W, Wt)
        ctx.set_materialize_grads(False)
        return out

    @staticmethod
    def backward(ctx, dY):
        # (this runs in a thread where every call costs more than elsewhere: few of them)
        H, W, Wt = ctx.saved_tensors
        N, V, D = ctx.shape[:3]
        need_h, need_w, need_b = ctx.needs_input_grad[:3]
        need_b = need_b and ctx.has_bias
        dev = H.device
        dH = torch.empty((N, D), dtype=H.dtype, device=dev) if need_h else None
        dW = torch.empty((V, D), dtype=W.dtype, device=dev) if need_w else None
        db = torch.empty((V,), dtype=torch.float32, device=dev) if need_b else None
        if dY is None or not N:
            for g in (dH, dW, db):
                if g is not None:
                    g.zero_()
        elif need_h or need_w or need_b:
            y = _rows(dY)
            turned = (None, 0, None)
            if need_h:
                at = Wt.data_ptr()
                turned = (at, 0, at + _forward_bytes(N, V, D)[1])
            with _on(dev):
                ws = torch.empty(_backward_bytes(N, V, D, need_h, need_w, need_b), dtype=torch.uint8, device=dev)
                lsr.lsr_fp8_backward(*ctx.shape, y, _ld(y), H, _ld(H), *turned, dH, dW, db, ws)
            if torch.is_grad_enabled():
                dH, dW, db = first_order_only("fp8_logits", (dH, dW, db), (H, W, dY))
        return dH, dW, db, None


def fp8_logits(H: torch.Tensor, W: torch.Tensor, bias: torch.Tensor | None = None, dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """[..., V] logits H W^T + bias of hidden states H [..., D] and a matrix W [V, D] (both float32 or both bfloat16), multiplied in 8-bit
    floating point: H in blocks of 1 x 128 along its rows, W in blocks of 128 x 128.  `dtype` is that of the logits (float32 or bfloat16; sums as in
    Fp8Head.logits, those of a gradient by the type that it is stored in).
    Differentiable (once) in H, W and bias, the rounding to 8 bits passed over:  dH = q(dY) q(W),  dW = q(dY)^T q(H) with dY and H in blocks of
    128 tokens,  db = sum of dY.  Gradients come in the parameters' own dtypes.
    Where a step is captured into a graph, no result of an eager call on the same parameters may still hold its own autograd graph (autograd would
    run part of the captured backward on the eager call's stream)."""
    _on_gpu("fp8_logits", H, W, bias)
    if H.dtype != W.dtype or H.dtype not in _KIND:
        raise TypeError("fp8_logits: H and W must both be bfloat16 or both float32")
    if dtype not in _KIND:
        raise TypeError(f"fp8_logits: logits are float32 or bfloat16, not {dtype}")
    if W.dim() != 2 or H.dim() < 1 or H.shape[-1] != W.shape[1] or not W.numel():
        raise ValueError("fp8_logits: H [..., D] and W [V, D] do not fit together")
    if not torch.is_grad_enabled():
        H, W = H.detach(), W.detach()               # (no transposed matrix for a backward that will not come)
    lead = H.shape[:-1]
    out = _Fp8Logits.apply(_rows(_as(H, (-1, W.shape[1]))), _rows(W), _bias("fp8_logits", bias, W.shape[0]), dtype)
    return _as(out, (*lead, W.shape[0]))
