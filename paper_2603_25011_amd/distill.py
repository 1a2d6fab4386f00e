"""Training a head on a teacher's token logits: the teacher's head in 8 bits, its top logits, and the loss with its gradients.

    teacher = Int8Head(W_teacher, bias_teacher)
    values, ids, teacher_lse = teacher.top_logits(H_teacher, K, temperature)
    loss, _ = lsr_distill(H, W, bias, ids, values, teacher_lse, mask, temperature)
    (loss.sum() / mask.sum()).backward()

Argument checks and marshalling only: all arithmetic runs in the HIP library, on the current stream, and there is no CPU path.
"""
from __future__ import annotations

import contextlib
import functools

import torch

from . import binding as lsr
from .autograd import first_order_only

_KIND = {torch.float32: lsr.LSR_F32, torch.bfloat16: lsr.LSR_BF16}


def _kind(t: torch.Tensor, who: str, what: str) -> int:
    if t.dtype not in _KIND:
        raise TypeError(f"{who}: {what} must be float32 or bfloat16, not {t.dtype}")
    return _KIND[t.dtype]


def _on_gpu(who: str, *tensors) -> None:
    """All on one GPU."""
    dev = -1
    for t in tensors:
        if t is not None:
            at = t.get_device()
            if at < 0:
                raise RuntimeError(f"{who}: all tensors must live on the GPU; there is no CPU path")
            if dev not in (-1, at):
                raise RuntimeError(f"{who}: all tensors must live on one GPU")
            dev = at


_HERE = contextlib.nullcontext()


def _on(device):
    """With the tensors' device current, whose stream the work goes to."""
    return _HERE if device.index == torch._C._cuda_getDevice() else torch.cuda.device(device)


@functools.lru_cache(maxsize=256)
def _distill_bytes(shape: tuple, backward: bool) -> int:
    return lsr.lsr_distill_workspace_bytes(*shape, backward)


def _rows(x: torch.Tensor) -> torch.Tensor:
    """A matrix whose rows are contiguous, however far apart they lie."""
    return x if x.stride(1) == 1 and (x.shape[0] <= 1 or x.stride(0) >= x.shape[1]) else x.contiguous()


def _ld(x: torch.Tensor) -> int:
    return x.stride(0) if x.shape[0] > 1 else x.shape[1]


def _scratch(nbytes: int, device) -> torch.Tensor | None:
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def quantize_rows(X: torch.Tensor):
    """Rows of X [rows, cols] (float32 or bfloat16) to 8-bit integers: (Q int8 [rows, cols up to a multiple of 128], scale float32 [rows]),
    X[r, c] close to Q[r, c] scale[r] and Q zero behind cols."""
    _on_gpu("quantize_rows", X)
    kind = _kind(X, "quantize_rows", "X")
    if X.dim() != 2 or X.shape[1] < 1:
        raise ValueError("quantize_rows: X must be a matrix with at least one column")
    rows, cols = X.shape
    pitch = lsr.lsr_int8_row_bytes(cols)
    if not pitch:
        raise ValueError(f"quantize_rows: rows of {cols} values are longer than the library takes")
    Q = torch.empty((rows, pitch), dtype=torch.int8, device=X.device)
    scale = torch.empty((rows,), dtype=torch.float32, device=X.device)
    if rows:
        X = _rows(X.detach())
        with _on(X.device):
            lsr.lsr_quantize_rows(rows, cols, kind, X, _ld(X), Q, pitch, scale)
    return Q, scale


def top_logits(X: torch.Tensor, K: int, temperature: float = 1.0):
    """The K largest of each row of X [rows, V]: (values float32 [rows, K] in descending order, ids int32 [rows, K], equal values by ascending
    id, lse float32 [rows] = log sum exp(X / temperature))."""
    _on_gpu("top_logits", X)
    kind = _kind(X, "top_logits", "X")
    if X.dim() != 2:
        raise ValueError("top_logits: X must be a matrix")
    rows, V = X.shape
    K = int(K)
    values = torch.empty((rows, K), dtype=torch.float32, device=X.device)
    ids = torch.empty((rows, K), dtype=torch.int32, device=X.device)
    lse = torch.empty((rows,), dtype=torch.float32, device=X.device)
    if rows:
        X = _rows(X.detach())
        with _on(X.device):
            ws = _scratch(lsr.lsr_top_logits_workspace_bytes(rows, V, K), X.device)
            lsr.lsr_top_logits(rows, V, K, kind, temperature, X, _ld(X), values, ids, lse, ws)
    return values, ids, lse


class Int8Head:
    """A head whose matrix is held in 8 bits, one scale for each vocabulary entry (a teacher, or a head that is served): half the bytes of
    bfloat16, and products at twice its rate."""

    def __init__(self, W: torch.Tensor, bias: torch.Tensor | None = None):
        self.W8, self.w_scale = quantize_rows(W)
        self.V, self.D = W.shape
        if bias is not None:
            _on_gpu("Int8Head", W, bias)
            if bias.shape != (self.V,):
                raise ValueError("Int8Head: bias must have one value for each row of W")
            bias = bias.detach().float().contiguous()
        self.bias = bias

    def logits(self, H: torch.Tensor, dtype: torch.dtype = torch.float32) -> torch.Tensor:
        """[..., V] logits of hidden states H [..., D] (float32 or bfloat16), which are quantised by row within the call."""
        _on_gpu("Int8Head.logits", H, self.W8)
        kind = _kind(H, "Int8Head.logits", "H")
        if dtype not in _KIND:
            raise TypeError(f"Int8Head.logits: logits are float32 or bfloat16, not {dtype}")
        if H.shape[-1] != self.D:
            raise ValueError(f"Int8Head.logits: H has {H.shape[-1]} columns, the matrix {self.D}")
        A = H.detach().reshape(-1, self.D)
        N = A.shape[0]
        out = torch.empty((N, self.V), dtype=dtype, device=H.device)
        if N:
            A = _rows(A)
            with _on(H.device):
                ws = _scratch(lsr.lsr_int8_matmul_workspace_bytes(N, self.V, self.D, kind), H.device)
                lsr.lsr_int8_matmul(N, self.V, self.D, kind, _KIND[dtype], A, _ld(A), None, self.W8, self.W8.stride(0), self.w_scale, self.bias,
                                    out, self.V, ws)
        return out.reshape(*H.shape[:-1], self.V)

    def top_logits(self, H: torch.Tensor, K: int, temperature: float = 1.0, max_logits: int = 1 << 28):
        """The K largest logits of every row of H [..., D], their ids and the row's lse (see top_logits), shapes [..., K], [..., K], [...].
        The logits are formed for a block of rows at a time, at most max_logits of them (or one row's)."""
        lead = H.shape[:-1]
        A = H.reshape(-1, H.shape[-1])
        step = max(1, max_logits // self.V)
        parts = [top_logits(self.logits(a), K, temperature) for a in A.split(step)]
        values, ids, lse = (torch.cat(p) if len(p) > 1 else p[0] for p in zip(*parts))
        return values.reshape(*lead, K), ids.reshape(*lead, K), lse.reshape(lead)


class _LsrDistill(torch.autograd.Function):
    """Tensors as the library takes them: what autograd saves are then the inputs themselves, with their graphs."""

    @staticmethod
    def forward(ctx, H, W, bias, ids, logits, teacher_lse, mask, temperature):
        N, D = H.shape
        ctx.shape = (N, D, W.shape[0], ids.shape[1], _KIND[H.dtype], temperature)
        loss = torch.empty((N,), dtype=torch.float32, device=H.device)
        lse = torch.empty((N,), dtype=torch.float32, device=H.device)
        if N:
            with _on(H.device):
                ws = _scratch(_distill_bytes(ctx.shape, False), H.device)
                lsr.lsr_distill_forward(*ctx.shape, H, W, bias, ids, logits, teacher_lse, mask, loss, lse, ws)
        ctx.save_for_backward(H, W, bias, ids, logits, teacher_lse, mask, lse)
        ctx.mark_non_differentiable(lse)
        ctx.set_materialize_grads(False)
        return loss, lse

    @staticmethod
    def backward(ctx, dloss, _dlse):
        H, W, bias, ids, logits, teacher_lse, mask, lse = ctx.saved_tensors
        need_h, need_w, need_b = ctx.needs_input_grad[:3]
        dev = H.device
        dH = torch.empty_like(H) if need_h else None
        dW = torch.empty_like(W) if need_w else None
        db = torch.empty_like(bias) if need_b else None
        if dloss is None or not ctx.shape[0]:
            for g in (dH, dW, db):
                if g is not None:
                    g.zero_()
        elif need_h or need_w or need_b:
            with _on(dev):
                ws = _scratch(_distill_bytes(ctx.shape, True), dev)
                lsr.lsr_distill_backward(*ctx.shape, H, W, bias, ids, logits, teacher_lse, mask, lse, _aligned(dloss.detach()), dH, dW, db, ws)
            dH, dW, db = first_order_only("lsr_distill", (dH, dW, db), (H, W, bias, dloss))
        return dH, dW, db, None, None, None, None, None


def _as(t: torch.Tensor, shape: tuple) -> torch.Tensor:
    return t if t.dim() == len(shape) else t.reshape(shape)


def _aligned(t: torch.Tensor) -> torch.Tensor:
    """Contiguous and on a 16-byte boundary, as the library takes it (a view into another tensor may be neither)."""
    t = t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


def lsr_distill(H: torch.Tensor, W: torch.Tensor, bias: torch.Tensor, teacher_ids: torch.Tensor, teacher_logits: torch.Tensor,
                teacher_lse: torch.Tensor | None = None, mask: torch.Tensor | None = None, temperature: float = 1.0):
    """Distillation loss of the head (W [V, D], bias [V]) at hidden states H [..., D] against a teacher's K top logits:

        loss = sum_j p_j (log p_j - log softmax((H W^T + bias) / temperature)[teacher_ids_j]),  p_j = exp(teacher_logits_j / temperature - L)

    L is teacher_lse [...] (log sum exp(logits / temperature) over the teacher's whole vocabulary, as top_logits returns it) or, without it, the same
    over the K entries.  Rows whose mask [...] is zero count nothing; an id outside the vocabulary or a logit of -inf is padding.
    Returns (loss float32 [...], lse float32 [...]): lse is the logarithm of the student's normaliser, not differentiable.
    Differentiable (once) in H, W and bias; gradients come in the parameters' own dtypes.  The N x V logits are never stored."""
    _on_gpu("lsr_distill", H, W, bias, teacher_ids, teacher_logits, teacher_lse, mask)
    if H.dtype != W.dtype or H.dtype not in _KIND:
        raise TypeError("lsr_distill: H and W must both be bfloat16 or both float32")
    if teacher_ids.dtype not in (torch.int32, torch.int64):
        raise TypeError("lsr_distill: teacher_ids must be whole numbers of 32 or 64 bits")
    lead, D = H.shape[:-1], H.shape[-1]
    V, K = W.shape[0], teacher_ids.shape[-1]
    if W.shape != (V, D) or bias.shape != (V,) or teacher_ids.shape != (*lead, K) or teacher_logits.shape != teacher_ids.shape:
        raise ValueError("lsr_distill: H [..., D], W [V, D], bias [V], teacher_ids and teacher_logits [..., K] do not fit together")
    if (teacher_lse is not None and teacher_lse.shape != lead) or (mask is not None and mask.shape != lead):
        raise ValueError("lsr_distill: teacher_lse and mask must have one value for each row of H")
    ids = teacher_ids
    if ids.dtype == torch.int64:
        # an id that 32 bits do not hold is padding like any other outside the vocabulary
        ids = torch.where((ids >= 0) & (ids < V), ids, -1).to(torch.int32)
    ids, logits = _aligned(_as(ids, (-1, K))), _aligned(_as(teacher_logits.float(), (-1, K)))
    if teacher_lse is not None:
        teacher_lse = _aligned(_as(teacher_lse.float(), (-1,)))
    if mask is not None:
        # the library takes any non-zero byte for a row that counts
        if mask.dtype not in (torch.bool, torch.uint8):
            mask = mask != 0
        mask = _aligned(_as(mask, (-1,))).view(torch.uint8)
    loss, lse = _LsrDistill.apply(_aligned(_as(H, (-1, D))), _aligned(W), _aligned(bias.float()), ids, logits, teacher_lse, mask, float(temperature))
    return _as(loss, lead), _as(lse, lead)
