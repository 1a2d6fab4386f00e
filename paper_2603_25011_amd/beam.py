"""A beam search over the head's dense logits: the next beams, and the reordering of what they keep.

    scores, parents, tokens = beam_select(head.logits(H), scores, beams)
    caches = beam_reorder(caches, parents)

Argument checks and marshalling only: all work runs in the HIP library, on the current stream, and there is no CPU path.
"""
from __future__ import annotations

import torch

from . import binding as lsr
from .distill import _aligned, _kind, _ld, _on, _on_gpu, _rows, _scratch


def beam_select(logits: torch.Tensor, scores: torch.Tensor, K: int, temperature: float = 1.0, finished: torch.Tensor | None = None, end_id: int = 0):
    """The K best continuations of every sequence's beams: (scores float32 [B, K] descending, beams int32 [B, K], tokens int32 [B, K]).

    logits [B, beams, V] (float32 or bfloat16), scores [B, beams] the beams' own: a continuation's score is score + log softmax(logits / temperature); equal
    ones come by beam and token.  A logit of -inf excludes a token, a score of -inf a beam (at the first step all but one are alike).  A beam whose
    `finished` [B, beams] is not zero goes on with end_id alone, its score unchanged.  Where there are fewer than K the places behind have score -inf, beam 0
    and end_id.  A beam whose logits hold a NaN or +inf comes first, with scores of NaN."""
    _on_gpu("beam_select", logits, scores, finished)
    kind = _kind(logits, "beam_select", "logits")
    if logits.dim() != 3:
        raise ValueError("beam_select: logits must be [B, beams, V]")
    B, beams, V = logits.shape
    if scores.shape != (B, beams) or (finished is not None and finished.shape != (B, beams)):
        raise ValueError("beam_select: scores and finished must have one value for each beam")
    K = int(K)
    dev = logits.device
    out_scores = torch.empty((B, K), dtype=torch.float32, device=dev)
    out_beams = torch.empty((B, K), dtype=torch.int32, device=dev)
    out_tokens = torch.empty((B, K), dtype=torch.int32, device=dev)
    if B:
        X = _rows(logits.detach().reshape(B * beams, V))
        scores = scores.detach().float().contiguous()
        if finished is not None:
            if finished.dtype not in (torch.bool, torch.uint8):
                finished = finished != 0
            finished = finished.contiguous().view(torch.uint8)
        with _on(dev):
            ws = _scratch(lsr.lsr_beam_select_workspace_bytes(B, beams, V, K), dev)
            lsr.lsr_beam_select(B, beams, V, K, kind, temperature, X, _ld(X), scores, finished, end_id, out_scores, out_beams, out_tokens, ws)
    return out_scores, out_beams, out_tokens


def _layout(x: torch.Tensor):
    """(bytes from sequence to sequence, from beam to beam, from piece to piece, pieces, bytes of a piece) of [B, beams, ...], or None if the rest is not
    pieces of equal length and distance."""
    e = x.element_size()
    if x.is_contiguous():
        row = x.numel() // (x.shape[0] * x.shape[1]) * e
        return x.shape[1] * row, row, row, 1, row
    # dimensions behind the beams, those of one entry left out, neighbours that lie behind each other joined
    dims = []
    for n, st in zip(x.shape[2:], x.stride()[2:]):
        if n == 1:
            continue
        if dims and dims[-1][1] == n * st:
            dims[-1] = (dims[-1][0] * n, st)
        else:
            dims.append((n, st))
    if dims and dims[-1][1] == 1:
        inner = dims.pop()[0]
    else:
        inner = 1
    if len(dims) > 1:
        return None
    pieces, step = dims[0] if dims else (1, inner)
    return x.stride(0) * e, x.stride(1) * e, step * e, pieces, inner * e


def _span(x: torch.Tensor):
    """Addresses from the first byte to behind the last."""
    first = x.data_ptr()
    n = x.numel() if x.is_contiguous() else sum((n - 1) * s for n, s in zip(x.shape, x.stride())) + 1
    return first, first + n * x.element_size()


def _once(x: torch.Tensor) -> bool:
    """Whether no two elements share an address (dimensions nest)."""
    if x.is_contiguous():
        return True
    reach = 0
    for st, n in sorted((st, n) for n, st in zip(x.shape, x.stride()) if n > 1):
        if st <= reach:
            return False
        reach += (n - 1) * st
    return True


def beam_reorder(states, parents: torch.Tensor, out=None):
    """What the beams keep, in the order of their children: new[b, k] = old[b, parents[b, k]] for every tensor [B, beams, ...] of `states` (one, or a list
    of any dtypes, all on one GPU), in one launch for up to 32 of them.  parents [B, K] int32 as beam_select gives them; a parent outside the beams gives zeros.
    `out`: tensors [B, K, ...] to write, whose addresses lie apart from each other's, the states' and the parents'; without it new ones.  Returns a tensor or a list, as
    `states` is one.  Strides are free; a tensor whose [b, m] is not pieces of equal length and distance (a cache of which only part of the length is in use
    is) is copied first, and refused as `out`.  A tensor whose addresses, strides or pieces are odd may have up to 16 GiB to write, in multiples of 2 bytes 32, and so on."""
    one = isinstance(states, torch.Tensor)
    states = [states] if one else list(states)
    if out is not None:
        out = [out] if isinstance(out, torch.Tensor) else list(out)
        if len(out) != len(states):
            raise ValueError("beam_reorder: as many tensors in out as in states")
    if parents.dim() != 2 or parents.dtype != torch.int32:
        raise ValueError("beam_reorder: parents must be an int32 matrix [B, K]")
    if not states:
        return []
    _on_gpu("beam_reorder", parents, *states, *(out or ()))
    B, K = parents.shape
    beams = states[0].shape[1] if states[0].dim() > 1 else 0
    new, table, spans, hold = [], [], [], []
    if out is not None:
        spans.append((*_span(parents), False))
    for i, x in enumerate(states):
        shape = x.shape
        if len(shape) < 2 or shape[0] != B or shape[1] != beams:
            raise ValueError("beam_reorder: every state must be [B, beams, ...]")
        if out is None:
            y = torch.empty((B, K, *shape[2:]), dtype=x.dtype, device=x.device)
        else:
            y = out[i]
            if y.shape != (B, K, *shape[2:]) or y.dtype != x.dtype:
                raise ValueError("beam_reorder: out must be [B, K, ...] of the states' dtypes")
            if y.is_conj() or y.is_neg():
                raise ValueError("beam_reorder: out must hold its values as they are, not conjugated or negated")
        if x.is_conj() or x.is_neg():
            x = x.resolve_conj().resolve_neg()
            hold.append(x)
        new.append(y)
        size = y.numel()
        if not size:
            continue
        if not beams:
            y.zero_()
            continue
        if x.is_contiguous() and y.is_contiguous():
            row = size // (B * K) * x.element_size()
            src, dst = x.data_ptr(), y.data_ptr()
            table.append((src, dst, beams * row, row, row, K * row, row, row, 1, row))
            if out is not None:
                spans.append((dst, dst + B * K * row, True))
                spans.append((src, src + B * beams * row, False))
            continue
        x = x.detach()
        src, dst = _layout(x), _layout(y)
        if dst is None or not _once(y):
            raise ValueError("beam_reorder: out[b, k] must be pieces of equal length and distance")
        if src is not None and src[3:] != dst[3:]:
            # pieces of one side are cut as the other's
            if src[3] == 1 and src[4] == dst[3] * dst[4]:
                src = (*src[:2], dst[4], *dst[3:])
            elif dst[3] == 1 and dst[4] == src[3] * src[4]:
                dst = (*dst[:2], src[4], *src[3:])
            else:
                src = None
        if src is None:
            x = x.contiguous()
            hold.append(x)
            src = _layout(x)
            src = (*src[:2], dst[4], *dst[3:])
        table.append((x.data_ptr(), y.data_ptr(), *src[:3], *dst))
        if out is not None:
            spans.append((*_span(y), True))
            spans.append((*_span(states[i]), False))
    # what is written shares no memory with anything else
    spans.sort()
    end, written = 0, False
    for first, last, writes in spans:
        if first < end and (writes or written):
            raise ValueError("beam_reorder: the addresses of out overlap the states', the parents' or its own")
        if last > end:
            end, written = last, writes
    if table:
        with _on(parents.device):
            lsr.lsr_beam_reorder(B, beams, K, _aligned(parents), table)
    return new[0] if one else new
