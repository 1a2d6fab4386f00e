"""A beam search's selection over logits that hold NaN where a batch of them passes the list: the beam comes first with scores of NaN and its K largest logits that are
numbers, then the end.  Tokens and beams are compared exactly with the float64 definition's, and repeat from call to call."""
import math

import pytest
import torch

from tests.test_gpu_beam import DEV, TYPES, check

pytestmark = pytest.mark.gpu
V = 25003            # of one segment: seven batches of float32 logits, four of bfloat16, and three logits behind the last whole vector
EMPTY = 1000         # sequences of no continuation beside them, so that a row is one segment


def rows_of(gen, dtype, K):
    """Rows of more logits at the threshold than the list holds, with NaN among the first logits, among later ones or behind the last whole vector."""
    t = torch.arange(V)
    lowest = torch.finfo(TYPES[dtype]).min
    masked = torch.full((V,), lowest)
    masked[torch.randperm(V, generator=gen)[:300]] = torch.randn(300, generator=gen)
    kinds = [torch.zeros(V), (torch.rand(V, generator=gen) < 0.5).float(), t * 1e-3, t // 5000 * 1.0, masked]
    out = []
    for x in kinds:
        places = [(first, n) for first in (0, 16384) for n in sorted({1, max(K - 1, 1), K, K + 1, 64, 600})]
        for first, n in places:
            y = x.clone()
            y[first + torch.randperm(4096, generator=gen)[:n]] = math.nan
            out.append(y)
        for n in (1, 3):
            y = x.clone()
            y[-n:] = math.nan
            out.append(y)
        y = x.clone()
        y[3:-3] = math.nan                  # six numbers in all
        out.append(y)
    y = masked.clone()
    y[y > lowest] = math.nan                # all that is not masked
    out.append(y)
    return torch.stack(out).to(TYPES[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [1, 4, 16, 128])
def test_nan_in_batches_that_pass_the_list(K, dtype):
    gen = torch.Generator().manual_seed(K)
    rows = rows_of(gen, dtype, K)
    n = rows.shape[0]
    x = torch.zeros(n + EMPTY, 1, V, dtype=TYPES[dtype], device=DEV)
    x[:n, 0] = rows.to(DEV)
    s = torch.full((n + EMPTY, 1), -math.inf, device=DEV)
    s[:n] = 0.0
    got = check(x, s, K, 1.0, None, 7)
    assert got[0][:n].isnan().all() and (got[2] >= 0).all() and (got[2] < V).all()
    # cut into segments: the same beams and tokens
    few = check(x[:n], s[:n], K, 1.0, None, 7)
    assert torch.equal(few[1], got[1][:n]) and torch.equal(few[2], got[2][:n])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [1, 2, 16])
@pytest.mark.parametrize("width", [65, 129, 131, 257, 515, 1031])
def test_nan_in_all_logits_of_a_thread(width, K, dtype):
    """The first vector and the logits behind the last whole one, which one thread has."""
    gen = torch.Generator().manual_seed(width)
    each = 128 // torch.finfo(TYPES[dtype]).bits
    tail = width % each
    x = torch.randn(24, 1, width, generator=gen).to(TYPES[dtype])
    for b in range(x.shape[0]):
        threads = torch.arange(1 + b % max(tail, 1))         # whose tail logit is NaN, and all that they have of whole vectors
        for i in threads.tolist():
            for first in range(i * each, width - tail, 256 * each):
                x[b, 0, first:first + each] = math.nan
            if tail:
                x[b, 0, width - tail + i] = math.nan
    x = x.to(DEV)
    s = torch.zeros(24, 1, device=DEV)
    got = check(x, s, K, 1.0, None, 3)
    assert (got[2] >= 0).all() and (got[2] < width).all()
