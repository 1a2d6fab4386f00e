"""The normaliser of a beam search's selection where most of it lies in logits below the collecting threshold, which are summed in float32 batch by batch.

With u = 2^-24, a term exp2(a), a = (x - reference) log2(e) / T <= 0, is off by
  u |a| ln 2    log2(e) / T as a float32            u |a| ln 2    the multiply-add that forms a
  2 u           the exponential, one unit in the last place
and by one u for each float32 addition behind it: 3 (float32) or 7 (bfloat16) along a vector, 4 vectors of a batch, one of a logit behind the last whole vector, at most
12 in all, whatever the number of logits: batches are added in 64 bits.  Together (2 ln 2 |a| + 14) u of the term, and as much of the sum for the share of it that such terms have."""
import math

import numpy as np
import pytest
import torch

from paper_2603_25011_amd.beam import beam_select

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
ROWS = 528           # enough that a row is one segment


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,T", [(1 << 21, 1.0), ((1 << 21) + 7, 0.7), (250002, 2.0), (30522, 1.0)])
def test_one_value_repeated_below_the_threshold(V, T, dtype):
    tops, high = 64, 3.25
    low = (high - torch.linspace(0.25, 12.0, ROWS)).to(dtype).to(DEV)
    x = low[:, None].expand(ROWS, V).contiguous()
    x[:, :4096:64] = high                            # so that every wave of the first batch has some, and they are the threshold
    d = (high - low.double().cpu().numpy()) / T
    below = (V - tops) * np.exp(-d)
    lse = np.log(tops + below)                       # relative to the largest
    s = torch.tensor(lse, dtype=torch.float32, device=DEV)
    got = beam_select(x[:, None], s[:, None], 4, T)
    assert torch.equal(got[2], torch.arange(0, 256, 64, dtype=torch.int32, device=DEV).expand(ROWS, 4))
    off = np.abs(got[0].double().cpu().numpy() - (s.double().cpu().numpy() - lse)[:, None])
    tol = below / (tops + below) * (2 * math.log(2) * d * math.log2(math.e) + 14) * U + 2.0 ** -40
    assert (off <= tol[:, None]).all(), (off / tol[:, None]).max()
