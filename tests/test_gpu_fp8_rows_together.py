"""What a row's logits in 8-bit floating point depend on: not on the rows beside it, in float32; in bfloat16 on whether there are few or many (float32 sums of few rows, the
matrix cores' 8-bit sums of many), within what either may be off."""
import numpy as np
import pytest
import torch

from oracle import fp8_oracle as orc
from paper_2603_25011_amd import fp8

from tests.test_gpu_fp8 import host, tolerance, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,K", [(300, 100), (700, 768), (515, 1024), (300, 4000)])
def test_rows_by_themselves_and_among_others(V, K, dtype):
    gen = torch.Generator().manual_seed(V + K)
    h, w = values(gen, (300, K), dtype, 0.5), values(gen, (V, K), dtype, 0.5)
    head = fp8.Fp8Head(w, torch.randn(V, generator=gen).to(w.device))
    together = head.logits(h)
    for n in (1, 2, 9, 16, 24, 25, 32, 33, 64, 129):
        assert torch.equal(head.logits(h[:n]), together[:n]), n
        assert torch.equal(fp8.fp8_logits(h[-n:], w, head.bias), together[-n:]), n
    many, one = head.logits(h, torch.bfloat16), head.logits(h[:1], torch.bfloat16)
    for n in (2, 24, 25, 33, 129, 300):
        got = head.logits(h[:n], torch.bfloat16)
        assert torch.equal(got, many[:n]) or torch.equal(got, together[:n].bfloat16()), n
        assert n < 25 or torch.equal(got, many[:n]), n
    assert torch.equal(one, together[:1].bfloat16())
    A, W = orc.blocks(host(h), 1, 128)[0], orc.blocks(host(w), 128, 128)[0]
    want = A @ W.T + host(head.bias)
    assert (np.abs(host(many) - host(together)) <= tolerance(A, W, want, "bf16", host(head.bias)) + tolerance(A, W, want, "f32", host(head.bias))).all()
