"""The head in 8-bit floating point where arrays hold more than 2^32 elements: results in either type, few rows far apart, logits and gradients of a training step, quantised
forms.  Values are few and small whole numbers, so that every result is exact."""
import numpy as np
import pytest
import torch

import paper_2603_25011_amd as lsr
from paper_2603_25011_amd import binding, fp8

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KIND = {torch.float32: lsr.LSR_F32, torch.bfloat16: lsr.LSR_BF16}
N, V = 1100, 1 << 22                         # N V is 2^32 at row 1024


def ones(rows):
    """e4m3 ones [rows, 128] with exponents of their own: row r stands for 2^(r % 3)."""
    e = torch.zeros((1, rows, 4), dtype=torch.uint8, device=DEV)
    e[0, :, 0] = 127 + torch.arange(rows, device=DEV) % 3
    return torch.full((rows, 128), 0x38, dtype=torch.uint8, device=DEV), e


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_results(dtype):
    a, ea = ones(N)
    w = torch.zeros((V, 128), dtype=torch.uint8, device=DEV)
    ew = torch.full((1, V, 4), 127, dtype=torch.uint8, device=DEV)
    at = torch.tensor([0, 1, 255, 256, (1 << 21) - 1, 1 << 21, V - 2, V - 1], device=DEV)
    w[at] = 0x38
    ew[0, V - 1, 0] = 128
    y = torch.full((N, V), 7.0, dtype=dtype, device=DEV)
    binding.lsr_fp8_matmul(N, V, 128, lsr.LSR_E4M3, KIND[dtype], a, 128, ea, w, 128, ew, None, y, V, None)
    want = (128.0 * 2.0 ** (torch.arange(N, device=DEV) % 3))[:, None].expand(N, len(at)).clone()
    want[:, -1] *= 2
    assert torch.equal(y[:, at].float(), want) and y.count_nonzero().item() == want.numel()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [20, 40])
def test_rows_far_apart(rows, dtype):
    ldo = (1 << 32) // (rows - 2) // 8 * 8
    assert (rows - 1) * ldo > 1 << 32
    a, ea = ones(rows)
    w, ew = ones(300)
    y = torch.full(((rows - 1) * ldo + 300,), 7.0, dtype=dtype, device=DEV)
    binding.lsr_fp8_matmul(rows, 300, 128, lsr.LSR_E4M3, KIND[dtype], a, 128, ea, w, 128, ew, None, y, ldo, None)
    got = y.as_strided((rows, 300), (ldo, 1))
    r, v = torch.arange(rows, device=DEV) % 3, torch.arange(300, device=DEV) % 3
    assert torch.equal(got.float(), 128.0 * 2.0 ** (r[:, None] + v))
    got.fill_(7.0)
    assert (y == 7).all()


def places(gen):
    """Some of the N x V, their corners and what lies on either side of the 2^31st and 2^32nd among them, none twice."""
    flat = torch.randint(0, N * V, (1500,), generator=gen)
    edge = torch.tensor([0, V - 1, 2 ** 31 - 1, 2 ** 31, 2 ** 32 - 1, 2 ** 32, 2 ** 32 + 5, N * V - V, N * V - 1])
    flat = torch.unique(torch.cat([flat, edge])).to(DEV)
    return flat // V, flat % V


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_training_step(dtype):
    gen = torch.Generator().manual_seed(1)
    D = 8

    def small(*shape):
        return torch.randint(-4, 5, shape, generator=gen).to(dtype).to(DEV)
    H, W, bias = small(N, D).requires_grad_(True), small(V, D).requires_grad_(True), torch.zeros(V, device=DEV).requires_grad_(True)
    n, v = places(gen)
    g = (torch.randint(0, 2, n.shape, generator=gen) * 2 - 1).to(DEV)
    y = fp8.fp8_logits(H, W, bias, dtype)
    some = torch.cat([v[:200], v[-200:]])
    with torch.no_grad():
        h, w = H.double(), W.double()
        assert torch.equal(y[:, some].double(), h @ w[some].t().contiguous())
    dY = torch.zeros((N, V), dtype=dtype, device=DEV)
    dY[n, v] = g.to(dtype)
    dH, dW, db = torch.autograd.grad(y, (H, W, bias), dY)
    with torch.no_grad():
        g = g.double()
        assert torch.equal(dH.double(), torch.zeros_like(h).index_add_(0, n, w[v] * g[:, None]))
        assert torch.equal(dW.double(), torch.zeros_like(w).index_add_(0, v, h[n] * g[:, None]))
        assert torch.equal(db.double(), torch.zeros(V, dtype=torch.float64, device=DEV).index_add_(0, v, g))


@pytest.mark.parametrize("transposed", [False, True])
def test_quantised_forms(transposed):
    gen = torch.Generator().manual_seed(2)
    n, v = places(gen)
    x = torch.zeros((N, V), dtype=torch.bfloat16, device=DEV)
    x[n, v] = 1.0
    q, e = fp8.quantize_blocks(x, False, transposed)
    r, c = (v, n) if transposed else (n, v)
    # one is 256 times 2^-8
    assert (q[r, c] == 0x78).all() and q.count_nonzero().item() == len(n)
    assert (e[c // 512, r, c // 128 % 4] == 119).all()
    assert e.count_nonzero().item() == len(np.unique((r * (1 << 22) + c // 128).cpu().numpy()))
