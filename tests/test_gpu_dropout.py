"""Dropout from a counter on the GPU: masks bit for bit those of the definition, products one float32 product and one rounding."""
import numpy as np
import pytest
import torch

from oracle import dropout_oracle as orc
from paper_2603_25011_amd import binding
from paper_2603_25011_amd import dropout as module
from paper_2603_25011_amd.dropout import dropout

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def host(t):
    return t.detach().double().cpu().numpy()


def want_of(x, p, seed, offset):
    mask, factor = orc.keep(x.size, p, seed, offset)
    return np.where(mask.reshape(x.shape), x * factor, 0.0)


def check(got, x, p, seed, offset, dtype):
    want = want_of(host(x), p, seed, offset)
    got = host(got)
    assert np.array_equal(got == 0, want == 0)
    # the factor and the product are rounded to float32, the result to its type
    step = 2 * U + (2.0 ** -8 if dtype == "bf16" else U)
    assert (np.abs(got - want) <= step * 1.01 * np.abs(want)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,p,seed,offset", [((1,), 0.5, 0, 0), ((7,), 0.1, 1, 2), ((3, 5, 9), 0.3, 2 ** 63 + 5, 2 ** 40 + 1), ((64, 33), 0.9, -1, 2 ** 64 - 1), ((8,), 0.0, 3, 4),
                                                 ((2055,), 0.15, 12345678901234, 77), ((40, 8), 1.0, 5, 6), ((41,), 2.0 ** -17, 1, 1), ((41,), 1 - 2.0 ** -16, 1, 1)])
def test_forward_and_backward(shape, p, seed, offset, dtype):
    gen = torch.Generator().manual_seed(len(shape))
    x = (torch.rand(shape, generator=gen) + 0.5).to(TYPES[dtype]).to(DEV).requires_grad_(True)
    dy = (torch.rand(shape, generator=gen) + 0.5).to(TYPES[dtype]).to(DEV)
    y = dropout(x, p, seed, offset)
    assert y.dtype == x.dtype and y.shape == x.shape
    check(y, x, p, seed, offset, dtype)
    dx, = torch.autograd.grad(y, x, dy)
    check(dx, dy, p, seed, offset, dtype)


def test_the_mask_goes_by_the_index_whatever_the_strides():
    x = torch.rand(6, 5, 16, device=DEV) + 0.5
    for v in (x[:, 1:], x.transpose(0, 2), x[..., ::2], x[1:].reshape(-1)[3:], x[:1].expand(4, 5, 16), x.bfloat16().reshape(-1)[1:]):
        assert torch.equal(dropout(v, 0.4, 9, 9), dropout(v.contiguous().clone(), 0.4, 9, 9))
    v = x.transpose(0, 2).detach().requires_grad_(True)
    dy = torch.rand(5, 6, 16, device=DEV).permute(2, 0, 1)
    dx, = torch.autograd.grad(dropout(v, 0.4, 9, 9), v, dy)
    assert torch.equal(dx, dropout(dy.contiguous(), 0.4, 9, 9))


def test_other_seeds_and_offsets_draw_other_masks():
    x = torch.ones(1 << 16, device=DEV)
    masks = [dropout(x, 0.5, s, o) != 0 for s, o in ((1, 0), (2, 0), (1, 1), (1, 1 << 32), (1 << 32, 0), (1 + (1 << 32), 0))]
    for i in range(len(masks)):
        # halves of each: 2^16 independent bits, 6 standard deviations
        assert abs(masks[i].float().mean().item() - 0.5) <= 6 * 0.5 / 256
        for j in range(i):
            assert abs((masks[i] == masks[j]).float().mean().item() - 0.5) <= 6 * 0.5 / 256
    assert torch.equal(dropout(x, 0.5, 1, 0) != 0, masks[0])


def test_what_is_dropped_is_zero_whatever_it_was():
    x = torch.full((4096,), float("nan"), device=DEV)
    x[::2] = float("inf")
    y = dropout(x, 0.5, 3)
    mask, _ = orc.keep(4096, 0.5, 3, 0)
    y = y.cpu().numpy()
    assert (y[~mask] == 0).all() and not np.signbit(y[~mask]).any() and not np.isfinite(y[mask]).any()


def test_state_on_the_device_and_replays():
    x = (torch.rand(3000, device=DEV) + 0.5).requires_grad_(True)
    dy = torch.rand(3000, device=DEV) + 0.5
    state = torch.tensor([5, 7], dtype=torch.int64, device=DEV)
    y = dropout(x, 0.3, 10, 20, state)
    assert torch.equal(y, dropout(x, 0.3, 15, 27))
    assert torch.equal(torch.autograd.grad(y, x, dy)[0], dropout(dy, 0.3, 15, 27))
    minus = torch.tensor([-6, -21], dtype=torch.int64, device=DEV)
    assert torch.equal(dropout(x, 0.3, 5, 20, minus), dropout(x, 0.3, -1, -1))
    # advanced before the backward: said, not answered with another mask
    y = dropout(x, 0.3, 10, 20, state)
    state.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        torch.autograd.grad(y, x, dy)
    # a captured step draws new numbers at every replay
    leaf = x.detach().clone().requires_grad_(True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(dropout(leaf, 0.3, 1, 2, state), leaf, dy)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = dropout(leaf, 0.3, 1, 2, state)
        dx, = torch.autograd.grad(y, leaf, dy)
    seen = []
    for k in range(4):
        state.copy_(torch.tensor([k, 3 * k], device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, dropout(x.detach(), 0.3, 1 + k, 2 + 3 * k)) and torch.equal(dx, dropout(dy, 0.3, 1 + k, 2 + 3 * k))
        seen.append(y.detach().clone())
    assert not any(torch.equal(seen[0], s) for s in seen[1:])


def test_gradients_of_gradients_and_in_place():
    x = torch.rand(100, device=DEV, dtype=torch.float32).requires_grad_(True)
    dy = torch.rand(100, device=DEV).requires_grad_(True)
    dx, = torch.autograd.grad(dropout(x, 0.5, 1), x, dy, create_graph=True)
    w = torch.rand(100, device=DEV)
    assert torch.equal(torch.autograd.grad(dx, dy, w)[0], dropout(w, 0.5, 1))
    y = x.detach().clone()
    binding.lsr_dropout(100, 0, y, y, 0.5, 1, 0, None)
    assert torch.equal(y, dropout(x.detach(), 0.5, 1))


def test_indices_beyond_32_bits():
    n = (1 << 32) + 11
    x = torch.ones(n, dtype=torch.bfloat16, device=DEV)
    y = dropout(x, 0.5, 21, 22)
    for first in (0, (1 << 31) - 4, (1 << 32) - 5, n - 16):
        mask, _ = orc.keep(16, 0.5, 21, 22, first)
        assert np.array_equal((y[first:first + 16] != 0).cpu().numpy()[: n - first], mask[: n - first])


def test_nothing_and_refusals():
    assert dropout(torch.zeros(0, 5, device=DEV), 0.5, 1).shape == (0, 5)
    x = torch.ones(8, device=DEV)
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(ValueError):
            dropout(x, p, 1)
    for state in (torch.zeros(2, device=DEV), torch.zeros(3, dtype=torch.int64, device=DEV), torch.zeros(4, dtype=torch.int64, device=DEV)[::2]):
        with pytest.raises(ValueError):
            dropout(x, 0.5, 1, 0, state)
    with pytest.raises(TypeError):
        dropout(x.half(), 0.5, 1)
    with pytest.raises(RuntimeError):
        dropout(x, 0.5, 1, 0, torch.zeros(2, dtype=torch.int64))
    assert module.dropout is dropout
