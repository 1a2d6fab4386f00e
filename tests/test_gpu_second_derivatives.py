"""The library's gradients come without a graph: a second derivative through them raises, it is not left out."""
import pytest
import torch

from paper_2603_25011_amd import distill
from paper_2603_25011_amd.autograd import lsr_head
from tests import test_gpu_dense_logits as base

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def penalised(loss, by, of, grad_outputs=None):
    """The loss plus a penalty on its gradient: what a caller would differentiate."""
    g, = torch.autograd.grad(loss, of, grad_outputs, create_graph=True, retain_graph=True)
    return g, by + g.float().pow(2).sum()


@pytest.mark.parametrize("N,dtype", [(20, "bf16"), (300, "f32")])
def test_distill_second_derivatives_raise(N, dtype):
    H, W, bias, ids, logits, L, _, T, dloss = base.distill_case(N, 64, 600, 5, dtype, 41)
    rest = (base.dev(ids), base.dev(logits), base.dev(L), None, T)
    args = [t.to(DEV).requires_grad_(True) for t in (H, W, bias)]
    for of in args:
        loss, _ = distill.lsr_distill(*args, *rest)
        plain, = torch.autograd.grad(loss.sum(), of, retain_graph=True)
        g, total = penalised(loss.sum(), (args[0].float() ** 2).sum(), of)
        assert torch.equal(g, plain)                    # the first derivative is what it is without a graph
        with pytest.raises(RuntimeError, match="lsr_distill"):
            total.backward(retain_graph=True)
        for to in args:                                 # towards either of the inputs
            with pytest.raises(RuntimeError, match="lsr_distill"):
                torch.autograd.grad(total, to, retain_graph=True)
    # a graph that nobody goes through stops nobody
    for a in args:
        a.grad = None
    distill.lsr_distill(*args, *rest)[0].sum().backward(create_graph=True)
    first = [a.grad.detach().clone() for a in args]
    assert torch.equal(first[0], torch.autograd.grad(distill.lsr_distill(*args, *rest)[0].sum(), args[0])[0])


def test_distill_second_derivatives_raise_through_copies_and_weights():
    H, W, bias, ids, logits, L, _, T, dloss = base.distill_case(48, 64, 600, 5, "f32", 42)
    wide = torch.zeros(48, 70, device=DEV)
    wide[:, 3:67] = H.to(DEV)
    wide.requires_grad_(True)
    Wt = W.to(DEV).t().contiguous().requires_grad_(True)
    b = bias.to(DEV).double().requires_grad_(True)
    rest = (base.dev(ids).reshape(6, 8, 5), base.dev(logits).reshape(6, 8, 5), base.dev(L).reshape(6, 8), None, T)
    weight = base.dev(dloss).reshape(6, 8).requires_grad_(True)
    for of in (wide, Wt, b):
        loss, lse = distill.lsr_distill(wide[:, 3:67].reshape(6, 8, 64), Wt.t(), b, *rest)
        assert loss.shape == lse.shape == (6, 8) and not lse.requires_grad
        g, total = penalised(loss, (wide ** 2).sum() + (Wt ** 2).sum() + (b ** 2).sum().float(), of, weight)
        assert g.shape == of.shape and g.dtype == of.dtype
        for to in (wide, Wt, b, weight):
            with pytest.raises(RuntimeError, match="lsr_distill"):
                torch.autograd.grad(total, to, retain_graph=True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_head_second_derivatives_raise(dtype):
    gen = torch.Generator(device=DEV).manual_seed(43)
    H = torch.randn(64, 70, 2, device=DEV, generator=gen).to(dtype).requires_grad_(True)       # (a transposed view goes in: a copy is saved)
    W = torch.randn(300, 64, device=DEV, generator=gen).to(dtype).requires_grad_(True)
    b = torch.randn(300, device=DEV, generator=gen).to(dtype).requires_grad_(True)
    weight = torch.rand(2, 300, device=DEV, generator=gen).requires_grad_(True)
    mask = torch.ones(2, 70, dtype=torch.bool, device=DEV)
    for of in (H, W, b):
        Y, I = lsr_head(H.permute(2, 1, 0), W, b, mask)
        plain, = torch.autograd.grad(Y, of, weight.detach(), retain_graph=True)
        g, total = penalised(Y, sum((x.float() ** 2).sum() for x in (H, W, b)), of, weight)
        assert torch.equal(g, plain)
        for to in (H, W, b, weight):
            with pytest.raises(RuntimeError, match="lsr_head"):
                torch.autograd.grad(total, to, retain_graph=True)
        with pytest.raises(RuntimeError, match="lsr_head"):
            total.backward(retain_graph=True)
