"""The operators around the dense logits at the ends of what they accept."""
import math

import pytest
import torch

import paper_2603_25011_amd as lsr
from paper_2603_25011_amd import distill
from tests import test_gpu_dense_logits as base

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_quantize_the_most_rows_that_are_accepted():
    # 2^26 - 1 rows: as many workgroups as would be 2^32 threads in one launch
    n = (1 << 26) - 1
    x = torch.ones((n, 1), dtype=torch.bfloat16, device=DEV)
    x[::3] = -2.0
    q, s = distill.quantize_rows(x)
    assert torch.equal(q[:, 0], torch.where(x[:, 0] < 0, -127, 127).to(torch.int8))
    assert not q.view(torch.int32)[:, 1:].any() and not q[:, 1:4].any()
    assert torch.equal(s, x[:, 0].float().abs() / 127)


def test_int8_matmul_the_most_rows_that_are_accepted():
    # the product reads the levels that the same call has quantised
    n = (1 << 26) - 1
    x = torch.ones((n, 1), dtype=torch.bfloat16, device=DEV)
    x[::3] = -2.0
    w = torch.zeros((1, 128), dtype=torch.int8, device=DEV)
    w[0, 0] = 127
    out = torch.full((n, 1), math.nan, dtype=torch.float32, device=DEV)
    ws = torch.empty(lsr.lsr_int8_matmul_workspace_bytes(n, 1, 1, lsr.LSR_BF16), dtype=torch.uint8, device=DEV)
    ws.fill_(255)                                       # scales that are not written are NaN
    lsr.lsr_int8_matmul(n, 1, 1, lsr.LSR_BF16, lsr.LSR_F32, x, 1, None, w, 128, torch.full((1,), 1 / 127, device=DEV), None, out, 1, ws)
    # two scales of a rounding each, their product, and the sum's product with it (and the squares of those)
    assert ((out - x.float()).abs() <= 4.001 * base.U * x.float().abs()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [20, 300])
def test_distill_a_row_that_is_not_a_number_says_so(N, dtype):
    # every logit of the row is NaN: so are its normaliser and its loss; the other rows do not see it
    H, W, bias, ids, logits, L, _, T, _ = base.distill_case(N, 64, 600, 5, dtype, 31)
    rest = (W.to(DEV), bias.to(DEV), base.dev(ids), base.dev(logits), base.dev(L), None, T)
    want = distill.lsr_distill(H.to(DEV), *rest)
    H[3, 7] = math.nan
    loss, lse = distill.lsr_distill(H.to(DEV), *rest)
    others = torch.arange(N, device=DEV) != 3
    assert lse[3].isnan() and loss[3].isnan()
    assert torch.equal(loss[others], want[0][others]) and torch.equal(lse[others], want[1][others])
    # entries that the bias excludes change nothing about it; a NaN in the matrix is in every row's logits
    out = torch.where(torch.arange(600, device=DEV) < 590, -math.inf, rest[1])
    assert distill.lsr_distill(H.to(DEV), rest[0], out, *rest[2:])[1][3].isnan()
    W2 = rest[0].clone()
    W2[599, 1] = math.nan
    assert distill.lsr_distill(H.to(DEV), W2, *rest[1:])[1].isnan().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [20, 300])
def test_distill_a_row_without_entries_has_no_gradient_where_nothing_is_allowed_either(N, dtype):
    # the bias excludes the whole vocabulary (lse = -inf), and the teacher has no entry: no loss, and zeros as gradients
    H, W, bias, ids, logits, _, _, T, dloss = base.distill_case(N, 64, 600, 5, dtype, 32)
    args = [t.to(DEV).requires_grad_(True) for t in (H, W, torch.full_like(bias, -math.inf))]
    loss, lse = distill.lsr_distill(*args, torch.full_like(base.dev(ids), -1), base.dev(logits), None, None, T)
    assert not loss.any() and (lse == -math.inf).all()
    assert not any(g.any() for g in torch.autograd.grad(loss, args, base.dev(dloss)))


@pytest.mark.parametrize("V,K", [(30522, 768), (70001, 384), (250002, 1024)])
def test_int8_rows_do_not_depend_on_how_many_come_along(V, K):
    # the kernels for few rows and for many give the same bits, wherever the one hands over to the other
    gen = torch.Generator(device=DEV).manual_seed(V)
    head = distill.Int8Head(torch.randn(V, K, device=DEV, generator=gen, dtype=torch.bfloat16), torch.randn(V, device=DEV, generator=gen))
    H = torch.randn(40, K, device=DEV, generator=gen)
    for dtype in (torch.float32, torch.bfloat16):
        want = torch.cat([head.logits(h, dtype) for h in H.split(1)])
        for n in (8, 9, 16, 17, 32, 33, 40):
            assert torch.equal(head.logits(H[:n], dtype), want[:n]), (n, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 40, 9000, 70000])
def test_top_logits_infinite_normalisers_are_exactly_that(V, dtype):
    # in one segment and in several (70000 entries of few rows), wherever the infinity lies
    td = base.TYPES[dtype]
    x = torch.zeros(6, V, dtype=td)
    x[0] = -math.inf
    x[1, V - 1] = math.inf
    x[2, 0] = math.inf
    x[3] = math.inf
    x[4] = -math.inf
    x[4, V // 2] = math.inf
    x[5] = -math.inf
    x[5, V // 2] = 1.5
    v, i, lse = distill.top_logits(x.to(DEV), 1, 2.0)
    assert lse.tolist() == [-math.inf, *[math.inf] * 4, 0.75]
    assert v[:, 0].tolist() == [-math.inf, *[math.inf] * 4, 1.5] and i[:, 0].tolist() == [0, V - 1, 0, 0, V // 2, V // 2]


def test_distill_infinite_normalisers_are_exactly_that():
    for N in (20, 300):
        H, W, bias, ids, logits, _, _, T, _ = base.distill_case(N, 64, 600, 5, "bf16", 33)
        rest = (base.dev(ids), base.dev(logits))
        loss, lse = distill.lsr_distill(H.to(DEV), W.to(DEV), torch.full((600,), -math.inf, device=DEV), torch.full_like(rest[0], 600), rest[1])
        assert (lse == -math.inf).all() and not loss.any()
