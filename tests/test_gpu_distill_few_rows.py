"""Distillation of up to 64 rows whose hidden states fit LDS: g goes into the bfloat16 products as two bfloat16 whose sum has 16 bits, and the tolerance says so.

The hidden states fit where (rows up to a multiple of 32) x (bytes of a row up to a multiple of 32, and 16) is at most 136 KiB: 64 rows of 1024 in bfloat16 do, 64 of
1080 do not; 32 of 1024 in float32 do, 33 of 768 do not.
"""
import math

import numpy as np
import pytest
import torch

from oracle import distill_oracle as orc
from paper_2603_25011_amd import distill
from tests import test_gpu_dense_logits as base
from tests.test_gpu_dense_logits import B, U, dev, host

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("N,D,V,K", [(1, 64, 300, 5), (20, 768, 2001, 64), (33, 264, 1025, 16), (50, 40, 3000, 3), (64, 1024, 700, 17)])
def test_g_keeps_sixteen_bits(N, D, V, K):
    H, W, bias, ids, logits, L, mask, T, dloss = base.distill_case(N, D, V, K, "bf16", N + V, keep=1.0 if N % 2 else 0.8)
    args = [t.to(DEV).requires_grad_(True) for t in (H, W, bias)]
    loss, _ = distill.lsr_distill(*args, dev(ids), dev(logits), dev(L), None if mask is None else dev(mask), T)
    dH, dW = torch.autograd.grad(loss, args[:2], dev(dloss))
    h, w, b = H.double().numpy(), W.double().numpy(), bias.double().numpy()
    want = orc.distill(h, w, b, ids, logits, L, mask, T, dloss)
    # errors of g as the kernel has it in float32: logits (sums of D products), their normaliser, exp, the teacher's p
    size = np.abs(h) @ np.abs(w).T + np.abs(b)
    dz = (8 * math.sqrt(D) + 8) * U * size / T
    z = np.abs(want["lse"]) + size.max(axis=1) / T
    dlse = dz.max(axis=1) + (64 + 2 * z) * U
    dp = (8 + 4 * (np.abs(logits).max(axis=1) / T + np.abs(L) + 1)) * U
    p = orc._teacher(ids, logits, L, V, T)[0]
    zz = (h @ w.T + b) / T
    on = np.ones(N) if mask is None else mask != 0
    q = np.abs(dloss * on / T)[:, None] * p.sum(axis=1)[:, None] * np.exp(zz - orc.log_sum_exp(zz)[:, None])
    g = np.abs(want["g"])
    rel = 2 * (dz + dlse[:, None]) + (16 + 2 * (z[:, None] + 20)) * U + 8 * math.sqrt(K) * U + dp[:, None]
    dg = q * rel + (g + q) * (dp[:, None] + 4 * U)
    # two bfloat16: what the first leaves (2^-8 of g at most) is rounded to 8 bits, so 2^-16 of g is lost; sums of two products a term; the result rounded once
    once = torch.from_numpy(want["g"]).to(torch.bfloat16).double().numpy()
    for key, got, e, a, y, n in (("dH", dH, dg, g, w, V), ("dW", dW, dg.T, g.T, h, N)):
        tol = e @ np.abs(y) + ((8 * math.sqrt(2 * n) + 8) * U + 2.0 ** -16) * (a @ np.abs(y))
        tol = tol + B * (np.abs(want[key]) + tol) + 1e-37
        base.close(host(got), want[key], tol, key)
        # and the tolerance tells one bfloat16 from two
        planted = torch.from_numpy((once if key == "dH" else once.T) @ y).to(torch.bfloat16).double().numpy()
        assert (np.abs(planted - want[key]) > tol).any(), key


# (536 in float32 and 1072 in bfloat16 are the widest that fit for 64 rows)
@pytest.mark.parametrize("N,D,V,K,dtype", [(64, 1080, 700, 17, "bf16"), (33, 2112, 515, 8, "bf16"), (33, 768, 700, 9, "f32"), (40, 768, 515, 33, "f32"), (64, 1024, 700, 17, "f32"),
                                           (64, 536, 300, 6, "f32"), (64, 1072, 300, 6, "bf16")])
def test_up_to_64_rows_on_either_side_of_what_fits(N, D, V, K, dtype):
    base.run_and_check(base.distill_case(N, D, V, K, dtype, N + D + V, keep=0.7, given=N % 2 == 0, T=[1.0, 2.0][N % 2]))
