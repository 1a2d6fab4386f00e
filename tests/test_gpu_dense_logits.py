"""The operators around the dense logits on the GPU against float64 definitions, at the sizes, strides and masks where they can go wrong.

Tolerances follow from the arithmetic, with u = 2^-24 (half a unit of float32) and b = 2^-8 (bfloat16: 8 significant bits):
  products   float32 sums of n products, each addition rounded: |error| <= 8 sqrt(n) u sum|a b| (errors of either sign; 8 standard deviations),
             plus 8 u sum|a b| for the roundings at either end; float32 operands as six plane products: n becomes 6 n
  exp        v_exp_f32 and the multiplication of its argument x: relative error <= (4 + 2 |x|) u
  bfloat16   one rounding: b |result|; g as an operand: b |g| each, independent: 4 b sqrt(sum g^2 W^2) (7 standard deviations)
"""
import math

import numpy as np
import pytest
import torch

import paper_2603_25011_amd as lsr
from oracle import distill_oracle as orc
from paper_2603_25011_amd import distill

pytestmark = pytest.mark.gpu
U, B = 2.0 ** -24, 2.0 ** -8
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
KIND = {"f32": lsr.LSR_F32, "bf16": lsr.LSR_BF16}


def dev(x, dtype=None):
    return torch.as_tensor(np.asarray(x), device=DEV).to(dtype) if dtype is not None else torch.as_tensor(np.asarray(x), device=DEV)


def host(t):
    return t.detach().double().cpu().numpy()


def close(got, want, tol, what):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape, what
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    bad = ~same & ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(got - want)[bad])} at {np.argwhere(bad)[0]}"


# ---- quantize ----

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,pitch", [(1, 1, 1), (3, 7, 9), (5, 127, 127), (4, 128, 128), (9, 312, 320), (66, 768, 768), (7, 1000, 1001),
                                             (3, 2048, 2048), (2, 2050, 2056), (2, 4100, 4104), (1, 65536, 65536)])
def test_quantize_rows(rows, cols, pitch, dtype):
    gen = torch.Generator().manual_seed(rows * 7919 + cols)
    x = (torch.randn(rows, pitch, generator=gen) * torch.rand(rows, 1, generator=gen).mul(8).exp()).to(TYPES[dtype]).to(DEV)[:, :cols]
    q, s = distill.quantize_rows(x)
    assert q.shape == (rows, lsr.lsr_int8_row_bytes(cols)) and not q[:, cols:].any()
    levels, scale = orc.quantize_rows(host(x))
    close(host(s), scale, U * scale, "scale")                       # one float32 division
    got = host(q[:, :cols])
    if dtype == "bf16":
        assert np.array_equal(got, levels)                          # 127 x is exact
    else:
        # 127 x is rounded once: another level only where the exact quotient is within 127 u of half-way
        frac = host(x) * 127 / np.abs(host(x)).max(axis=1, keepdims=True)
        near = np.abs(np.abs(frac - np.floor(frac)) - 0.5) <= 127 * U
        assert np.array_equal(got[~near], levels[~near]) and np.abs(got - levels).max() <= 1


def test_quantize_special_rows():
    x = torch.zeros(9, 200)
    x[1] = torch.linspace(-1, 1, 200) * 3.3e38        # 127 x leaves the range of float32
    x[2] = torch.linspace(-1, 1, 200) * 1e-38
    x[3, 5] = 1e-45                                    # the smallest subnormal
    x[4], x[5], x[6] = 1.0, 2.0, 3.0
    x[4, 17], x[5, 199], x[6, 0] = math.inf, -math.inf, math.nan
    x[7, 100] = -0.0
    x[8] = torch.arange(200) % 128 - 63.5              # halves everywhere
    x[8, 0] = 127.0
    q, s = distill.quantize_rows(x.to(DEV))
    levels, scale = orc.quantize_rows(x.double().numpy())
    assert np.array_equal(host(q[:, :200]), levels)
    assert np.array_equal(np.isnan(host(s)), np.isnan(scale))
    fine = ~np.isnan(scale)
    close(host(s)[fine], scale[fine], U * scale[fine] + 2.0 ** -150, "scale")


def test_quantize_leaves_the_rest_of_a_wider_row():
    x = torch.randn(5, 130, device=DEV)
    Q = torch.full((5, 512), 77, dtype=torch.int8, device=DEV)
    s = torch.empty(5, device=DEV)
    lsr.lsr_quantize_rows(5, 130, lsr.LSR_F32, x, 130, Q, 512, s)
    assert (Q[:, 256:] == 77).all() and not Q[:, 130:256].any()


# ---- 8-bit product ----

def int8_case(N, V, K, seed, lda=None, ldw=None):
    rng = np.random.default_rng(seed)
    kp = lsr.lsr_int8_row_bytes(K)
    A = np.zeros((N, lda or kp), np.int8)
    W = np.zeros((V, ldw or kp), np.int8)
    A[:, :K] = rng.integers(-127, 128, (N, K))
    W[:, :K] = rng.integers(-127, 128, (V, K))
    A[:, kp:], W[:, kp:] = 99, 98                      # what lies behind a row is not its own
    a, w = rng.random(N).astype(np.float32), rng.random(V).astype(np.float32)
    return A, a, W, w, rng.standard_normal(V).astype(np.float32) * 100


SIZES = [(1, 1, 1), (1, 30522, 768), (2, 33, 100), (12, 517, 1024), (31, 257, 130), (32, 64, 64), (33, 300, 312), (64, 255, 500), (65, 256, 128),
         (197, 1031, 312), (256, 256, 256), (300, 513, 1000), (520, 777, 72), (1, 130, 65536), (3, 97, 20000)]


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("N,V,K", SIZES)
def test_int8_matmul(N, V, K, out):
    kp = lsr.lsr_int8_row_bytes(K)
    wide = (N + V) % 2 == 0
    A, a, W, w, bias = int8_case(N, V, K, N + V + K, kp + 48 if wide else None, kp + 16 if wide else None)
    if K == 65536:
        A[:], W[:, :K] = 127, 127                      # the largest sum there is
    bias = None if N == 2 else bias
    ldo = V + (5 if wide else 0)
    Y = torch.full((N, ldo), -7.0, dtype=TYPES[out], device=DEV)
    lsr.lsr_int8_matmul(N, V, K, lsr.LSR_I8, KIND[out], dev(A), A.shape[1], dev(a), dev(W), W.shape[1], dev(w),
                        None if bias is None else dev(bias), Y, ldo, None)
    want = orc.int8_matmul(A[:, :K], a, W[:, :K], w, bias)
    scaled = np.abs(want - (0 if bias is None else bias))
    # the sum becomes a float32, the scales' product, their product, and the sum with the bias: a rounding each
    tol = 3 * U * scaled + U * np.abs(want)
    close(host(Y[:, :V]), want, tol + (B * (np.abs(want) + tol) if out == "bf16" else 0), "logits")
    assert (Y[:, V:] == -7.0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V,K,pitch", [(1, 700, 768, 768), (5, 300, 100, 101), (40, 300, 312, 320), (64, 1000, 1100, 1100), (70, 300, 1100, 1103),
                                         (300, 520, 200, 200)])
def test_int8_matmul_quantises_values_as_quantize_rows_does(N, V, K, pitch, dtype):
    gen = torch.Generator().manual_seed(N + V)
    H = torch.randn(N, pitch, generator=gen).to(TYPES[dtype]).to(DEV)[:, :K]
    W = torch.randn(V, K, generator=gen).to(DEV)
    head = distill.Int8Head(W, torch.randn(V, generator=gen).to(DEV))
    got = head.logits(H)
    q, s = distill.quantize_rows(H)
    want = torch.empty_like(got)
    lsr.lsr_int8_matmul(N, V, K, lsr.LSR_I8, lsr.LSR_F32, q, q.stride(0), s, head.W8, head.W8.stride(0), head.w_scale, head.bias, want, V, None)
    assert torch.equal(got, want)


def test_int8_rows_that_are_not_finite_show_in_their_logits_only():
    for N in (4, 80):
        H = torch.randn(N, 64, device=DEV)
        H[1, 3], H[2, 5], H[3] = math.nan, math.inf, 0.0
        head = distill.Int8Head(torch.randn(50, 64, device=DEV), torch.randn(50, device=DEV))
        y = head.logits(H)
        assert y[1:3].isnan().all() and y[[0, *range(3, N)]].isfinite().all() and torch.equal(y[3], head.bias)


def test_int8_offsets_beyond_32_bits():
    # 16 rows of logits that lie 2^28 elements apart (4 GiB and more behind the first), rows of W at odd pitches of 2^23
    N, V, K = 9, 300, 128
    A, a, W, w, bias = int8_case(N, V, K, 5)
    Wide = torch.zeros((V, 1 << 23), dtype=torch.int8, device=DEV)
    Wide[:, :128] = dev(W)
    Y = torch.empty(((N - 1) << 28) + V, dtype=torch.bfloat16, device=DEV)
    lsr.lsr_int8_matmul(N, V, K, lsr.LSR_I8, lsr.LSR_BF16, dev(A), 128, dev(a), Wide, 1 << 23, dev(w), dev(bias), Y, 1 << 28, None)
    want = orc.int8_matmul(A[:, :K], a, W[:, :K], w, bias)
    got = np.stack([host(Y[n << 28:(n << 28) + V]) for n in range(N)])
    close(got, want, 4 * U * (np.abs(want) + 200) + 1.01 * B * np.abs(want), "logits")
    A2, a2, *_ = int8_case(100, V, K, 6)
    out = torch.empty((100, V), device=DEV)
    lsr.lsr_int8_matmul(100, V, K, lsr.LSR_I8, lsr.LSR_F32, dev(A2), 128, dev(a2), Wide, 1 << 23, dev(w), dev(bias), out, V, None)
    want = orc.int8_matmul(A2[:, :K], a2, W[:, :K], w, bias)
    close(host(out), want, 4 * U * (np.abs(want) + 200), "logits")


# ---- top logits ----

def lse_tolerance(x, T):
    # the largest exponent that still counts is about 20; the sum adds V terms, 32 at a time per thread
    with np.errstate(invalid="ignore"):
        return 64 * U + 2 * U * np.abs(orc.log_sum_exp(x / T)) + 16 * U * math.sqrt(x.shape[1] / 32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V,K,pitch,T", [(1, 1, 1, 1, 1.0), (3, 5, 5, 5, 2.0), (2, 300, 256, 301, 1.0), (7, 1031, 33, 1031, 0.5), (1, 30522, 64, 30522, 1.0),
                                              (4, 8192, 128, 8193, 1.0), (5, 8207, 1, 8210, 4.0), (2, 50001, 256, 50001, 1.0), (1, 250002, 10, 250002, 2.0),
                                              (3, 40000, 100, 40003, 1.0), (2100, 700, 16, 701, 1.0)])
def test_top_logits(rows, V, K, pitch, T, dtype):
    gen = torch.Generator().manual_seed(rows + V + K)
    x = (torch.randn(rows, pitch, generator=gen) * 3).to(TYPES[dtype])[:, :V]
    wide = torch.empty(rows, pitch, dtype=x.dtype, device=DEV)
    wide[:, :V] = x.to(DEV)
    v, i, lse = distill.top_logits(wide[:, :V], K, T)
    xv, xi, xl = orc.top_logits(x.double().numpy(), K, T)
    assert np.array_equal(host(i), xi) and np.array_equal(host(v), xv)         # bfloat16 has many ties
    close(host(lse), xl, lse_tolerance(x.double().numpy(), T), "lse")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 9000, 70000])
def test_top_logits_hard_rows(V, dtype):
    K = 37
    x = torch.zeros(12, V)
    ramp = torch.arange(V).float()
    x[0] = ramp                                        # every logit beats the ones before it
    x[1] = -ramp
    x[2] = 0.0                                         # all equal: the lowest ids
    x[3] = -math.inf                                   # nothing allowed
    x[4] = -math.inf
    x[4, V - 1], x[4, 3], x[4, V // 2] = -5.0, 1.0, 1.0
    x[5] = torch.finfo(TYPES[dtype]).min               # masks of the type's lowest value
    x[5, V // 3] = 0.25
    x[6] = torch.sin(ramp)
    x[6, 7], x[6, V - 2] = math.inf, math.inf
    x[7] = torch.cos(ramp)
    x[7, V - 1], x[7, 0], x[7, 5] = math.nan, math.inf, -math.nan
    x[8] = torch.where(ramp % 2 == 0, 0.0, -0.0)       # both zeros are one value
    x[9] = torch.floor(ramp / 100) % 7                 # long runs of ties
    x[10] = torch.where(ramp % 1024 < 3, ramp, -1.0)
    x[11] = math.nan
    x = x.to(TYPES[dtype])
    v, i, lse = distill.top_logits(x.to(DEV), K, 1.5)
    xv, xi, xl = orc.top_logits(x.double().numpy(), K, 1.5)
    assert np.array_equal(host(i), xi)
    assert np.array_equal(host(v), xv, equal_nan=True)
    close(host(lse), xl, lse_tolerance(np.where(np.isnan(x.double().numpy()), 0, x.double().numpy()), 1.5), "lse")


def test_top_logits_rows_beyond_4_gib_and_without_lse():
    x = torch.zeros((5, 1 << 30), dtype=torch.bfloat16, device=DEV)
    x[4, 1000], x[4, 17] = 3.0, 2.0
    v, i = torch.empty((5, 2), device=DEV), torch.empty((5, 2), dtype=torch.int32, device=DEV)
    lsr.lsr_top_logits(5, 2000, 2, lsr.LSR_BF16, 1.0, x, 1 << 30, v, i, None, None)
    assert i.tolist() == [[0, 1]] * 4 + [[1000, 17]] and v[4].tolist() == [3.0, 2.0]


# ---- distillation ----

def distill_case(N, D, V, K, dtype, seed, keep=1.0, given=True, T=1.0, spread=0.05):
    rng = np.random.default_rng(seed)
    td = TYPES[dtype]
    H = torch.from_numpy(rng.standard_normal((N, D)).astype(np.float32)).to(td)
    W = torch.from_numpy((rng.standard_normal((V, D)) * spread).astype(np.float32)).to(td)
    bias = torch.from_numpy((rng.standard_normal(V) * 0.1).astype(np.float32))
    ids = np.stack([rng.permutation(V)[:K] if K <= V else rng.integers(0, V, K) for _ in range(N)])
    logits = (rng.standard_normal((N, K)) * 2.5).astype(np.float32)
    L = (orc.log_sum_exp(logits.astype(np.float64) / T) + rng.random(N) * 0.5).astype(np.float32) if given else None
    mask = (rng.random(N) < keep).astype(np.uint8) if keep < 1 else None
    dloss = (rng.standard_normal(N)).astype(np.float32)
    return H, W, bias, ids.astype(np.int32), logits, L, mask, T, dloss


def run_and_check(case, need=(True, True, True)):
    H, W, bias, ids, logits, L, mask, T, dloss = case
    f32 = H.dtype == torch.float32
    D, N, V, K = H.shape[1], H.shape[0], W.shape[0], ids.shape[1]
    args = [t.to(DEV).requires_grad_(n) for t, n in zip((H, W, bias), need)]
    loss, lse = distill.lsr_distill(*args, dev(ids), dev(logits), None if L is None else dev(L), None if mask is None else dev(mask), T)
    h, w, b = H.double().numpy(), W.double().numpy(), bias.double().numpy()
    want = orc.distill(h, w, b, ids, logits, L, mask, T, dloss)
    on = np.ones(N) if mask is None else (mask != 0)
    size = np.abs(h) @ np.abs(w).T + np.where(np.isfinite(b), np.abs(b), 0)       # sum |h w| per logit
    n_add = 6 * D if f32 else D
    dz = (8 * math.sqrt(n_add) + 8) * U * size / T                                # error of a logit (over T)
    dzm = dz.max(axis=1)
    with np.errstate(invalid="ignore"):
        z = np.where(np.isfinite(want["lse"]), np.abs(want["lse"]), 0) + size.max(axis=1) / T
    dlse = dzm + (64 + 2 * z) * U
    close(host(lse), want["lse"], dlse, "lse")
    p, logp, _ = orc._teacher(ids, logits, L, V, T)
    mass = p.sum(axis=1)
    t_size = np.abs(np.where(np.isfinite(logits), logits, 0)).max(axis=1) / T + (np.abs(L) if L is not None else 0) + 1
    dp = (8 + 4 * t_size) * U                                                     # relative error of p, a value for each row
    terms = (p * (np.abs(logp) + z[:, None])).sum(axis=1)
    with np.errstate(invalid="ignore"):
        dloss_tol = mass * (dzm + dlse) + 2 * dp * terms + 8 * math.sqrt(K) * U * terms + 4 * U * z * mass
    close(host(loss), want["loss"], dloss_tol, "loss")
    if not any(need):
        return None
    grads = torch.autograd.grad(loss, [a for a, n in zip(args, need) if n], dev(dloss))
    got = dict(zip([k for k, n in zip(("dH", "dW", "db"), need) if n], grads))
    # g = s mass q - s p: q to dz + dlse + exp, p to dp
    s = np.abs(dloss * on / T)[:, None]
    zz = h @ w.T / T
    q_part = s * mass[:, None] * np.exp(zz + b / T - orc.log_sum_exp(zz + b / T)[:, None])
    p_part = np.abs(want["g"]) + q_part
    rel = 2 * (dz + dlse[:, None]) + (16 + 2 * (z[:, None] + 20)) * U + 8 * math.sqrt(K) * U + dp[:, None]
    dg = q_part * rel + p_part * (dp[:, None] + 4 * U)
    for key, x, y, wide in (("dH", dg, np.abs(w), V), ("dW", dg.T, np.abs(h), N)):
        if key not in got:
            continue
        g = np.abs(want["g"]) if key == "dH" else np.abs(want["g"]).T
        n_sum = 6 * wide if f32 else wide
        tol = x @ y + (8 * math.sqrt(n_sum) + 8) * U * (g @ y)
        if not f32:
            tol = tol + 4 * B * np.sqrt((g ** 2) @ (y ** 2)) + B * (np.abs(want[key]) + tol)
        close(host(got[key]), want[key], tol + 1e-37, key)
    if "db" in got:
        close(host(got["db"]), want["db"], dg.sum(axis=0) + (8 * math.sqrt(N) + 8) * U * np.abs(want["g"]).sum(axis=0) + 1e-37, "db")
    return got


SHAPES = [(1, 8, 1, 1), (1, 64, 300, 5), (3, 72, 257, 256), (5, 312, 1000, 33), (17, 64, 5, 5), (64, 768, 2001, 64), (255, 128, 256, 7),
          (256, 136, 513, 16), (257, 64, 511, 100), (300, 1024, 700, 3), (513, 200, 777, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,V,K", SHAPES)
def test_distill(N, D, V, K, dtype):
    seed = N + D + V + K
    run_and_check(distill_case(N, D, V, K, dtype, seed, keep=1.0 if N % 2 else 0.6, given=N % 3 != 0, T=[1.0, 2.0, 0.7][N % 3]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_distill_masks_and_padding(dtype):
    H, W, bias, ids, logits, L, mask, T, dloss = distill_case(300, 64, 600, 9, dtype, 5, keep=0.5)
    mask[:40] = 0                                       # no valid row in front
    mask[290:] = 0
    ids[100:110, 2:] = -1                               # short lists of a teacher
    ids[111, 4], ids[112, 1], ids[113, 0] = 600, 2 ** 31 - 1, -2 ** 31
    logits[120:130, 5] = -np.inf
    logits[131] = -np.inf                               # a row without any entry, either way
    ids[132] = -1
    mask[100:133] = 7                                   # any non-zero byte counts
    ids[140, 1] = ids[140, 0]                           # an id that comes twice
    ids[141] = ids[141, 0]
    mask[140:142] = 1
    for given in (L, None):
        got = run_and_check((H, W, bias, ids, logits, given, mask, T, dloss))
        assert not got["dH"][dev(mask == 0)].any() and not got["dH"][131:133].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_distill_with_every_row_left_out(dtype):
    case = list(distill_case(70, 64, 300, 4, dtype, 6))
    case[6] = np.zeros(70, np.uint8)
    got = run_and_check(tuple(case))
    assert not any(got[k].any() for k in got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_distill_with_excluded_entries(dtype):
    case = list(distill_case(100, 64, 700, 6, dtype, 7))
    gone = np.zeros(700, bool)
    gone[[0, 255, 256, 699]] = True
    gone[300:560] = True                                # a whole tile of logits among them
    case[2] = torch.where(torch.from_numpy(gone), -math.inf, case[2].double()).float()
    case[3] = np.where(gone[case[3]], -1, case[3]).astype(np.int32)
    got = run_and_check(tuple(case))
    assert not got["dW"][dev(gone)].any() and not got["db"][dev(gone)].any()
    # a teacher that insists on an excluded entry: an infinite loss, in that row only
    case[3][5, 0] = 300
    H, W, bias, ids, logits, L, mask, T, _ = case
    loss, _ = distill.lsr_distill(H.to(DEV), W.to(DEV), bias.to(DEV), dev(ids), dev(logits), dev(L), None, T)
    assert loss[5] == math.inf and loss[[0, 1, 2, 3, 4, *range(6, 100)]].isfinite().all()


@pytest.mark.parametrize("need", [(True, False, False), (False, True, False), (False, False, True), (True, False, True), (False, True, True),
                                  (True, True, False), (False, False, False)])
def test_distill_gradients_that_are_wanted_only(need):
    run_and_check(distill_case(40, 72, 520, 5, "bf16", 8, keep=0.7), need)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_distill_crowded_tiles(dtype):
    # all entries of all rows in one or two tiles of logits, in the same few columns
    case = list(distill_case(300, 64, 2000, 200, dtype, 9))
    rng = np.random.default_rng(10)
    case[3] = np.stack([512 + rng.permutation(256)[:200] for _ in range(300)]).astype(np.int32)
    run_and_check(tuple(case))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_distill_large_logits(dtype):
    # peaked distributions: most of the vocabulary underflows
    run_and_check(distill_case(60, 64, 900, 8, dtype, 11, spread=3.0))


# up to 64 rows whose hidden states fit LDS take a path of their own; 64 x 1024 in bfloat16 still fit, 40 x 1024 in float32 and rows of 8192 do not
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,D,V,K", [(2, 1024, 31, 3), (31, 40, 33, 9), (32, 264, 1025, 64), (33, 24, 640, 200), (40, 1024, 515, 8), (63, 520, 129, 2), (64, 1024, 700, 17),
                                     (65, 64, 300, 5), (7, 8192, 300, 4)])
def test_distill_few_rows(N, D, V, K, dtype):
    run_and_check(distill_case(N, D, V, K, dtype, N + D + V, keep=0.7, given=N % 2 == 0, T=[1.0, 2.0][N % 2]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [20, 50])
def test_distill_few_rows_masks_padding_and_excluded_entries(N, dtype):
    H, W, bias, ids, logits, L, mask, T, dloss = distill_case(N, 96, 600, 9, dtype, 21, keep=0.8)
    gone = np.zeros(600, bool)
    gone[[0, 255, 256, 599]] = True
    gone[300:360] = True
    bias = torch.where(torch.from_numpy(gone), -math.inf, bias.double()).float()
    ids = np.where(gone[ids], -1, ids).astype(np.int32)
    mask[:3], mask[-2:] = 0, 0
    ids[4, 2:] = -1
    ids[5], logits[6], ids[7, 1] = -1, -np.inf, 600
    ids[8, 1] = ids[8, 0]
    mask[4:9] = 9
    for given in (L, None):
        got = run_and_check((H, W, bias, ids, logits, given, mask, T, dloss))
        assert not got["dH"][dev(mask == 0)].any() and not got["dH"][5:7].any()
        assert not got["dW"][dev(gone)].any() and not got["db"][dev(gone)].any()
    got = run_and_check((H, W, bias, ids, logits, L, np.zeros(N, np.uint8), T, dloss))
    assert not any(got[k].any() for k in got)


@pytest.mark.parametrize("need", [(True, False, False), (False, True, False), (False, False, True), (False, False, False)])
def test_distill_few_rows_gradients_that_are_wanted_only(need):
    run_and_check(distill_case(33, 72, 520, 5, "bf16", 22, keep=0.7), need)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [30, 300])
def test_distill_reads_nothing_of_rows_and_entries_that_are_left_out(N, dtype):
    H, W, bias, ids, logits, L, mask, T, dloss = distill_case(N, 96, 600, 9, dtype, 25, keep=0.7)
    ids[::3, 4] = -1
    rest = lambda i, l, t: (dev(i), dev(l), dev(t), dev(mask), T)                # noqa: E731
    args = [t.to(DEV).requires_grad_(True) for t in (H, W, bias)]
    loss, lse = distill.lsr_distill(*args, *rest(ids, logits, L))
    want = [loss.detach(), lse, *torch.autograd.grad(loss, args, dev(dloss))]
    off = mask == 0
    H2, ids2, logits2, L2, dloss2 = H.clone(), ids.copy(), logits.copy(), L.copy(), dloss.copy()
    H2[torch.from_numpy(off)] = math.nan
    H2[int(np.flatnonzero(off)[0])] = math.inf
    ids2[off], logits2[off], L2[off], dloss2[off] = 2 ** 30, np.nan, np.inf, np.nan
    logits2[::3, 4] = np.nan                            # of an entry that is padding by its id
    args = [t.to(DEV).requires_grad_(True) for t in (H2, W, bias)]
    loss, lse = distill.lsr_distill(*args, *rest(ids2, logits2, L2))
    got = [loss.detach(), lse, *torch.autograd.grad(loss, args, dev(dloss2))]
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_distill_few_rows_crowded_tile():
    case = list(distill_case(48, 64, 2000, 200, "bf16", 23))
    rng = np.random.default_rng(24)
    case[3] = np.stack([512 + rng.permutation(256)[:200] for _ in range(48)]).astype(np.int32)
    run_and_check(tuple(case))


def test_distill_in_pieces_of_the_vocabulary():
    # so many rows that the backward walks the vocabulary in pieces
    N, D, V, K = 262144, 64, 3000, 2
    case = distill_case(64, D, V, K, "bf16", 12)
    H, W, bias, ids, logits, L, _, T, dloss = case
    reps = N // 64
    mask = torch.zeros(N, dtype=torch.uint8, device=DEV)
    mask[:64], mask[-64:] = 1, 1
    big = [H.to(DEV).repeat(reps, 1).requires_grad_(True), W.to(DEV).requires_grad_(True), bias.to(DEV).requires_grad_(True)]
    loss, _ = distill.lsr_distill(*big, dev(ids).repeat(reps, 1), dev(logits).repeat(reps, 1), dev(L).repeat(reps), mask, T)
    got = torch.autograd.grad(loss, big, dev(dloss).repeat(reps))
    two = [H.repeat(2, 1).to(DEV).requires_grad_(True), W.to(DEV).requires_grad_(True), bias.to(DEV).requires_grad_(True)]
    loss2, _ = distill.lsr_distill(*two, dev(ids).repeat(2, 1), dev(logits).repeat(2, 1), dev(L).repeat(2), None, T)
    want = torch.autograd.grad(loss2, two, dev(dloss).repeat(2))
    assert torch.equal(loss[:64], loss2[:64]) and torch.equal(loss[-64:], loss2[64:]) and not loss[64:-64].any()
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
    # dH: the contracted axis is cut at other places, so its float32 sums round differently: by a step of bfloat16 at most, and rarely
    for a, b in ((got[0][:64], want[0][:64]), (got[0][-64:], want[0][64:])):
        close(host(a), host(b), 2 * B * np.abs(host(b)) + 64 * U * np.abs(host(b)).max(), "dH")
    assert not got[0][64:-64].any()
    run_and_check((H.repeat(2, 1), W, bias, np.tile(ids, (2, 1)), np.tile(logits, (2, 1)), np.tile(L, 2), None, T, np.tile(dloss, 2)))


def test_distill_shapes_types_and_views():
    H, W, bias, ids, logits, L, mask, T, dloss = distill_case(48, 64, 300, 4, "bf16", 13, keep=0.7)
    flat = distill.lsr_distill(H.to(DEV), W.to(DEV), bias.to(DEV), dev(ids), dev(logits), dev(L), dev(mask), T)[0]
    pad = torch.zeros(48, 71, dtype=torch.bfloat16, device=DEV)
    pad[:, 3:67] = H.to(DEV)
    wide = torch.zeros(48, 9, dtype=torch.int64, device=DEV)
    wide[:, ::2][:, :4] = dev(ids).long()
    got, lse = distill.lsr_distill(pad[:, 3:67].reshape(6, 8, 64), W.to(DEV).t().contiguous().t(), bias.double().to(DEV), wide[:, ::2][:, :4].reshape(6, 8, 4),
                                   dev(logits).double().reshape(6, 8, 4), dev(L).reshape(6, 8), dev(mask).bool().reshape(6, 8), T)
    assert got.shape == (6, 8) and lse.shape == (6, 8) and torch.equal(got.reshape(-1), flat)
    far = dev(ids).long()
    far[0, 0] = (1 << 32) + 3                           # not entry 3
    near = dev(ids).clone()
    near[0, 0] = -1
    a = distill.lsr_distill(H.to(DEV), W.to(DEV), bias.to(DEV), far, dev(logits), dev(L), None, T)[0]
    b = distill.lsr_distill(H.to(DEV), W.to(DEV), bias.to(DEV), near, dev(logits), dev(L), None, T)[0]
    assert torch.equal(a, b)
    empty = distill.lsr_distill(H.to(DEV)[:0].requires_grad_(True), W.to(DEV).requires_grad_(True), bias.to(DEV), dev(ids)[:0], dev(logits)[:0])[0]
    empty.sum().backward()
    assert empty.shape == (0,)
    with pytest.raises(TypeError):
        distill.lsr_distill(H.to(DEV), W.float().to(DEV), bias.to(DEV), dev(ids), dev(logits))
    with pytest.raises(TypeError):
        distill.lsr_distill(H.to(DEV), W.to(DEV), bias.to(DEV), dev(ids).float(), dev(logits))
    with pytest.raises(ValueError):
        distill.lsr_distill(H.to(DEV), W.to(DEV), bias.to(DEV)[:-1], dev(ids), dev(logits))
    with pytest.raises(ValueError):
        distill.lsr_distill(H.to(DEV), W.to(DEV), bias.to(DEV), dev(ids), dev(logits), dev(L)[:-1])
    with pytest.raises(RuntimeError):
        distill.lsr_distill(H.to(DEV), W, bias.to(DEV), dev(ids), dev(logits))


def test_distill_gradients_by_differences():
    H, W, bias, ids, logits, L, mask, T, dloss = distill_case(40, 64, 300, 6, "f32", 14, keep=0.8, T=2.0)
    args = [t.to(DEV).requires_grad_(True) for t in (H, W, bias)]
    rest = (dev(ids), dev(logits), dev(L), dev(mask), T)
    weight = dev(dloss)
    grads = torch.autograd.grad((distill.lsr_distill(*args, *rest)[0] * weight).sum(), args)
    gen = torch.Generator(device=DEV).manual_seed(15)
    eps = 2.0 ** -6
    for k in range(3):
        d = torch.randn(args[k].shape, device=DEV, generator=gen)
        d /= d.norm()
        sums = []
        for f in (1, -1, 2, -2):
            moved = [a.detach() + (f * eps * d if i == k else 0) for i, a in enumerate(args)]
            sums.append((distill.lsr_distill(*moved, *rest)[0].double() * weight.double()).sum().item())
        # five points: the error is of order eps^4 times the fifth derivative, and the rounding of 32 losses over eps
        diff = (8 * (sums[0] - sums[1]) - (sums[2] - sums[3])) / (12 * eps)
        want = (grads[k].double() * d.double()).sum().item()
        noise = 40 * 64 * U * 10 / eps
        assert abs(diff - want) <= noise + 1e-4 * abs(want), (k, diff, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_distill_repeats_its_bits_on_other_streams(dtype):
    H, W, bias, ids, logits, L, mask, T, dloss = distill_case(600, 136, 1500, 40, dtype, 16, keep=0.8)
    rest = (dev(ids), dev(logits), dev(L), dev(mask), T)
    args = [t.to(DEV).requires_grad_(True) for t in (H, W, bias)]

    def once():
        loss, lse = distill.lsr_distill(*args, *rest)
        return [loss.detach(), lse, *torch.autograd.grad(loss, args, dev(dloss))]

    first = once()
    torch.cuda.synchronize()
    for stream in (torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.Stream()):
        with torch.cuda.stream(stream):
            again = once()
        stream.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_all_operators_in_a_graph():
    N, D, V, K = 200, 128, 3000, 16
    H, W, bias, ids, logits, L, mask, T, dloss = distill_case(N, D, V, K, "bf16", 17, keep=0.8)
    H, W, bias, mask, weight = H.to(DEV), W.to(DEV), bias.to(DEV), dev(mask), dev(dloss)
    head = distill.Int8Head(torch.randn(V, D, device=DEV) * 0.05, bias)
    lg = torch.empty((N, V), device=DEV)
    v, i, l = torch.empty((N, K), device=DEV), torch.empty((N, K), dtype=torch.int32, device=DEV), torch.empty(N, device=DEV)
    loss, lse = torch.empty(N, device=DEV), torch.empty(N, device=DEV)
    dH, dW, db = torch.empty_like(H), torch.empty_like(W), torch.empty_like(bias)
    ws = torch.empty(max(lsr.lsr_int8_matmul_workspace_bytes(N, V, D, 1), lsr.lsr_top_logits_workspace_bytes(N, V, K),
                         *(lsr.lsr_distill_workspace_bytes(N, D, V, K, 1, T, b) for b in (False, True))), dtype=torch.uint8, device=DEV)
    shape = (N, D, V, K, lsr.LSR_BF16, T)

    def work():
        lsr.lsr_int8_matmul(N, V, D, lsr.LSR_BF16, lsr.LSR_F32, H, D, None, head.W8, head.W8.stride(0), head.w_scale, head.bias, lg, V, ws)
        lsr.lsr_top_logits(N, V, K, lsr.LSR_F32, T, lg, V, v, i, l, ws)
        lsr.lsr_distill_forward(*shape, H, W, bias, i, v, l, mask, loss, lse, ws)
        lsr.lsr_distill_backward(*shape, H, W, bias, i, v, l, mask, lse, weight, dH, dW, db, ws)

    outs = (lg, v, i, l, loss, lse, dH, dW, db)
    graph = torch.cuda.CUDAGraph()
    work()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        work()
    for k in range(3):
        H.copy_(torch.randn(N, D, device=DEV))
        work()
        want = [o.clone() for o in outs]
        for o in outs:
            o.zero_()
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), k


def test_teacher_to_student():
    # the operators as they are used together: a student that starts far from its teacher comes near it
    torch.manual_seed(18)
    N, D, V, K, T = 512, 64, 1200, 32, 2.0
    H = torch.randn(N, D, device=DEV, dtype=torch.bfloat16)
    Wt, bt = torch.randn(V, D, device=DEV) * 0.3, torch.randn(V, device=DEV)
    teacher = distill.Int8Head(Wt, bt)
    values, ids, tl = teacher.top_logits(H, K, T, max_logits=100 * V)
    whole = distill.top_logits(teacher.logits(H), K, T)
    assert torch.equal(values, whole[0]) and torch.equal(ids, whole[1]) and torch.equal(tl, whole[2])
    W = torch.zeros(V, D, device=DEV, dtype=torch.float32, requires_grad=True)
    b = torch.zeros(V, device=DEV, requires_grad=True)
    opt = torch.optim.Adam([W, b], lr=0.05)
    losses = []
    for _ in range(40):
        loss = distill.lsr_distill(H.float(), W, b, ids, values, None, None, T)[0].mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(loss.item())
    assert losses[-1] < 0.1 * losses[0]
