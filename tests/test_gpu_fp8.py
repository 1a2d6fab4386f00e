"""The head's dense logits in 8-bit floating point on the GPU against float64 definitions, at the sizes, strides and values where they can go wrong.

Quantisation is exact: bytes and exponents are those of the definition.  Tolerances of the products follow from the arithmetic, with u = 2^-24 and b = 2^-8:
  exact sums   (float32 results) float32 sums of n exact products, each addition rounded: 8 sqrt(n) u sum|a b| (errors of either sign; 8 standard deviations) and
               8 u (sum|a b| + |bias|) for the roundings at either end
  fast sums    (bfloat16 results) as well, every product loses less than 2^-13 of the largest of its group of 8, toward zero: its square is at most 2^-26 times the
               sum of the group's squares, so all errors' squares together at most 8 2^-26 sum (a b)^2; with products of either sign 8 standard deviations are
               8 sqrt(8) 2^-13 sqrt(sum (a b)^2)
  bfloat16     one rounding: b |result|
"""
import numpy as np
import pytest
import torch

import paper_2603_25011_amd as lsr
from oracle import fp8_oracle as orc
from paper_2603_25011_amd import binding, distill, fp8

pytestmark = pytest.mark.gpu
U, B = 2.0 ** -24, 2.0 ** -8
DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
KIND = {"f32": lsr.LSR_F32, "bf16": lsr.LSR_BF16}


def host(t):
    return t.detach().double().cpu().numpy()


def close(got, want, tol, what):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape, what
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    bad = ~same & ~(np.abs(got - want) <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, worst {np.nanmax(np.abs(got - want)[bad])} at {np.argwhere(bad)[0]}"


def values(gen, shape, dtype, spread=2.0):
    """Normal values, rows and columns of different magnitude."""
    x = torch.randn(shape, generator=gen) * torch.randn(shape[0], 1, generator=gen).mul(spread).exp2() * torch.randn(1, shape[1], generator=gen).mul(spread).exp2()
    return x.to(TYPES[dtype]).to(DEV)


def tolerance(A, W, want, out, bias=None, n=None):
    """Of A W^T (float64 arrays of the values multiplied)."""
    a, w = np.abs(A), np.abs(W)
    total = a @ w.T
    n = A.shape[1] if n is None else n
    tol = 8 * U * (np.sqrt(n) + 1) * total + (0 if bias is None else 8 * U * np.abs(bias)) + 2.0 ** -126
    if out == "bf16":
        tol = tol + 8 * np.sqrt(8.0) * 2.0 ** -13 * np.sqrt((a * a) @ (w * w).T) + B * (np.abs(want) + tol)
    return tol


# ---- quantisation ----

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,pitch", [(1, 1, 1), (3, 7, 9), (127, 129, 129), (128, 128, 128), (130, 312, 320), (5, 1000, 1001), (300, 1030, 1040), (2, 70000, 70000),
                                             (1025, 40, 41)])
def test_quantize_is_the_definition(rows, cols, pitch, dtype):
    gen = torch.Generator().manual_seed(rows * 7919 + cols)
    x = values(gen, (rows, pitch), dtype)[:, :cols]
    for square in (False, True):
        for transposed in (False, True):
            q, e = fp8.quantize_blocks(x, square, transposed)
            X = host(x).T if transposed else host(x)
            n, m = X.shape
            assert q.shape == (n, binding.lsr_fp8_row_bytes(m)) and e.numel() == binding.lsr_fp8_exp_bytes(n, m) and not q[:, m:].any()
            want, exps = orc.blocks(X, 128 if square else 1, 128)
            assert np.array_equal(orc.unpack(q.cpu().numpy(), e.cpu().numpy(), m), want)
            got = e.cpu().numpy().reshape(-1, n, 4).astype(int)
            for b in range((m + 127) // 128):
                assert np.array_equal(got[b // 4, :, b % 4] - 127, exps[:, 128 * b]), (square, transposed, b)


def test_quantize_writes_both_forms_and_nothing_else():
    x = values(torch.Generator().manual_seed(0), (200, 300), "bf16")
    ldq, ldqt = 384 + 32, 256 + 16
    for square in (0, 1):
        Q = torch.full((200, ldq), 99, dtype=torch.uint8, device=DEV)
        Qt = torch.full((300, ldqt), 99, dtype=torch.uint8, device=DEV)
        E = torch.zeros(4 * 200, dtype=torch.uint8, device=DEV)
        Et = torch.zeros(4 * 300, dtype=torch.uint8, device=DEV)
        binding.lsr_fp8_quantize(200, 300, lsr.LSR_BF16, x, 300, square, Q, ldq, E, Qt, ldqt, Et)
        q, e = fp8.quantize_blocks(x, bool(square))
        qt, et = fp8.quantize_blocks(x, bool(square), True)
        assert torch.equal(Q[:, :384], q) and torch.equal(Qt[:, :256], qt) and (Q[:, 384:] == 99).all() and (Qt[:, 256:] == 99).all()
        assert torch.equal(E.view(-1, 200, 4)[..., :3], e[..., :3]) and torch.equal(Et.view(-1, 300, 4)[..., :2], et[..., :2])


@pytest.mark.parametrize("rows,cols", [(1, 1), (200, 300), (130, 700)])
def test_quantize_by_slab(rows, cols):
    x = values(torch.Generator().manual_seed(rows), (rows, cols), "f32")
    for square in (0, 1):
        n = binding.lsr_fp8_slab_bytes(cols, rows)
        Qt = torch.full((n,), 99, dtype=torch.uint8, device=DEV)
        Et = torch.zeros(binding.lsr_fp8_exp_bytes(cols, rows), dtype=torch.uint8, device=DEV)
        binding.lsr_fp8_quantize(rows, cols, lsr.LSR_F32, x, cols, square, None, 0, None, Qt, 0, Et)
        q, e = fp8.quantize_blocks(x, bool(square), True)
        slabs = Qt.view(-1, q.shape[1] // 64, 256, 64).permute(0, 2, 1, 3).reshape(-1, q.shape[1])
        assert torch.equal(slabs[:cols], q) and (slabs[cols:] == 99).all()


def test_backward_takes_the_matrix_by_rows_too():
    gen = torch.Generator().manual_seed(20)
    N, V, D = 70, 300, 130
    H, W, dY = values(gen, (N, D), "bf16", 0.5), values(gen, (V, D), "bf16", 0.5), values(gen, (N, V), "bf16")
    want = train(H, W, None, dY, "bf16")[1]
    Wt, Et = fp8.quantize_blocks(W, True, True)
    dH = torch.empty_like(H)
    ws = torch.empty(binding.lsr_fp8_backward_workspace_bytes(N, V, D, True, False, False), dtype=torch.uint8, device=DEV)
    binding.lsr_fp8_backward(N, V, D, lsr.LSR_BF16, lsr.LSR_BF16, dY, V, None, 0, Wt, Wt.shape[1], Et, dH, None, None, ws)
    assert torch.equal(dH, want)


def test_quantize_extremes():
    big, tiny = 3.4028234e38, 1e-45
    rows = [[0.0] * 128, [big] * 128, [tiny] * 128, [448.0, -448.0] * 64, [448.0001] + [1.0] * 127, [float("inf"), 3.0] + [0.5] * 126, [float("nan")] * 128,
            [1e-40, 2e-39] * 64, [1.0] * 64 + [-2.0 ** -20] * 64, [-0.0] * 128]
    x = torch.tensor(rows, device=DEV)
    with np.errstate(all="ignore"):
        want = orc.blocks(host(x), 1, 128)[0]
    for transposed in (False, True):
        q, e = fp8.quantize_blocks(x.t() if transposed else x, False, transposed)
        got = orc.unpack(q.cpu().numpy(), e.cpu().numpy(), 128)
        assert np.array_equal(got, want, equal_nan=True)
    q, e = fp8.quantize_blocks(x, True)
    assert np.array_equal(orc.unpack(q.cpu().numpy(), e.cpu().numpy(), 128), orc.blocks(host(x), 128, 128)[0], equal_nan=True)
    # every bfloat16 there is, in blocks of one power and of all
    x = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).to(DEV).view(512, 128)
    for y in (x, x.t().contiguous()):
        for square in (False, True):
            q, e = fp8.quantize_blocks(y, square)
            assert np.array_equal(orc.unpack(q.cpu().numpy(), e.cpu().numpy(), y.shape[1]), orc.blocks(host(y), 128 if square else 1, 128)[0], equal_nan=True)


# ---- the product ----

SIZES = [(1, 1, 1), (1, 1000, 8), (5, 300, 100), (31, 129, 312), (32, 1000, 1100), (33, 257, 128), (64, 255, 129), (129, 513, 640), (200, 31, 768), (300, 1000, 2700),
         (128, 256, 512), (2, 40, 65536), (3, 300, 4000), (40, 300, 65536), (1, 70000, 256), (257, 300, 576)]


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("N,V,K", SIZES)
def test_matmul_of_blocks(N, V, K, out):
    """Operands as bytes with exponents of their own for every row and block, result rows of a wider array."""
    gen = torch.Generator().manual_seed(N + 1000 * V + K)
    a, w = values(gen, (N, K), "f32"), values(gen, (V, K), "f32")
    (qa, ea), (qw, ew) = fp8.quantize_blocks(a), fp8.quantize_blocks(w)
    A, W = (orc.unpack(q.cpu().numpy(), e.cpu().numpy(), K) for q, e in ((qa, ea), (qw, ew)))
    bias = torch.randn(V, generator=gen).to(DEV)
    for b in (None, bias):
        wide = torch.full((N, V + 3), 7.0, dtype=TYPES[out], device=DEV)
        binding.lsr_fp8_matmul(N, V, K, lsr.LSR_E4M3, KIND[out], qa, qa.shape[1], ea, qw, qw.shape[1], ew, b, wide, V + 3, None)
        want = A @ W.T + (0 if b is None else host(b))
        close(host(wide[:, :V]), want, tolerance(A, W, want, out, None if b is None else host(b)), "out")
        assert (wide[:, V:] == 7).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V,K,pitch", [(1, 700, 768, 768), (5, 300, 100, 101), (20, 300, 1000, 1003), (32, 1100, 312, 320), (40, 300, 312, 313), (300, 700, 1024, 1024)])
def test_matmul_quantises_values_as_quantize_does(N, V, K, pitch, dtype):
    gen = torch.Generator().manual_seed(N + V)
    x, w = values(gen, (N, pitch), dtype)[:, :K], values(gen, (V, K), "f32")
    head = fp8.Fp8Head(w)
    qa, ea = fp8.quantize_blocks(x)
    for out in ("f32", "bf16"):
        want = torch.empty((N, V), dtype=TYPES[out], device=DEV)
        binding.lsr_fp8_matmul(N, V, K, lsr.LSR_E4M3, KIND[out], qa, qa.shape[1], ea, head.W8, head.W8.shape[1], head.exps, None, want, V, None)
        assert torch.equal(head.logits(x, TYPES[out]), want)


def test_rows_that_are_not_finite_show_in_their_logits_only():
    gen = torch.Generator().manual_seed(3)
    for N in (6, 140):
        h, w = values(gen, (N, 300), "f32", 0.5), values(gen, (400, 300), "f32", 0.5)
        clean = fp8.Fp8Head(w).logits(h)
        h[2, 5], h[4, 299] = float("inf"), float("nan")
        got = fp8.Fp8Head(w).logits(h)
        rest = [n for n in range(N) if n not in (2, 4)]
        assert torch.isnan(got[2]).all() and torch.isnan(got[4]).all()
        # (the other values of a block that holds an infinity keep their own scale; other rows do not see it)
        assert torch.equal(got[rest], clean[rest])
        h2, w2 = values(gen, (N, 300), "bf16", 0.5), w.clone()
        w2[7, 1] = float("-inf")
        got = fp8.Fp8Head(w2).logits(h2)
        assert torch.isnan(got[:, 7]).all() and not torch.isnan(got[:, :7]).any() and not torch.isnan(got[:, 8:]).any()


@pytest.mark.parametrize("N", [4, 100])
def test_blocks_of_extreme_magnitude(N):
    """Powers far apart that cancel in the product, blocks of zeros, powers at either end."""
    gen = torch.Generator().manual_seed(4)
    h, w = torch.randn(N, 512, generator=gen), torch.randn(300, 512, generator=gen)
    h[:, :128] *= 2.0 ** 100
    w[:, :128] *= 2.0 ** -100
    h[:, 128:256] *= 2.0 ** -60
    w[:, 128:256] *= 2.0 ** 60
    h[1:3, 256:384] = 0
    w[:128, 384:] = 0
    for out in ("f32", "bf16"):
        got = fp8.Fp8Head(w.to(DEV)).logits(h.to(DEV), TYPES[out])
        A, W = orc.blocks(h.numpy(), 1, 128)[0], orc.blocks(w.numpy(), 128, 128)[0]
        close(host(got), A @ W.T, tolerance(A, W, A @ W.T, out), out)


def test_offsets_beyond_32_bits():
    """A matrix and a result of more than 4 GiB each."""
    V, K, N = 2300000, 2048, 130
    q = torch.zeros((V, K), dtype=torch.uint8, device=DEV)
    e = torch.full((4, V, 4), 127, dtype=torch.uint8, device=DEV)
    at = torch.tensor([0, 1, 255, 2097151, 2097152, 2200003, V - 1], device=DEV)
    q[at] = 0x38                                      # ones
    e[3, at[-1], 3] = 128
    a = torch.ones(N, K, device=DEV)
    for out, rows in ((torch.float32, N), (torch.float32, 3)):
        y = torch.empty((rows, V), dtype=out, device=DEV)
        ws = torch.empty(binding.lsr_fp8_matmul_workspace_bytes(rows, V, K, lsr.LSR_F32), dtype=torch.uint8, device=DEV)
        binding.lsr_fp8_matmul(rows, V, K, lsr.LSR_F32, lsr.LSR_F32, a, K, None, q, K, e, None, y, V, ws)
        assert y.count_nonzero().item() == rows * len(at)
        assert (y[:, at[:-1]] == 2048).all() and (y[:, -1] == 2048 + 128).all()


# ---- the head ----

def test_head_shapes_views_and_largest_logits():
    gen = torch.Generator().manual_seed(5)
    w, bias = values(gen, (500, 200), "bf16", 0.5), torch.randn(500, generator=gen).to(DEV).to(torch.bfloat16)
    head = fp8.Fp8Head(w, bias)
    h = values(gen, (2 * 3 * 200, 2), "bf16", 0.5).t()[0].reshape(2, 3, 200)
    y = head.logits(h)
    assert y.shape == (2, 3, 500) and torch.equal(y, head.logits(h.contiguous()))
    assert torch.equal(head.logits(h[:, ::2]), y[:, ::2]) and head.logits(h[:, :0]).shape == (2, 0, 500)
    v, ids, lse = head.top_logits(h, 9, 2.0)
    v2, ids2, lse2 = distill.top_logits(y.reshape(-1, 500), 9, 2.0)
    assert torch.equal(v.reshape(-1, 9), v2) and torch.equal(ids.reshape(-1, 9), ids2) and torch.equal(lse.reshape(-1), lse2)
    for bad in (lambda: head.logits(h[..., :-1]), lambda: fp8.Fp8Head(w, bias[1:]), lambda: fp8.quantize_blocks(w[0])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: head.logits(h.half()), lambda: head.logits(h, torch.float16), lambda: fp8.quantize_blocks(w.int())):
        with pytest.raises(TypeError):
            bad()


# ---- training ----

def train(H, W, bias, dY, dtype):
    H, W = H.detach().requires_grad_(True), W.detach().requires_grad_(True)
    bias = None if bias is None else bias.detach().requires_grad_(True)
    y = fp8.fp8_logits(H, W, bias, TYPES[dtype])
    leaves = [H, W] + ([] if bias is None else [bias])
    return (y.detach(), *torch.autograd.grad(y, leaves, dY))


@pytest.mark.parametrize("dtype,out", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("N,V,D", [(1, 1, 8), (1, 300, 128), (7, 1000, 312), (33, 129, 100), (130, 515, 768), (513, 2500, 40), (300, 700, 1030)])
def test_training(N, V, D, dtype, out):
    gen = torch.Generator().manual_seed(N * 31 + V)
    H, W = values(gen, (N, D), dtype, 0.5), values(gen, (V, D), dtype, 0.5)
    bias = torch.randn(V, generator=gen).to(DEV)
    dY = values(gen, (N, V), out, 2.0)
    y, dH, dW, db = train(H, W, bias, dY, out)
    assert y.dtype == TYPES[out] and dH.dtype == dW.dtype == TYPES[dtype] and db.dtype == torch.float32
    h, w, g = host(H), host(W), host(dY)
    hq, wq, gq = orc.blocks(h, 1, 128)[0], orc.blocks(w, 128, 128)[0], orc.blocks(g, 1, 128)[0]
    ht, gt = orc.blocks(h, 128, 1)[0], orc.blocks(g, 128, 1)[0]
    want = hq @ wq.T + host(bias)
    close(host(y), want, tolerance(hq, wq, want, out, host(bias)), "logits")
    close(host(dH), gq @ wq, tolerance(gq, wq.T, gq @ wq, dtype), "dH")
    close(host(dW), gt.T @ ht, tolerance(gt.T, ht.T, gt.T @ ht, dtype), "dW")
    close(host(db), g.sum(axis=0), 8 * U * (np.sqrt(N) + 1) * np.abs(g).sum(axis=0), "db")


def test_training_where_the_contracted_axis_is_cut():
    """Few tiles and a long axis: partial sums joined by a second launch; repeated bits."""
    gen = torch.Generator().manual_seed(8)
    for N, V, D in ((50, 30000, 64), (4000, 90, 136)):
        H, W = values(gen, (N, D), "f32", 0.5), values(gen, (V, D), "f32", 0.5)
        dY = values(gen, (N, V), "f32", 1.0)
        got = train(H, W, None, dY, "f32")
        h, w, g = host(H), host(W), host(dY)
        wq, gq = orc.blocks(w, 128, 128)[0], orc.blocks(g, 1, 128)[0]
        ht, gt = orc.blocks(h, 128, 1)[0], orc.blocks(g, 128, 1)[0]
        close(host(got[1]), gq @ wq, tolerance(gq, wq.T, gq @ wq, "f32"), "dH")
        close(host(got[2]), gt.T @ ht, tolerance(gt.T, ht.T, gt.T @ ht, "f32"), "dW")
        for a, b in zip(got, train(H, W, None, dY, "f32")):
            assert torch.equal(a, b)


@pytest.mark.parametrize("N", [3, 200])
def test_gradients_by_differences(N):
    """Whole numbers of few bits are held exactly, so the logits are linear in every operand and differences are exact."""
    gen = torch.Generator().manual_seed(9)

    def small(*shape):
        return torch.randint(-4, 5, shape, generator=gen).float().to(DEV)
    H, W, bias, dY = small(N, 24), small(150, 24), small(150), small(N, 150)
    _, dH, dW, db = train(H, W, bias, dY, "f32")

    def f(h, w, b):
        return (fp8.fp8_logits(h, w, b).double() * dY.double()).sum().item()
    for k in range(12):
        i = torch.randint(0, N, (1,), generator=gen).item(), torch.randint(0, 24, (1,), generator=gen).item()
        j = torch.randint(0, 150, (1,), generator=gen).item(), torch.randint(0, 24, (1,), generator=gen).item()
        dh, dw, d = torch.zeros_like(H), torch.zeros_like(W), torch.zeros_like(bias)
        dh[i], dw[j], d[j[0]] = 1, 1, 1
        assert (f(H + dh, W, bias) - f(H - dh, W, bias)) / 2 == dH[i].item()
        assert (f(H, W + dw, bias) - f(H, W - dw, bias)) / 2 == dW[j].item()
        assert (f(H, W, bias + d) - f(H, W, bias - d)) / 2 == db[j[0]].item()


@pytest.mark.parametrize("need", [(True, False, False), (False, True, False), (False, False, True), (True, True, False), (False, True, True), (False, False, False)])
def test_gradients_that_are_wanted_only(need):
    gen = torch.Generator().manual_seed(10)
    full = None
    H, W, bias, dY = values(gen, (70, 200), "bf16", 0.5), values(gen, (300, 200), "bf16", 0.5), torch.randn(300, generator=gen).to(DEV), values(gen, (70, 300), "f32")
    full = train(H, W, bias, dY, "f32")[1:]
    leaves = [t.detach().requires_grad_(n) for t, n in zip((H, W, bias), need)]
    y = fp8.fp8_logits(*leaves)
    assert y.requires_grad == any(need)
    if any(need):
        got = iter(torch.autograd.grad(y, [t for t, n in zip(leaves, need) if n], dY))
        for n, g in zip(need, full):
            if n:
                assert torch.equal(next(got), g)


def test_shapes_types_and_views_in_training():
    gen = torch.Generator().manual_seed(11)
    H, W = values(gen, (2 * 3, 64), "bf16", 0.5).reshape(2, 3, 64), values(gen, (90, 64), "bf16", 0.5)
    bias = torch.randn(90, generator=gen).to(DEV).to(torch.bfloat16)
    y = fp8.fp8_logits(H, W, bias)
    assert y.shape == (2, 3, 90) and torch.equal(y, fp8.Fp8Head(W, bias).logits(H))
    # strided operands, a gradient that is broadcast, a bias of another type
    wide = torch.zeros(6, 100, dtype=torch.bfloat16, device=DEV)
    wide[:, :64] = H.reshape(6, 64)
    h, w, b = wide[:, :64].requires_grad_(True), W.t().contiguous().t().requires_grad_(True), bias.clone().requires_grad_(True)
    y2 = fp8.fp8_logits(h, w, b)
    assert torch.equal(y2, y.reshape(6, 90))
    y2.sum().backward()
    ones = train(H.reshape(6, 64), W, bias.float(), torch.ones(6, 90, device=DEV), "f32")
    assert torch.equal(h.grad, ones[1]) and torch.equal(w.grad, ones[2]) and b.grad.dtype == torch.bfloat16 and (b.grad == 6).all()
    # no rows at all
    h0 = torch.zeros(0, 64, dtype=torch.bfloat16, device=DEV, requires_grad=True)
    w0 = W.clone().requires_grad_(True)
    y0 = fp8.fp8_logits(h0, w0, bias)
    y0.sum().backward()
    assert y0.shape == (0, 90) and h0.grad.shape == (0, 64) and not w0.grad.any()
    for bad in (lambda: fp8.fp8_logits(H[..., :-1], W), lambda: fp8.fp8_logits(H, W[0]), lambda: fp8.fp8_logits(H, W, bias[1:])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: fp8.fp8_logits(H.float(), W), lambda: fp8.fp8_logits(H, W, bias, torch.float16)):
        with pytest.raises(TypeError):
            bad()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,V,D", [(1, 1, 1), (20, 700, 768), (33, 129, 100), (300, 1000, 312), (5, 300, 4000)])
def test_forward_is_quantize_and_matmul(N, V, D, dtype):
    gen = torch.Generator().manual_seed(N)
    H, W = values(gen, (N, D + 3), dtype, 0.5)[:, 1:D + 1], values(gen, (V, D + 5), dtype, 0.5)[:, 3:D + 3]
    bias = torch.randn(V, generator=gen).to(DEV)
    ws = torch.empty(binding.lsr_fp8_forward_workspace_bytes(N, V, D), dtype=torch.uint8, device=DEV)
    head = fp8.Fp8Head(W, bias)
    qt, et = fp8.quantize_blocks(W, True, True)
    for out in TYPES:
        for wide in (0, 32):
            Y = torch.full((N, V + 3), 7.0, dtype=TYPES[out], device=DEV)
            Wt = torch.full((D, qt.shape[1] + wide), 99, dtype=torch.uint8, device=DEV)
            Et = torch.zeros(et.numel(), dtype=torch.uint8, device=DEV)
            binding.lsr_fp8_forward(N, V, D, KIND[dtype], KIND[out], H, D + 3, W, D + 5, bias, Y, V + 3, *((Wt, Wt.shape[1], Et) if wide else (None, 0, None)), ws)
            assert torch.equal(Y[:, :V], head.logits(H, TYPES[out])) and (Y[:, V:] == 7).all()
            if wide:
                used = (V + 127) // 128
                assert torch.equal(Wt[:, :qt.shape[1]], qt) and (Wt[:, qt.shape[1]:] == 99).all()
                for b in range(used):
                    assert torch.equal(Et.view(-1, D, 4)[b // 4, :, b % 4], et[b // 4, :, b % 4])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_is_not_finite_in_training_shows_where_it_belongs(dtype):
    """A gradient, a token or a row of the matrix that is not finite: in its own rows and columns, and all else as without it but for the blocks that it shares."""
    gen = torch.Generator().manual_seed(21)
    N, V, D = 300, 517, 200
    H, W, dY = values(gen, (N, D), dtype, 0.0), values(gen, (V, D), dtype, 0.0), values(gen, (N, V), dtype, 0.0)
    H[7, 3], W[400, 150], dY[130, 20], dY[131, 21] = float("nan"), float("inf"), float("inf"), float("nan")
    y, dH, dW, db = train(H, W, torch.zeros(V, device=DEV), dY, dtype)
    h, w, g = host(H), host(W), host(dY)
    with np.errstate(invalid="ignore"):
        hq, wq, gq = orc.blocks(h, 1, 128)[0], orc.blocks(w, 128, 128)[0], orc.blocks(g, 1, 128)[0]
        ht, gt = orc.blocks(h, 128, 1)[0], orc.blocks(g, 128, 1)[0]
        for got, a, b in ((y, hq, wq), (dH, gq, wq.T), (dW, gt.T, ht.T)):
            want = a @ b.T
            got = host(got)
            assert np.array_equal(np.isnan(got), np.isnan(want)) and 0 < np.isnan(want).sum() < want.size
            fine = np.where(np.isnan(want), 0.0, want)
            close(np.where(np.isnan(got), 0.0, got), fine, tolerance(np.nan_to_num(a, nan=0.0), np.nan_to_num(b, nan=0.0), fine, dtype), "values")
        want = g.sum(axis=0)
    assert np.isinf(host(db)[20]) and np.isnan(host(db)[21]) and np.isfinite(np.delete(host(db), [20, 21])).all() and np.isnan(want[21])


def test_no_gradient_recorded():
    gen = torch.Generator().manual_seed(22)
    H, W = values(gen, (50, 64), "bf16").requires_grad_(True), values(gen, (90, 64), "bf16").requires_grad_(True)
    with torch.no_grad():
        y = fp8.fp8_logits(H, W)
    assert not y.requires_grad and torch.equal(y, fp8.fp8_logits(H, W).detach())


def test_second_derivatives_raise():
    gen = torch.Generator().manual_seed(12)
    H, W = values(gen, (5, 32), "f32", 0.5).requires_grad_(True), values(gen, (40, 32), "f32", 0.5).requires_grad_(True)
    dY = torch.ones(5, 40, device=DEV, requires_grad=True)
    dH, dW = torch.autograd.grad(fp8.fp8_logits(H, W), (H, W), dY, create_graph=True)
    for g in (dH, dW):
        for to in (H, W, dY):
            with pytest.raises(RuntimeError, match="not implemented"):
                torch.autograd.grad(g.sum(), to, retain_graph=True)


def test_matrix_changed_between_forward_and_backward():
    """The gradient belongs to the matrix that was multiplied."""
    gen = torch.Generator().manual_seed(13)
    H, W, dY = values(gen, (5, 32), "f32", 0.5), values(gen, (40, 32), "f32", 0.5), values(gen, (5, 40), "f32")
    want = train(H, W, None, dY, "f32")
    h, w = H.clone().requires_grad_(True), W.clone().requires_grad_(True)
    y = fp8.fp8_logits(h, w)
    with torch.no_grad():
        w.mul_(3)
    with pytest.raises(RuntimeError, match="modified by an inplace"):
        torch.autograd.grad(y, h, dY)
    assert want[1].shape == h.shape


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_repeats_its_bits_on_other_streams(dtype):
    gen = torch.Generator().manual_seed(14)
    jobs = [(values(gen, (n, 312), dtype, 0.5), values(gen, (v, 312), dtype, 0.5), values(gen, (n, v), dtype)) for n, v in ((3, 3000), (150, 2000), (700, 500))]
    want = [train(h, w, None, g, dtype) for h, w, g in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    got = []
    for s, (h, w, g) in zip(streams, jobs):
        with torch.cuda.stream(s):
            got.append(train(h, w, None, g, dtype))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
