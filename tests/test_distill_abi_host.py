"""Host-side checks of the operators around the dense logits that need no GPU: refusals come before any device work."""
import os

import pytest
import torch

import paper_2603_25011_amd as lsr
from paper_2603_25011_amd import binding, distill

P = 1 << 20          # an aligned address that is never dereferenced
WS = (P, 1 << 40)


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(lsr.library_path()):
        from paper_2603_25011_amd import build
        build.build()
    return lsr.load_library()


def status(f, *args, **kw):
    with pytest.raises(lsr.LsrError) as e:
        f(*args, stream=0, **kw)
    return e.value.status


NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, ARCH = 1, 2, 3, 4, 5, 6


def test_int8_row_bytes():
    assert [lsr.lsr_int8_row_bytes(c) for c in (1, 128, 129, 768, 312, 65536)] == [128, 128, 256, 768, 384, 65536]
    assert lsr.lsr_int8_row_bytes(0) == 0 and lsr.lsr_int8_row_bytes(65537) == 0 and lsr.lsr_int8_row_bytes(-1) == 0


def test_quantize_refusals():
    def q(rows=4, cols=100, dtype=lsr.LSR_BF16, X=P, ldx=100, Q=P, ldq=128, scale=P):
        return status(lsr.lsr_quantize_rows, rows, cols, dtype, X, ldx, Q, ldq, scale)
    assert q(dtype=lsr.LSR_I8) == DTYPE and q(dtype=9) == DTYPE
    assert q(rows=0) == SHAPE and q(rows=1 << 31) == SHAPE and q(cols=0) == SHAPE and q(cols=65537, ldx=65537, ldq=1 << 20) == SHAPE
    assert q(ldx=99) == SHAPE and q(ldq=112) == SHAPE
    assert q(X=None) == NULL and q(Q=None) == NULL and q(scale=None) == NULL
    assert q(X=P + 1) == ALIGN and q(Q=P + 8) == ALIGN and q(ldq=136) == ALIGN and q(scale=P + 2) == ALIGN


def test_int8_matmul_refusals():
    def m(N=100, V=300, K=100, a=lsr.LSR_BF16, o=lsr.LSR_F32, A=P, lda=100, sa=None, W=P, ldw=128, sw=P, bias=P, out=P, ldo=300, ws=WS):
        return status(lsr.lsr_int8_matmul, N, V, K, a, o, A, lda, sa, W, ldw, sw, bias, out, ldo, ws)
    assert m(a=7) == DTYPE and m(o=lsr.LSR_I8) == DTYPE and m(sa=P) == DTYPE
    for bad in ({"N": 0}, {"V": 0}, {"K": 0}, {"K": 65537, "lda": 65537, "ldw": 1 << 17}, {"N": 1 << 31}, {"V": 1 << 31, "ldo": 1 << 32},
                {"lda": 99}, {"ldw": 112}, {"ldo": 299}, {"ldw": (1 << 23) + 16}, {"N": 1 << 30, "V": 1 << 30, "ldo": 1 << 30}):
        assert m(**bad) == SHAPE, bad
    assert m(a=lsr.LSR_I8, sa=P, lda=112) == SHAPE and m(a=lsr.LSR_I8, sa=P, lda=(1 << 23) + 16) == SHAPE
    assert m(A=None) == NULL and m(W=None) == NULL and m(sw=None) == NULL and m(out=None) == NULL and m(a=lsr.LSR_I8, lda=128) == NULL
    assert m(A=P + 1) == ALIGN and m(W=P + 4) == ALIGN and m(ldw=136) == ALIGN and m(sw=P + 1) == ALIGN and m(bias=P + 2) == ALIGN
    assert m(out=P + 2) == ALIGN and m(a=lsr.LSR_I8, sa=P, lda=136) == ALIGN
    need = lsr.lsr_int8_matmul_workspace_bytes(100, 300, 100, lsr.LSR_BF16)
    assert need >= 100 * 128 + 400
    assert m(ws=None) == WORKSPACE and m(ws=(P, need - 1)) == WORKSPACE and m(ws=(P + 8, need)) == ALIGN
    assert lsr.lsr_int8_matmul_workspace_bytes(100, 300, 100, lsr.LSR_I8) == 0 and lsr.lsr_int8_matmul_workspace_bytes(0, 300, 100, 0) == 0


def test_top_logits_refusals():
    def t(rows=4, V=50000, K=8, dtype=lsr.LSR_F32, T=1.0, X=P, ldx=50000, values=P, ids=P, lse=P, ws=WS):
        return status(lsr.lsr_top_logits, rows, V, K, dtype, T, X, ldx, values, ids, lse, ws)
    assert t(dtype=lsr.LSR_I8) == DTYPE
    for bad in ({"rows": 0}, {"K": 0}, {"K": 257}, {"V": 7, "ldx": 7}, {"ldx": 49999}, {"V": 1 << 31, "ldx": 1 << 31}, {"T": 0.0}, {"T": -1.0},
                {"T": float("inf")}, {"T": float("nan")}, {"T": 1e-42}):
        assert t(**bad) == SHAPE, bad
    assert t(X=None) == NULL and t(values=None) == NULL and t(ids=None) == NULL
    assert t(X=P + 2) == ALIGN and t(values=P + 2) == ALIGN and t(ids=P + 1) == ALIGN and t(lse=P + 2) == ALIGN
    need = lsr.lsr_top_logits_workspace_bytes(4, 50000, 8)
    assert need > 0 and t(ws=(P, need - 1)) == WORKSPACE and t(ws=None) == WORKSPACE and t(ws=(P + 8, need)) == ALIGN
    assert lsr.lsr_top_logits_workspace_bytes(1 << 20, 50000, 8) == 0        # enough rows: no row is cut
    assert lsr.lsr_top_logits_workspace_bytes(0, 50000, 8) == 0
    # a joining launch never has more keys than it holds, and scratch stays small
    for rows in (1, 3, 100, 2047):
        for K in (1, 7, 64, 256):
            assert lsr.lsr_top_logits_workspace_bytes(rows, 250002, K) <= 4096 * (K * 8 + 8) + 256


def test_distill_refusals():
    base = dict(N=64, D=768, V=30522, K=8, dt=lsr.LSR_BF16, T=1.0)

    def args(kw):
        k = {**base, **kw}
        return [k[x] for x in ("N", "D", "V", "K", "dt", "T")]

    names_f = ["H", "W", "bias", "ids", "logits", "tlse", "mask", "loss", "lse"]
    names_b = ["H", "W", "bias", "ids", "logits", "tlse", "mask", "lse", "dloss", "dH", "dW", "db"]

    def call(f, names, ws=WS, **kw):
        return status(f, *args(kw), *[kw.get(n, P) for n in names], ws)

    for f, names, back, needed in ((lsr.lsr_distill_forward, names_f, False, {"H", "W", "bias", "ids", "logits", "loss", "lse"}),
                                   (lsr.lsr_distill_backward, names_b, True, {"H", "W", "bias", "ids", "logits", "lse", "dloss"})):
        assert call(f, names, dt=lsr.LSR_I8) == DTYPE
        for bad in ({"N": 0}, {"N": (1 << 22) + 1}, {"D": 0}, {"D": 12}, {"D": 8200}, {"V": 0}, {"V": (1 << 21) + 1}, {"K": 0}, {"K": 257},
                    {"T": 0.0}, {"T": float("nan")}, {"T": float("inf")}, {"T": 1e-42}):
            assert call(f, names, **bad) == SHAPE, bad
            assert lsr.lsr_distill_workspace_bytes(*args(bad), back) == 0
        for n in needed:
            assert call(f, names, **{n: None}) == NULL, n
        for n in names:
            assert call(f, names, **{n: P + 4}) == ALIGN, n
        need = lsr.lsr_distill_workspace_bytes(*args({}), back)
        assert call(f, names, ws=None) == WORKSPACE and call(f, names, ws=(P, need - 1)) == WORKSPACE and call(f, names, ws=(P + 4, need)) == ALIGN


def test_distill_workspace_is_bounded():
    f = lsr.lsr_distill_workspace_bytes
    # nothing of the size of the logits in the forward, at most two pieces of 2^28 + 256 N bfloat16 in the backward
    N, D, V, K = 16384, 768, 30522, 64
    assert f(N, D, V, K, lsr.LSR_BF16, 1.0, False) < N * V // 4
    assert f(N, D, V, K, lsr.LSR_BF16, 1.0, True) < 4 * ((1 << 28) + 256 * N) + 16 * N * (D + K + V // 32) * 4
    N = 1 << 17
    assert f(N, 1024, 250002, K, lsr.LSR_BF16, 1.0, True) < 4 * ((1 << 28) + 256 * N) + 16 * N * (1024 + K + 250002 // 32) + 8 * 250002 * 1024


def test_launches_stay_below_their_limits():
    assert status(lsr.lsr_quantize_rows, 1 << 26, 100, lsr.LSR_BF16, P, 100, P, 128, P) == SHAPE
    assert status(lsr.lsr_int8_matmul, 1 << 20, 1 << 18, 100, lsr.LSR_BF16, lsr.LSR_F32, P, 100, None, P, 128, P, P, P, 1 << 18, WS) == SHAPE
    assert lsr.lsr_top_logits_workspace_bytes(1 << 23, 50000, 8) == 0
    assert status(lsr.lsr_top_logits, 1 << 23, 50000, 8, lsr.LSR_F32, 1.0, P, 50000, P, P, P, WS) == SHAPE
    for n, d, v in ((1 << 20, 768, 1 << 18), (1 << 21, 4096, 1000)):
        assert lsr.lsr_distill_workspace_bytes(n, d, v, 8, lsr.LSR_BF16, 1.0, False) == 0
    assert lsr.lsr_distill_workspace_bytes((1 << 20) - 1, 768, 1 << 18, 8, lsr.LSR_BF16, 1.0, False) > 0


def test_no_cpu_path_and_wrong_types():
    x = torch.zeros(4, 64)
    with pytest.raises(RuntimeError):
        distill.quantize_rows(x)
    with pytest.raises(RuntimeError):
        distill.top_logits(x, 2)
    with pytest.raises(RuntimeError):
        distill.Int8Head(x)
    with pytest.raises(RuntimeError):
        distill.lsr_distill(x, torch.zeros(9, 64), torch.zeros(9), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2))
