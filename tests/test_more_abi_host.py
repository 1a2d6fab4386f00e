"""Host-side checks of the head in 8-bit floating point, the beam search and dropout that need no GPU: refusals come before any device work."""
import os

import pytest
import torch

import paper_2603_25011_amd as lsr
from paper_2603_25011_amd import beam, binding, dropout, fp8

P = 1 << 20          # an aligned address that is never dereferenced
WS = (P, 1 << 60)
NULL, SHAPE, DTYPE, ALIGN, WORKSPACE, ARCH = 1, 2, 3, 4, 5, 6


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


def test_sizes_of_rows_and_exponents():
    f = binding.lsr_fp8_row_bytes
    assert [f(c) for c in (1, 128, 129, 768, 312, 1 << 22)] == [128, 128, 256, 768, 384, 1 << 22] and f(0) == f(-1) == f((1 << 22) + 1) == 0
    g = binding.lsr_fp8_exp_bytes
    assert g(3, 1) == g(3, 512) == 12 and g(3, 513) == 24 and g(0, 1) == g(1, 0) == g(1 << 22, 1 << 22) == 0


def test_fp8_quantize_refusals():
    def q(rows=40, cols=300, dtype=lsr.LSR_BF16, X=P, ldx=300, square=0, Q=P, ldq=384, E=P, Qt=P, ldqt=128, Et=P):
        return status(binding.lsr_fp8_quantize, rows, cols, dtype, X, ldx, square, Q, ldq, E, Qt, ldqt, Et)
    assert q(dtype=lsr.LSR_I8) == DTYPE and q(dtype=3) == DTYPE
    for bad in ({"rows": 0}, {"cols": 0}, {"rows": (1 << 22) + 1}, {"cols": (1 << 22) + 1, "ldx": 1 << 23}, {"rows": 1 << 20, "cols": 1 << 20, "ldx": 1 << 20},
                {"ldx": 299}, {"ldq": 368}, {"ldqt": 112}):
        assert q(**bad) == SHAPE, bad
    assert q(X=None) == NULL and q(Q=None, Qt=None) == NULL and q(E=None) == NULL and q(Et=None) == NULL
    assert q(X=P + 1) == ALIGN and q(Q=P + 8) == ALIGN and q(Qt=P + 4) == ALIGN and q(E=P + 2) == ALIGN and q(Et=P + 1) == ALIGN
    assert q(ldq=392) == ALIGN and q(ldqt=136) == ALIGN


def test_fp8_matmul_refusals():
    def m(N=100, V=300, K=100, a=lsr.LSR_BF16, o=lsr.LSR_F32, A=P, lda=100, ea=None, W=P, ldw=128, ew=P, bias=P, out=P, ldo=300, ws=WS):
        return status(binding.lsr_fp8_matmul, N, V, K, a, o, A, lda, ea, W, ldw, ew, bias, out, ldo, ws)
    assert m(a=lsr.LSR_I8) == DTYPE and m(o=3) == DTYPE and m(o=lsr.LSR_I8) == DTYPE and m(ea=P) == DTYPE
    for bad in ({"N": 0}, {"V": 0}, {"K": 0}, {"K": 65537, "lda": 65537, "ldw": 1 << 17}, {"N": (1 << 22) + 1}, {"V": (1 << 22) + 1, "ldo": 1 << 23},
                {"lda": 99}, {"ldw": 112}, {"ldo": 299}, {"ldw": (1 << 23) + 16}, {"N": 1 << 20, "V": 1 << 20, "ldo": 1 << 20}):
        assert m(**bad) == SHAPE, bad
    assert m(a=3, ea=P, lda=112) == SHAPE and m(a=3, ea=P, lda=(1 << 23) + 16) == SHAPE
    assert m(A=None) == NULL and m(W=None) == NULL and m(ew=None) == NULL and m(out=None) == NULL and m(a=3, lda=128) == NULL
    assert m(A=P + 1) == ALIGN and m(W=P + 4) == ALIGN and m(ldw=136) == ALIGN and m(ew=P + 1) == ALIGN and m(bias=P + 2) == ALIGN
    assert m(out=P + 2) == ALIGN and m(a=3, ea=P, lda=136) == ALIGN and m(a=3, ea=P + 2, lda=128) == ALIGN and m(a=3, A=P + 8, ea=P, lda=128) == ALIGN
    need = binding.lsr_fp8_matmul_workspace_bytes(100, 300, 100, lsr.LSR_BF16)
    assert need >= 100 * 132 and m(ws=None) == WORKSPACE and m(ws=(P, need - 1)) == WORKSPACE and m(ws=(P + 8, need)) == ALIGN
    assert binding.lsr_fp8_matmul_workspace_bytes(100, 300, 100, 3) == 0 and binding.lsr_fp8_matmul_workspace_bytes(0, 300, 100, 0) == 0


def test_fp8_forward_refusals():
    def f(N=100, V=300, D=100, h=lsr.LSR_BF16, o=lsr.LSR_F32, H=P, ldh=100, W=P, ldw=100, bias=P, out=P, ldo=300, Wt=P, ldwt=384, et=P, ws=WS):
        return status(binding.lsr_fp8_forward, N, V, D, h, o, H, ldh, W, ldw, bias, out, ldo, Wt, ldwt, et, ws)
    assert f(h=3) == f(h=lsr.LSR_I8) == f(o=3) == DTYPE
    for bad in ({"N": 0}, {"V": 0}, {"D": 0}, {"D": 65537, "ldh": 65537, "ldw": 65537}, {"ldh": 99}, {"ldw": 99}, {"ldo": 299}, {"ldwt": 368},
                {"N": 1 << 20, "V": 1 << 20, "ldo": 1 << 20, "ldwt": 0}, {"N": 1 << 22, "D": 1 << 15, "ldh": 1 << 15, "ldw": 1 << 15},
                {"N": 40, "V": 1 << 22, "ldo": 1 << 22, "D": 1 << 15, "ldh": 1 << 15, "ldw": 1 << 15, "ldwt": 0}):
        assert f(**bad) == SHAPE, bad
    assert f(H=None) == f(W=None) == f(out=None) == f(et=None) == NULL
    assert f(H=P + 1) == f(W=P + 1) == f(bias=P + 2) == f(out=P + 2) == f(Wt=P + 8) == f(ldwt=392) == f(et=P + 2) == f(h=lsr.LSR_F32, W=P + 2) == ALIGN
    g = binding.lsr_fp8_forward_workspace_bytes
    need = g(100, 300, 100)
    assert need >= 400 * 132 and f(ws=None) == WORKSPACE and f(ws=(P, need - 1)) == WORKSPACE and f(ws=(P + 8, need)) == ALIGN
    assert g(0, 300, 100) == g(100, 300, 65537) == 0 and g(1, 300, 100) >= 300 * 132


def test_fp8_backward_refusals():
    def b(N=100, V=300, D=100, y=lsr.LSR_BF16, h=lsr.LSR_BF16, dY=P, ldy=300, H=P, ldh=100, Wt=P, ldwt=384, et=P, dH=P, dW=P, db=P, ws=WS):
        return status(binding.lsr_fp8_backward, N, V, D, y, h, dY, ldy, H, ldh, Wt, ldwt, et, dH, dW, db, ws)
    assert b(y=3) == DTYPE and b(h=lsr.LSR_I8) == DTYPE
    for bad in ({"N": 0}, {"V": 0}, {"D": 0}, {"D": 65537, "ldh": 65537}, {"ldy": 299}, {"ldh": 99}, {"ldwt": 368}, {"ldwt": (1 << 23) + 16},
                {"N": 1 << 20, "V": 1 << 20, "ldy": 1 << 20}, {"N": 1 << 22, "D": 1 << 15, "ldh": 1 << 15}, {"V": 1 << 22, "ldy": 1 << 22, "D": 1 << 15, "ldh": 1 << 15, "ldwt": 0}):
        assert b(**bad) == SHAPE, bad
    assert b(dY=None) == NULL and b(H=None) == NULL and b(Wt=None) == NULL and b(et=None) == NULL and b(dH=None, dW=None, db=None) == NULL
    assert b(dY=P + 1) == ALIGN and b(H=P + 1) == ALIGN and b(Wt=P + 8) == ALIGN and b(ldwt=392) == ALIGN and b(et=P + 2) == ALIGN
    assert b(dH=P + 8) == ALIGN and b(dW=P + 4) == ALIGN and b(db=P + 2) == ALIGN
    need = binding.lsr_fp8_backward_workspace_bytes(100, 300, 100)
    assert b(ws=None) == WORKSPACE and b(ws=(P, need - 1)) == WORKSPACE and b(ws=(P + 8, need)) == ALIGN
    some = [binding.lsr_fp8_backward_workspace_bytes(100, 300, 100, *(i == j for j in range(3))) for i in range(3)]
    assert 0 < some[0] < need and 0 < some[1] < need and some[2] == 0 < binding.lsr_fp8_backward_workspace_bytes(129, 300, 100, False, False, True)


def test_beam_select_refusals():
    def s(B=4, beams=5, V=50000, K=10, dtype=lsr.LSR_F32, T=1.0, X=P, ldx=50000, scores=P, fin=P, end=2, os=P, ob=P, ot=P, ws=WS):
        return status(binding.lsr_beam_select, B, beams, V, K, dtype, T, X, ldx, scores, fin, end, os, ob, ot, ws)
    assert s(dtype=lsr.LSR_I8) == DTYPE
    for bad in ({"B": 0}, {"beams": 0}, {"beams": 65}, {"V": 0}, {"K": 0}, {"K": 129}, {"V": 1, "ldx": 1, "K": 6, "end": 0}, {"ldx": 49999}, {"end": -1},
                {"end": 50000}, {"T": 0.0}, {"T": -1.0}, {"T": float("inf")}, {"T": float("nan")}, {"T": 1e-42}, {"B": 1 << 22}, {"V": 1 << 31, "ldx": 1 << 31}):
        assert s(**bad) == SHAPE, bad
    assert s(X=None) == NULL and s(scores=None) == NULL and s(os=None) == NULL and s(ob=None) == NULL and s(ot=None) == NULL
    assert s(X=P + 2) == ALIGN and s(dtype=lsr.LSR_BF16, X=P + 1) == ALIGN and s(scores=P + 2) == ALIGN and s(os=P + 1) == ALIGN and s(ob=P + 2) == ALIGN
    assert s(ot=P + 2) == ALIGN
    f = binding.lsr_beam_select_workspace_bytes
    need = f(4, 5, 50000, 10)
    assert need > 0 and s(ws=None) == WORKSPACE and s(ws=(P, need - 1)) == WORKSPACE and s(ws=(P + 8, need)) == ALIGN
    # a joining launch never has more keys of a sequence than it holds
    for beams in (1, 7, 64):
        for K in (1, 16, 128):
            for B in (1, 30, 3000):
                assert f(B, beams, 250002, K) <= B * (max(8192, beams * K) * 8 + 64 * beams * 16) + 256


def test_beam_reorder_refusals():
    good = (P, P + (1 << 24), 64, 16, 16, 64, 16, 16, 1, 16)

    def r(B=4, beams=4, K=4, parents=P, states=(good,)):
        return status(binding.lsr_beam_reorder, B, beams, K, parents, list(states))

    def but(**kw):
        names = ("src", "dst", "src_batch", "src_beam", "src_piece", "dst_batch", "dst_beam", "dst_piece", "pieces", "piece_bytes")
        return [tuple(kw.get(n, v) for n, v in zip(names, good))]
    assert r(B=0) == r(beams=0) == r(K=0) == r(B=1 << 20, K=1 << 20) == r(states=[good] * 4097) == SHAPE
    assert r(parents=None) == NULL and r(states=but(src=None)) == NULL and r(states=but(dst=None)) == NULL and r(parents=P + 2) == ALIGN
    for bad in ({"pieces": 0}, {"piece_bytes": 0}, {"pieces": 1 << 20, "piece_bytes": 1 << 20}, {"src_batch": -1}, {"dst_piece": -1}, {"src_beam": -16}):
        assert r(states=[good] + but(**bad)) == SHAPE, bad
    # more single bytes than a launch has threads for, behind an array that is in order: nothing is enqueued before the refusal
    odd = dict(src=P + 1, src_batch=1 << 31, src_beam=1 << 30, dst_batch=1 << 31, dst_beam=1 << 30, piece_bytes=(1 << 30) + 1)
    assert r(B=16, states=[good] * 40 + but(**odd)) == SHAPE


def test_dropout_refusals():
    def d(n=100, dtype=lsr.LSR_BF16, X=P, Y=P, p=0.1, seed=1, offset=2, state=None):
        return status(binding.lsr_dropout, n, dtype, X, Y, p, seed, offset, state)
    assert d(dtype=lsr.LSR_I8) == DTYPE
    assert d(n=0) == d(n=1 << 40) == d(p=-0.1) == d(p=1.01) == d(p=float("nan")) == SHAPE
    assert d(X=None) == d(Y=None) == NULL
    assert d(X=P + 1) == d(Y=P + 1) == d(state=P + 4) == d(dtype=lsr.LSR_F32, X=P + 2) == ALIGN


@pytest.mark.parametrize("f", [lambda x: fp8.quantize_blocks(x), lambda x: fp8.Fp8Head(x), lambda x: fp8.fp8_logits(x, x),
                               lambda x: beam.beam_select(x[None], x[:1], 1), lambda x: dropout.dropout(x, 0.1),
                               lambda x: beam.beam_reorder([x], torch.zeros(4, 8, dtype=torch.int32))])
def test_cpu_tensors_are_refused(f):
    with pytest.raises(RuntimeError, match="no CPU path"):
        f(torch.zeros(4, 8))


def test_parents_that_are_no_int32_matrix_are_refused():
    for bad in (torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32), torch.zeros(4, 8, dtype=torch.int64)):
        with pytest.raises(ValueError, match="int32"):
            beam.beam_reorder([torch.zeros(4, 8)], bad)


@pytest.mark.parametrize("shape,view,want", [
    ((3, 4, 5), lambda x: x, (80, 20, 20, 1, 20)),
    ((3, 4), lambda x: x, (16, 4, 4, 1, 4)),
    ((3, 4, 5, 6, 7), lambda x: x[:, :, :, :2], (3360, 840, 168, 5, 56)),
    ((3, 4, 5, 6, 7), lambda x: x[:, :, 1:3], (3360, 840, 336, 1, 336)),
    ((3, 4, 6, 1), lambda x: x.transpose(2, 3), (96, 24, 24, 1, 24)),
    ((3, 4, 6), lambda x: x.transpose(0, 1), (24, 96, 24, 1, 24)),
    ((3, 4, 6, 5), lambda x: x[:, :, ::2, ::2], None),
    ((3, 4, 6, 5), lambda x: x[..., 1], (480, 120, 20, 6, 4)),
    ((3, 1, 6), lambda x: x.expand(3, 4, 6), (24, 0, 24, 1, 24)),
])
def test_layouts_of_states(shape, view, want):
    x = view(torch.zeros(shape))
    got = beam._layout(x)
    if want is None:
        assert got is None
        return
    assert (got[0], got[1]) == (want[0], want[1]) and got[3] * got[4] == want[3] * want[4]
    if got[3] > 1:
        assert got[2:] == want[2:]


def test_tensors_that_overlap_themselves_are_seen():
    x = torch.zeros(3, 4, 5)
    assert beam._once(x) and beam._once(x[:, ::2, 1:]) and beam._once(x.transpose(0, 1))
    assert not beam._once(x[:, :1].expand(3, 4, 5)) and not beam._once(x.as_strided((3, 4, 5), (5, 5, 1)))
