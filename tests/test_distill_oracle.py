"""Pins of oracle/distill_oracle.py by things other than itself: pure-Python loops, hand-worked values, central differences."""
import math

import numpy as np
import pytest

from oracle import distill_oracle as orc


def test_quantize_by_hand():
    q, s = orc.quantize_rows([[1.0, -2.0, 0.5, 0.0], [0.0] * 4, [np.inf, 1, 2, 3], [np.nan, 1, 2, 3]])
    # half of the maximum is level 63.5: to the even 64; a quarter 31.75
    assert q[0].tolist() == [64.0, -127.0, 32.0, 0.0] and s[0] == 2.0 / 127
    assert not q[1].any() and s[1] == 0.0
    assert not q[2].any() and math.isnan(s[2]) and not q[3].any() and math.isnan(s[3])


def test_int8_product_by_loops():
    rng = np.random.default_rng(1)
    A, W = rng.integers(-127, 128, (3, 5)), rng.integers(-127, 128, (4, 5))
    a, w, b = rng.random(3), rng.random(4), rng.random(4)
    got = orc.int8_matmul(A, a, W, w, b)
    for n in range(3):
        for v in range(4):
            assert got[n, v] == pytest.approx(a[n] * w[v] * sum(int(A[n, k]) * int(W[v, k]) for k in range(5)) + b[v], rel=1e-14)


def test_top_logits_orders_ties_and_nan():
    x = [[1.0, 3.0, 3.0, -np.inf, 2.0], [np.inf, np.nan, 5.0, np.nan, 5.0], [-np.inf] * 5, [-0.0, 0.0, -1.0, 0.0, -0.0]]
    v, i, lse = orc.top_logits(x, 4, 2.0)
    assert i.tolist() == [[1, 2, 4, 0], [1, 3, 0, 2], [0, 1, 2, 3], [0, 1, 3, 4]]
    assert v[0].tolist() == [3, 3, 2, 1]
    assert lse[0] == pytest.approx(math.log(sum(math.exp(y / 2) for y in (1, 3, 3, 2))), rel=1e-14)
    assert math.isnan(lse[1]) and lse[2] == -np.inf


def _case(seed, N=4, D=8, V=11, K=3, given=True, mask=True):
    rng = np.random.default_rng(seed)
    H, W, b = rng.standard_normal((N, D)), rng.standard_normal((V, D)), rng.standard_normal(V)
    ids = np.stack([rng.permutation(V)[:K] for _ in range(N)])
    t = rng.standard_normal((N, K)) * 2
    lse = orc.log_sum_exp(t / 1.5) + 0.3 if given else None
    m = np.array([1, 0, 1, 1][:N]) if mask else None
    return H, W, b, ids, t, lse, m


@pytest.mark.parametrize("given", [False, True])
def test_loss_by_loops(given):
    H, W, b, ids, t, L, m = _case(3, given=given)
    ids[2, 1], t[3, 0] = -1, -np.inf          # padding of either kind
    got = orc.distill(H, W, b, ids, t, L, m, 1.5)
    for n in range(4):
        z = [(sum(H[n, d] * W[v, d] for d in range(8)) + b[v]) / 1.5 for v in range(11)]
        lse = math.log(sum(math.exp(y) for y in z))
        real = [(int(i), x / 1.5) for i, x in zip(ids[n], t[n]) if i >= 0 and x != -np.inf]
        norm = L[n] if given else math.log(sum(math.exp(x) for _, x in real))
        want = sum(math.exp(x - norm) * (x - norm - z[i] + lse) for i, x in real)
        assert got["loss"][n] == pytest.approx(want if m[n] else 0.0, rel=1e-12, abs=1e-14)
        assert got["lse"][n] == pytest.approx(lse if m[n] else 0.0, rel=1e-12)


def test_a_teacher_that_the_student_equals_has_no_loss_and_no_gradient():
    H, W, b, *_ = _case(5)
    z = H @ W.T + b
    ids = np.tile(np.arange(11), (4, 1))
    got = orc.distill(H, W, b, ids, z, None, None, 1.0, np.ones(4))
    assert np.abs(got["loss"]).max() < 1e-13
    assert max(np.abs(got[k]).max() for k in ("dH", "dW", "db")) < 1e-12


@pytest.mark.parametrize("given", [False, True])
def test_gradients_by_differences(given):
    H, W, b, ids, t, L, m = _case(7, given=given)
    ids[0, 2] = ids[0, 0]                      # an id that comes twice counts twice
    ids[3] = -1                                # a row without a teacher
    rng = np.random.default_rng(9)
    dloss = rng.standard_normal(4)
    got = orc.distill(H, W, b, ids, t, L, m, 1.5, dloss)

    def f(H, W, b):
        return float((orc.distill(H, W, b, ids, t, L, m, 1.5)["loss"] * dloss).sum())

    eps = 1e-5
    for name, x in (("dH", H), ("dW", W), ("db", b)):
        args = {"dH": 0, "dW": 1, "db": 2}[name]
        for flat in rng.permutation(x.size)[:20]:
            at = np.unravel_index(flat, x.shape)
            parts = []
            for sign in (1, -1):
                y = [H.copy(), W.copy(), b.copy()]
                y[args][at] += sign * eps
                parts.append(f(*y))
            # central difference: error of order eps^2 times the third derivative, and rounding 1e-16 / eps
            assert (parts[0] - parts[1]) / (2 * eps) == pytest.approx(got[name][at], rel=1e-6, abs=1e-8)


def test_a_masked_bias_excludes_an_entry():
    H, W, b, ids, t, L, m = _case(11, mask=False)
    keep = np.array([v for v in range(11) if v != 6])
    ids = np.where(ids == 6, 5, ids)
    b2 = b.copy()
    b2[6] = -np.inf
    got = orc.distill(H, W, b2, ids, t, L, None, 1.0, np.ones(4))
    place = {int(v): i for i, v in enumerate(keep)}
    want = orc.distill(H, W[keep], b[keep], np.vectorize(place.get)(ids), t, L, None, 1.0, np.ones(4))
    assert np.allclose(got["loss"], want["loss"], rtol=1e-13) and np.allclose(got["dW"][keep], want["dW"], rtol=1e-12, atol=1e-15)
    assert not got["dW"][6].any() and got["db"][6] == 0.0
