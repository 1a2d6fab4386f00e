"""Pins of the definitions in oracle/fp8_oracle.py, oracle/beam_oracle.py and oracle/dropout_oracle.py: hand-worked values, published answers, loops, differences."""
import math

import numpy as np
import pytest

from oracle import beam_oracle, dropout_oracle, fp8_oracle


def test_e4m3_table():
    t = fp8_oracle.TABLE
    assert len(t) == 127 and t[0] == 0 and t[1] == 2.0 ** -9 and t[8] == 2.0 ** -6 and t[0x38] == 1.0 and t[126] == 448.0 and (np.diff(t) > 0).all()
    assert list(fp8_oracle.decode([0x38, 0xb8, 0x7e, 0x00])) == [1.0, -1.0, 448.0, 0.0] and np.isnan(fp8_oracle.decode([0x7f, 0xff])).all()


@pytest.mark.parametrize("x,want", [(1.0625, 1.0), (1.1875, 1.25), (-1.0625, 1.0), (1.06251, 1.125), (448.0, 448.0), (2.0 ** -10, 0.0), (1.5 * 2.0 ** -9, 2.0 ** -8),
                                    (2.0 ** -10 * 1.001, 2.0 ** -9), (0.0, 0.0), (17.0, 16.0), (19.0, 20.0)])
def test_rounding_by_hand(x, want):
    assert fp8_oracle.TABLE[fp8_oracle.nearest(x)] == want


@pytest.mark.parametrize("most,e", [(448.0, 0), (448.1, 1), (224.0, -1), (1.75, -8), (1.7500001, -7), (1.0, -8), (0.0, -127), (2.0 ** -149, -127), (3.4e38, 120),
                                    (1.75 * 2.0 ** 127, 119)])
def test_exponents_by_hand(most, e):
    assert fp8_oracle.exponent(most) == e


def test_blocks_hold_what_they_say():
    rng = np.random.default_rng(0)
    X = rng.standard_normal((130, 200)) * np.exp(rng.standard_normal((130, 200)))
    for rows, cols in ((1, 128), (128, 1), (128, 128)):
        v, e = fp8_oracle.blocks(X, rows, cols)
        assert (np.abs(v - X) <= np.maximum(2.0 ** -4 * np.abs(X), 2.0 ** (e - 10.0))).all()
        assert (e[:rows, :cols] == e[0, 0]).all()
        assert np.array_equal(fp8_oracle.blocks(v, rows, cols)[0], v)
    assert np.array_equal(fp8_oracle.blocks(X.T, 1, 128)[0], fp8_oracle.blocks(X, 128, 1)[0].T)


def test_gradients_are_those_of_the_product_where_nothing_is_rounded():
    rng = np.random.default_rng(1)
    H, W, dY = (rng.integers(-8, 9, s).astype(float) for s in ((5, 7), (6, 7), (5, 6)))
    dH, dW, db = fp8_oracle.gradients(H, W, dY)
    for x, g in ((H, dH), (W, dW)):
        d = np.zeros_like(x)
        for i in np.ndindex(x.shape):
            for sign in (1, -1):
                x[i] += sign
                d[i] += sign * (fp8_oracle.logits(H, W) * dY).sum() / 2
                x[i] -= sign
        assert np.allclose(d, g, rtol=0, atol=1e-9)
    assert np.array_equal(db, dY.sum(axis=0))


def test_selection_by_hand():
    # two beams, three tokens of probabilities 1/2, 1/4, 1/4 and 1/4, 1/4, 1/2
    X = np.log(np.array([[[0.5, 0.25, 0.25], [0.25, 0.25, 0.5]]]))
    s, m, t = beam_oracle.select(X, [[0.0, math.log(0.5)]], 4)
    assert np.allclose(np.exp(s), [[0.5, 0.25, 0.25, 0.25]]) and m.tolist() == [[0, 0, 0, 1]] and t.tolist() == [[0, 1, 2, 2]]
    # a finished beam, excluded tokens, too few continuations
    X[0, 1, 1:] = -np.inf
    s, m, t = beam_oracle.select(X, [[0.0, math.log(0.5)]], 4, finished=[[True, False]], end_id=2)
    assert np.allclose(np.exp(s), [[1.0, 0.5, 0.0, 0.0]]) and m.tolist() == [[0, 1, 0, 0]] and t.tolist() == [[2, 0, 2, 2]]
    X[0, 1, 0] = np.nan
    s, m, t = beam_oracle.select(X, [[0.0, 0.0]], 2, end_id=1)
    assert np.isnan(s).all() and m.tolist() == [[1, 1]] and t.tolist() == [[1, 1]]


def test_philox_published_answers():
    # known answers that its authors publish with the generator: counter and key of zeros, of ones, and of digits of pi
    assert dropout_oracle.philox([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    ones = 0xFFFFFFFF
    assert dropout_oracle.philox([ones] * 4, [ones] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert dropout_oracle.philox([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0]) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]


def test_dropout_numbers():
    words = dropout_oracle.philox([3, 0, 7, 0], [5, 0])
    assert [dropout_oracle.number(24 + j, 5, 7) for j in range(8)] == [h for w in words for h in (w % 65536, w >> 16)]
    mask, factor = dropout_oracle.keep(4000, 0.25, 1, 2)
    assert factor == 4 / 3 and abs(mask.mean() - 0.75) < 5 * math.sqrt(0.25 * 0.75 / 4000)
    assert not dropout_oracle.keep(64, 1.0, 1, 2)[0].any() and dropout_oracle.keep(64, 0.0, 1, 2)[0].all()
