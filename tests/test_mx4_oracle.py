"""The oracle of the microscaled 4-bit operators and of the router's gradient against closed forms and differences.  No GPU needed."""
import itertools
import math

import numpy as np
import pytest

from oracle import mx4_oracle as Q


def test_codes_of_every_tie_and_end():
    m = np.array([0, 0.2, 0.25, 0.26, 0.5, 0.75, 0.76, 1.25, 1.26, 1.75, 1.76, 2.5, 2.51, 3.5, 3.6, 5, 5.01, 6, 7.99])
    assert Q.to_code(m).tolist() == [0, 0, 0, 1, 1, 2, 2, 2, 3, 4, 4, 4, 5, 6, 6, 6, 7, 7, 7]


def test_exponents():
    peak = np.array([0.0, 1.0, 1.999, 4.0, 7.9, 8.0, 2.0 ** -149, 2.0 ** -126, 2.0 ** -124, 3e38, math.inf, math.nan])
    assert Q.exponent(peak).tolist() == [0, 125, 125, 127, 127, 128, 0, 0, 1, 252, 255, 255]


def test_values_of_numbers_of_the_format_are_the_numbers():
    rng = np.random.default_rng(0)
    x = Q.NUMBERS[rng.integers(0, 8, (5, 300))] * rng.choice([-1, 1], (5, 300))
    x[:, ::32] = 6.0                                                 # every block's unit is then 1
    codes, byte = Q.quantize(x)
    assert np.array_equal(Q.values(codes, byte)[:, :300], x)
    assert codes.shape == (5, 512) and (codes[:, 300:] == 0).all() and (byte[:, 10:] == 0).all()


def test_a_value_is_off_by_a_quarter_of_a_binade_at_most():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((40, 256)) * np.exp(rng.standard_normal((40, 1)) * 10)
    v = Q.values(*Q.quantize(x))
    peak = np.abs(x).reshape(40, 8, 32).max(2).repeat(32, 1)
    unit = 2.0 ** (np.floor(np.log2(peak)) - 2)
    assert (np.abs(v - x) <= np.where(np.abs(x) > 6 * unit, 2 * unit, np.where(np.abs(x) >= 4 * unit, unit, np.where(np.abs(x) >= 2 * unit, unit / 2, unit / 4)))).all()


def test_a_block_that_is_no_number_stays_alone():
    x = np.ones((2, 100))
    x[0, 40], x[1, 5] = math.inf, math.nan
    v = Q.values(*Q.quantize(x))[:, :100]
    assert np.isnan(v[0, 32:64]).all() and (v[0, :32] == 1).all() and (v[0, 64:] == 1).all() and np.isnan(v[1, :32]).all() and (v[1, 32:] == 1).all()


def test_tiles_hold_what_the_layout_says():
    rng = np.random.default_rng(2)
    codes, byte = rng.integers(0, 16, (40, 512)).astype(np.uint8), rng.integers(0, 256, (40, 16)).astype(np.uint8)
    q, s = (a.reshape(-1) for a in Q.tiles(codes, byte))
    for r, c in itertools.product((0, 31, 32, 39), (0, 1, 31, 33, 127, 128, 255, 256, 511)):
        tile, lane, j = r // 32 * 2 + c // 256, 32 * (c % 256 // 128) + r % 32, c % 128
        at = tile * 4096 + j // 32 * 1024 + lane * 16 + j % 32 // 2
        assert (q[at] >> (4 * (c & 1))) & 15 == codes[r, c]
        assert s[tile * 256 + lane * 4 + j // 32] == byte[r, c // 32]


@pytest.mark.parametrize("sigmoid", [True, False])
def test_balance_of_an_even_router_is_its_coefficient(sigmoid):
    T, E, k = 12, 6, 2
    idx = np.array([[(2 * t) % E, (2 * t + 1) % E] for t in range(T)])
    counts, mean, loss = Q.balance(np.full((T, E), -3.0), idx, 0.25, sigmoid)
    assert (counts[:E] == T * k // E).all() and counts[E] == T and np.allclose(mean, 1 / E) and abs(loss - 0.25) < 1e-15
    keep = np.arange(T) % 2
    assert Q.balance(np.zeros((T, E)), idx, 1.0, sigmoid, keep=keep)[0][E] == T // 2
    assert Q.balance(np.zeros((T, E)), idx, 1.0, sigmoid, keep=0 * keep)[2] == 0.0


def total(l, idx, dw, sigmoid, renorm, factor, counts, coef, dloss, keep):
    T, E = l.shape
    k = idx.shape[1]
    s = 1 / (1 + np.exp(-l)) if sigmoid else np.exp(l) / np.exp(l).sum(1, keepdims=True)
    w = np.take_along_axis(s, idx, 1)
    w = factor * (w / w.sum(1, keepdims=True) if renorm else w)
    M = counts[E]
    mean = (s / s.sum(1, keepdims=True) * keep[:, None]).sum(0) / M
    return (w * dw).sum() + dloss * coef * E * (counts[:E] / (M * k) * mean).sum()


@pytest.mark.parametrize("sigmoid,renorm", itertools.product([True, False], [True, False]))
def test_gradient_against_differences(sigmoid, renorm):
    rng = np.random.default_rng(3)
    T, E, k = 4, 7, 3
    l, dw, keep = rng.standard_normal((T, E)), rng.standard_normal((T, k)), np.array([1, 0, 1, 1])
    idx = np.stack([rng.permutation(E)[:k] for _ in range(T)])
    idx[2, 1] = idx[2, 0]                                             # an expert in two slots
    counts = np.append(rng.integers(0, 5, E), 3)
    args = (idx, dw, sigmoid, renorm, 1.7, counts, 0.3, 0.9, keep)
    grad, size = Q.backward(l, idx, dw, sigmoid, renorm, 1.7, counts, 0.3, 0.9, keep)
    for t, e in itertools.product(range(T), range(E)):
        d = 1e-5
        hi, lo = l.copy(), l.copy()
        hi[t, e] += d
        lo[t, e] -= d
        # central differences: d^2 / 6 of a third derivative of a few, and rounding of 1e-16 / d
        assert abs((total(hi, *args) - total(lo, *args)) / (2 * d) - grad[t, e]) < 1e-8
    assert (np.abs(grad) <= size * (1 + 1e-12)).all()
