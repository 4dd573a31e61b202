"""Pins of the oracle of dropout, log probabilities and cross entropy (CPU only)."""
import math

import numpy as np
import pytest

from oracle import fxp_oracle as orc
from oracle import head_oracle as head

ALL_DRAWS = np.arange(65536, dtype=np.int64)


@pytest.mark.parametrize("p", [0.0, 1 / 65536, 0.1, 0.5, 0.9, 65535 / 65536])
@pytest.mark.parametrize("x", [-128, -77, -1, 0, 1, 3, 100, 127])
@pytest.mark.parametrize("step", [0, -1, 3])
def test_dropout_has_exactly_the_expectation_of_its_input(x, p, step):
    """Over all 65536 draws the outputs sum to x 2^step 65536 (a wide output, so nothing saturates): the decision and the
    rounding share one draw without any bias.  x 2^step 65536 is a whole number for the steps taken here."""
    y = head.dropout_with_bits(np.full(65536, x), 4, p, 32, 4 + step, ALL_DRAWS)
    assert int(y.sum()) * 2 ** 3 == x * 2 ** (step + 3) * 65536
    drop = head.drop_threshold(p)
    assert np.all(y[:drop] == 0) and len(np.unique(y[drop:])) <= 2


def test_dropout_of_nothing_is_a_change_of_format():
    x = np.arange(-128, 128)
    assert np.array_equal(head.dropout(x, 5, 0.0, 8, 5), x)
    # coarser: the requantizing rule's probabilities, floor((x 2^16 / 4 + R) / 2^16)
    bits = orc.rounding_bits(256, orc.SR, 3, 9)
    assert np.array_equal(head.dropout(x, 5, 0.0, 8, 3, seed=3, stream=9), ((x << 14) + bits) >> 16)


def test_half_dropped_doubles_the_rest():
    x = np.arange(-60, 60)
    bits = orc.rounding_bits(120, orc.SR, 1, 2)
    assert np.array_equal(head.dropout(x, 4, 0.5, 8, 4, seed=1, stream=2), np.where(bits >= 32768, 2 * x, 0))


def test_nearest_rounding_of_the_kept():
    # x / 0.9 in units of 2^-4: K = 58982, 7 65536 / 58982 = 7.778 -> 8, -7 -> -8
    y = head.dropout_with_bits(np.array([7, -7, 7]), 4, 0.1, 8, 4, np.array([65535, 6554, 6553]), mode=head.RN_HALF_UP)
    assert y.tolist() == [8, -8, 0]


def test_uniform_rows():
    for classes in (1, 2, 10, 1000):
        r = head.log_probs(np.full((1, classes), 3), 2, [classes - 1], min(classes, 3))
        assert float(r["logp"][0]) == pytest.approx(-math.log(classes), abs=1e-15)
        assert float(r["entropy"][0]) == pytest.approx(math.log(classes), abs=1e-13)
        assert r["top_idx"][0].tolist() == list(range(min(classes, 3)))


def test_two_classes_by_hand():
    # codes 8 and 4 of <8,2>: values 2 and 1, p = 1 / (1 + e^-1)
    p = 1 / (1 + math.exp(-1.0))
    g = head.gradient(np.array([[8, 4]]), 2, [0])
    assert float(g[0, 0]) == pytest.approx(p - 1, abs=1e-16) and float(g[0, 1]) == pytest.approx(1 - p, abs=1e-16)
    assert head.quantize_real(g, 8, 7, mode=orc.RN_HALF_UP).tolist() == [[round((p - 1) * 128), round((1 - p) * 128)]]


def test_gradient_against_differences():
    rng = np.random.default_rng(4)
    x, labels, w = rng.normal(size=(3, 17)), np.array([4, -1, 16]), np.array([1.0, 2.0, 0.5])
    g = head.gradient(x, None, labels, w)
    h = np.longdouble(1e-6)
    for i, j in ((0, 4), (0, 5), (1, 3), (2, 16), (2, 0)):
        up, down = x.astype(np.longdouble), x.astype(np.longdouble)
        up[i, j] += h
        down[i, j] -= h
        d = (head.loss(up, None, labels, w) - head.loss(down, None, labels, w)) / (2 * h)
        assert abs(d - g[i, j]) < 1e-11              # the third derivative is below 1: h^2 / 6 = 2e-13, and rounding


def test_rows_without_a_distribution():
    inf = np.inf
    x = np.array([[0.0, np.nan, 1.0], [0.0, inf, 1.0], [-inf, -inf, -inf], [-inf, 2.0, -inf]])
    r = head.log_probs(x, None, np.array([0, 0, 1, 0]), 2)
    assert np.isnan(r["logp"][:2].astype(float)).all() and r["lse"][2] == -inf and r["logp"][2] == -inf and r["entropy"][2] == 0
    assert r["logp"][3] == -inf and r["lse"][3] == 2.0 and r["entropy"][3] == 0
    assert r["top_idx"].tolist() == [[2, 0], [1, 2], [0, 1], [1, 0]]
    assert not head.gradient(x, None, np.array([0, 0, 1, 3])).any()
