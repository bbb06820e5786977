"""Pins of the log probabilities' oracle: worked by hand, and against the formula evaluated another way."""
import math

import numpy as np

from oracle import logprobs as L


def test_by_hand():
    r = L.row([math.log(1), math.log(2), math.log(5), -math.inf])
    assert np.allclose(np.exp(r["logp"]), [1 / 8, 2 / 8, 5 / 8, 0])
    assert np.isclose(r["entropy"], math.log(8) / 8 + math.log(4) / 4 + 5 / 8 * math.log(8 / 5))
    assert list(r["order"]) == [2, 1, 0, 3]
    assert list(L.ranks(r, [2, 0, 3, -1, 4])) == [0, 2, 3, -1, -1]


def test_temperature_and_ties():
    r = L.row([0.0, 2.0, 2.0, -0.0], inverse=0.5)
    e = math.e
    assert np.allclose(np.exp(r["logp"]), np.array([1, e, e, 1]) / (2 + 2 * e))
    assert list(r["order"]) == [1, 2, 0, 3]


def test_uniform_and_certain():
    assert np.isclose(L.row(np.full(1000, -3e38))["entropy"], math.log(1000))
    r = L.row([-math.inf, 7.0, -math.inf])
    assert r["entropy"] == 0 and list(r["logp"]) == [-math.inf, 0, -math.inf]


def test_not_a_number():
    for x in ([1.0, math.nan], [1.0, math.inf], [-math.inf, -math.inf]):
        r = L.row(x)
        assert np.isnan(r["entropy"]) and np.isnan(r["logp"]).all()
    assert list(L.row([math.nan, -1.0, -math.inf, math.inf])["order"]) == [3, 1, 0, 2]
    for bad in (0.0, -1.0, math.nan, math.inf):
        assert np.isnan(L.row([1.0, 2.0], bad)["logp"]).all()
