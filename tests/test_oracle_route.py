"""Pins of the router's oracle: hand cases, and its gradient against differences of its own forward pass."""
import math

import numpy as np
import pytest

from oracle import route


def test_by_hand():
    z = np.log(np.array([[1.0, 3.0], [3.0, 1.0], [1.0, 1.0]]))
    ids, gates, counts, loss = route.forward(z, 1)
    assert ids.tolist() == [[1], [0], [0]] and counts.tolist() == [2, 1]
    assert np.allclose(gates[:, 0], [0.75, 0.75, 0.5])
    assert math.isclose(loss, 2 * (2 / 3 * 0.5 + 1 / 3 * 0.5))        # mean p is one half for both


def test_balanced_loss_is_one():
    """Uniform probabilities and uniform counts: the loss's minimum, 1."""
    E = 8
    z = np.zeros((E, E))
    z[np.arange(E), np.arange(E)] = 1e-9                              # each token another expert
    assert math.isclose(route.forward(z, 1)[3], 1.0, rel_tol=1e-6)


@pytest.mark.parametrize("z,k,ids", [([1.0, 1.0, 1.0], 2, [0, 1]), ([-math.inf, 0.0, -math.inf], 3, [1, 0, 2]), ([math.nan, -math.inf, 5.0], 3, [2, 1, 0]),
                                     ([math.nan, math.nan], 1, [0]), ([0.0, math.inf], 1, [1]), ([-0.0, 0.0], 1, [0])])
def test_choice(z, k, ids):
    assert route.choose(z, k) == ids


def test_who_takes_part():
    z = np.array([[0.0, 1.0], [-math.inf, -math.inf], [math.nan, math.nan]])
    ids, gates, counts, loss = route.forward(z, 1, mask=[1, 1, 0])
    assert counts.tolist() == [0, 1] and gates[1, 0] == 0 and gates[2, 0] == 0
    assert route.forward(z, 1, mask=[0, 1, 0])[3] == 0.0


@pytest.mark.parametrize("k,normalize", [(1, False), (2, False), (2, True), (3, True)])
def test_gradient_against_differences(k, normalize):
    """Central differences of sum(gates * d_gates) + d_loss * loss, with counts as they are (no logit is near a tie)."""
    rng = np.random.default_rng(k * 2 + normalize)
    z = rng.standard_normal((5, 6)) * 2
    mask = [1, 1, 0, 1, 1]
    dg, dl = rng.standard_normal((5, k)), 0.7
    ids, _, counts, _ = route.forward(z, k, mask, normalize)
    got = route.backward(z, ids, counts, dg, dl, mask, normalize)

    def value(z):
        i, g, c, loss = route.forward(z, k, mask, normalize)
        assert np.array_equal(i, ids)
        return (g * dg).sum() + dl * loss

    h = 1e-5
    for t in range(5):
        for e in range(6):
            d = np.zeros_like(z)
            d[t, e] = h
            assert abs((value(z + d) - value(z - d)) / (2 * h) - got[t, e]) < 1e-8
