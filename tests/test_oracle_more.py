"""The oracle of routing by scores, dense products and the gradients' norm against differences and cases worked by hand (no GPU)."""
import math

import numpy as np
import pytest

from oracle import map_oracle as mo
from test_oracle_map import _difference


def test_routing_by_hand():
    inf, nan = math.inf, math.nan
    logits = np.array([[0.0, 2.0, 1.0, -1.0], [-inf, 0.0, nan, -inf], [3.0, 3.0, -inf, 3.0], [-inf] * 4])
    experts, weights, offsets, order, slots = mo.route_scored(logits, 2, bias=np.array([2.0, 0.0, 0.0, 0.0]), scale=2.0)
    s = 1.0 / (1.0 + np.exp(-np.array([0.0, 1.0, 2.0, 3.0])))
    assert experts.tolist() == [[0, 1], [1, -1], [0, 1], [-1, -1]]      # the bias lifts expert 0, whose weight stays its score's
    assert np.allclose(weights, [[2 * s[0] / (s[0] + s[2]), 2 * s[2] / (s[0] + s[2])], [2, 0], [1, 1], [0, 0]])
    assert offsets.tolist() == [0, 2, 5, 5, 5] and order.tolist() == [0, 4, 1, 2, 5, -1, -1, -1] and slots.tolist() == [[0, 2], [3, -1], [1, 4], [-1, -1]]
    # two groups of two: by their best the first one, by the sum of two the second
    logits = np.array([[4.0, -4.0, 1.0, 1.0]])
    for best, want in ((1, [0, 1]), (2, [2, 3])):
        assert mo.route_scored(logits, 2, bias=np.zeros(4), groups=2, top_groups=1, group_best=best)[0].tolist() == [want]
    assert mo.route_scored(logits, 2, groups=2, top_groups=1, group_best=2)[0].tolist() == [[2, 3]]


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("normalize", [True, False])
def test_route_gradient_against_differences(score, normalize):
    rng = np.random.default_rng(3)
    logits, c, bias = rng.normal(size=(5, 8)), rng.normal(size=(5, 3)), 0.1 * rng.normal(size=8)
    call = dict(score=score, normalize=normalize, scale=2.5)
    experts, weights, *_ = mo.route_scored(logits, 3, bias=bias, groups=4, top_groups=2, group_best=2, **call)
    got = mo.route_scored_gradient(logits, experts, weights, c, **call)
    want = _difference(lambda l: float((mo.route_scored(l, 3, bias=bias, groups=4, top_groups=2, group_best=2, **call)[1] * c).sum()), logits)
    assert np.abs(got - want).max() < 1e-8


def test_tiny_scores_keep_their_shares():
    weights = mo.route_scored(np.array([[-900.0, -901.0, -5000.0]]), 2)[1]
    assert np.allclose(weights, [[1 / (1 + math.exp(-1)), math.exp(-1) / (1 + math.exp(-1))]])


def test_balance_by_hand():
    assert np.allclose(mo.balance_bias([0.0, 1.0, 2.0], [0, 5, 6, 9], 0.5), [-0.5, 1.5, 2.0])


@pytest.mark.parametrize("name", ["none", "relu", "silu", "gelu"])
def test_dense_gradients_against_differences(name):
    rng = np.random.default_rng(5)
    x, w, b, c = rng.normal(size=(6, 4)), rng.normal(size=(3, 4)), rng.normal(size=3), rng.normal(size=(6, 3))
    r = rng.normal(size=(6, 3))
    _, z, _ = mo.dense(x, w, b, name, r)
    dx, dw, db, _ = mo.dense_gradient(c, x, w, name, z)
    loss = lambda x, w, b, r: float((mo.dense(x, w, b, name, r)[0] * c).sum())   # noqa: E731
    for got, want in ((dx, _difference(lambda v: loss(v, w, b, r), x)), (dw, _difference(lambda v: loss(x, v, b, r), w)), (db, _difference(lambda v: loss(x, w, v, r), b)),
                      (c, _difference(lambda v: loss(x, w, b, v), r))):
        assert np.abs(got - want).max() < 1e-7


def test_norm_by_hand():
    assert mo.gradient_norm([np.array([3.0]), np.array([[4.0, 0.0]])], 2.5, 0.5) == (2.5, 0.5)
    assert mo.gradient_norm([np.array([3.0]), np.array([4.0])], 2.5) == (5.0, 0.5)
