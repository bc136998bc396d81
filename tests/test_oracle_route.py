"""Pins of the routing oracle: rows worked by hand, ties, masks and groups, and
central differences for every gradient."""

import math

import numpy as np
import pytest

import oracle

INF = math.inf


def test_softmax_by_hand():
    row = [math.log(1), math.log(2), math.log(3), math.log(4)]
    ids, gates = oracle.route([row], 2)
    assert ids.tolist() == [[3, 2]]
    assert np.allclose(gates, [[4 / 7, 3 / 7]], rtol=1e-15)
    ids, gates = oracle.route([row], 2, renormalize=False, scale=2.0)
    assert np.allclose(gates, [[0.8, 0.6]], rtol=1e-15)


def test_sigmoid_by_hand():
    # sigmoid(log(p / (1 - p))) = p
    row = [math.log(p / (1 - p)) for p in (0.5, 0.2, 0.75)]
    ids, gates = oracle.route([row], 2, score="sigmoid")
    assert ids.tolist() == [[2, 0]] and np.allclose(gates, [[0.6, 0.4]], rtol=1e-14)
    # the bias moves the choice (0.2 + 0.4 first, 0.75 - 0.3 last) and leaves the scores
    ids, gates = oracle.route([row], 2, score="sigmoid", bias=[0.0, 0.4, -0.3], renormalize=False)
    assert ids.tolist() == [[1, 0]] and np.allclose(gates, [[0.2, 0.5]], rtol=1e-14)


def test_ties_go_to_the_lower_index():
    assert oracle.choose([1.0, 2.0, 2.0, 2.0], 2) == [1, 2]
    assert oracle.choose([0.0] * 4, 3, score="sigmoid", bias=[0.5, 0.5, 0.5, 0.25]) == [0, 1, 2]
    # groups of equal score: the first
    assert oracle.choose([1.0, 0.0, 0.0, 1.0], 1, groups=2, top_groups=1) == [0]


def test_masks():
    assert oracle.choose([-INF, 1.0, -INF], 2) == [1, -1]
    ids, gates = oracle.route([[-INF] * 3], 2, renormalize=False)
    assert ids.tolist() == [[-1, -1]] and gates.tolist() == [[0.0, 0.0]]
    assert oracle.choose([0.0, 5.0, 1.0], 2, bias=[0.0, -INF, 0.0]) == [2, 0]
    assert oracle.choose([0.0, math.nan, 1.0], 2) == [2, 0]


def test_groups_by_hand():
    row = [5.0, 0.0, 3.0, 2.9, 4.0, -9.0]
    # best of a group: 5, 3, 4
    assert oracle.choose(row, 2, groups=3, top_groups=2) == [0, 4]
    assert oracle.choose(row, 2, groups=3, top_groups=1) == [0, 1]
    # the two best scores (sigmoids): 0.9933 + 0.5, 0.9526 + 0.9478, 0.982 + 0.0001
    assert oracle.choose(row, 2, score="sigmoid", groups=3, top_groups=1,
                         group_score="top2") == [2, 3]
    # of a group with one expert left, that one counts alone: 0.99 < 0.952 + 0.948, > 0.5 + 0.4
    row = [5.0, -INF, 3.0, 2.9, 0.0, -0.4]
    assert oracle.choose(row, 1, score="sigmoid", groups=3, top_groups=2,
                         group_score="top2") == [0]


def test_small_scores_are_renormalized():
    _, gates = oracle.route([[-800.0, -800.0 + math.log(3), -900.0]], 2, score="sigmoid")
    assert np.allclose(gates, [[0.75, 0.25]], rtol=1e-12)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [True, False])
@pytest.mark.parametrize("ids", [[[3, 0, 5]], [[2, 2, 4]], [[1, -1, -1]], [[-1, -1, -1]]])
def test_gradient_against_differences(score, renormalize, ids):
    rng = np.random.default_rng(3)
    l = rng.normal(size=(1, 6))
    d = rng.normal(size=(1, 3))

    def loss(x):
        g = oracle.gates_of(x[0], ids[0], score, renormalize, 2.5)
        return sum(a * b for a, b in zip(g, d[0]))

    got = oracle.route_backward(l, ids, d, score, renormalize, 2.5)
    h = 1e-6
    for e in range(6):
        step = np.zeros((1, 6))
        step[0, e] = h
        want = (loss(l + step) - loss(l - step)) / (2 * h)
        assert abs(got[0, e] - want) < 1e-8, (e, got[0, e], want)
