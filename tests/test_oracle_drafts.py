"""Pins of the drafted-token oracle against cases worked by hand."""
import math

import numpy as np
import pytest

from oracle import attention as oa
from oracle import drafts as od


def test_ancestors():
    parents = [-1, 0, 0, 1, 9, -5]
    assert [od.ancestors(parents, i) for i in range(6)] == [[0], [1, 0], [2, 0], [3, 1, 0], [4], [5]]


def test_softmax_and_temperature():
    p = od.softmax([0.0, math.log(3.0), -np.inf], 1.0)
    assert np.allclose(p, [0.25, 0.75, 0.0], atol=1e-15)
    assert np.allclose(od.softmax([0.0, math.log(3.0)], 0.5), [0.1, 0.9], atol=1e-15)
    assert od.softmax([1.0, 2.0, 2.0], 0.0).tolist() == [0.0, 1.0, 0.0]
    assert od.softmax([-np.inf] * 3, 1.0) is None
    assert od.softmax([0.0, -693.0, -694.0], 1.0).tolist()[2] == 0.0 < od.softmax([0.0, -693.0, -694.0], 1.0)[1]


@pytest.mark.parametrize("u,token", [(0.0, 1), (0.2, 1), (0.3, 3), (0.99, 3), (1.0, 3), (7.0, 3), (-1.0, 1), (math.nan, 3)])
def test_draw(u, token):
    assert od.draw(np.array([0.0, 1.0, 0.0, 3.0, 0.0]), u)[0] == token


def test_draw_near_a_border():
    assert od.draw(np.array([1.0, 1.0, 2.0]), 0.25)[0] == 1
    assert od.draw(np.array([1.0, 1.0, 2.0]), 0.25)[1] == 0.0
    assert abs(od.draw(np.array([1.0, 1.0, 2.0]), 0.3)[1] - 0.05) < 1e-7


def test_a_chain_by_hand():
    rows = np.log(np.array([[0.5, 0.3, 0.2], [0.1, 0.6, 0.3]]))
    draft = np.log(np.array([[0.2, 0.7, 0.1], [1.0, 1.0, 1.0]]))
    # p(1) / q(1) = 3/7
    tokens, logp, _ = od.verify_draft(rows, [0, 1], draft, 1.0, [0.42, 0.0], 0.5)
    assert tokens == [1, 1] and np.allclose(logp, np.log([0.3, 0.6]))
    # it falls: max(p - q, 0) = (0.3, 0, 0.1)
    assert od.verify_draft(rows, [0, 1], draft, 1.0, [0.43, 0.0], 0.74)[0] == [0]
    assert od.verify_draft(rows, [0, 1], draft, 1.0, [0.43, 0.0], 0.76)[0] == [2]
    # a drafter without probabilities: u < p(1) = 0.3; then p without it: 5/7, 2/7
    assert od.verify_draft(rows, [0, 1], None, 1.0, [0.29, 0.0], 0.5)[0] == [1, 1]
    assert od.verify_draft(rows, [0, 1], None, 1.0, [0.31, 0.0], 0.71)[0] == [0]
    assert od.verify_draft(rows, [0, 1], None, 1.0, [0.31, 0.0], 0.72)[0] == [2]
    # greedy
    assert od.verify_draft(rows, [0, 0], None, 0.0, [0.9, 0.9], 0.9)[0] == [0, 1]
    assert od.verify_draft(rows, [0, 1], draft, 0.0, [0.0, 0.0], 0.0)[0] == [0]


def test_what_verification_returns_is_distributed_as_the_target():
    # over a grid of numbers the first token follows p, whatever the drafter
    p, q = np.array([0.5, 0.2, 0.3]), np.array([0.1, 0.6, 0.3])
    share = np.zeros(3)
    for x in range(3):
        for u in (np.arange(40) + 0.5) / 40:
            for w in (np.arange(40) + 0.5) / 40:
                share[od.verify_draft(np.log([p, p]), [0, x], np.log([q, q]), 1.0, [u, 0], w)[0][0]] += q[x] / 1600
    assert np.abs(share - p).max() < 0.02


def test_a_tree_by_hand():
    rows = np.log(np.array([[0.5, 0.5], [0.9, 0.1], [0.2, 0.8], [0.5, 0.5]]))
    parents, ids = [-1, 0, 0, 2], [0, 0, 1, 1]
    assert od.verify_tree(rows, ids, parents, 1.0, [0.7, 0.0, 0.3, 0.1])[:2] == ([0, 2, 3], [1, 1, 0])
    assert od.verify_tree(rows, ids, parents, 1.0, [0.7, 0.0, 0.1, 0.1])[:2] == ([0, 2], [1, 0])
    assert od.verify_tree(rows, ids, parents, 1.0, [0.4, 0.95, 0.1, 0.1])[:2] == ([0, 1], [0, 1])


def test_entries_move_whole():
    D = 96
    x = np.random.default_rng(0).normal(size=(64, D))
    cache = np.zeros((1, 2, 1, oa.tile_bytes(D)), dtype=np.uint8)
    for t in range(64):
        for value in (False, True):
            oa.put(cache[0, 0, 0], D, value, t, x[t])
            oa.put(cache[0, 1, 0], D, value, t, -x[t])
    before = cache.copy()
    # tokens 62 .. 66 are nodes 0 .. 4; 0, 2, 4 are kept
    assert od.keep(cache, D, [0, 1], 67, 5, [0, 2, 4], 3) == 65
    for place, source in (((0, 63), (1, 0)), ((1, 0), (1, 2))):
        for value in (False, True):
            assert np.array_equal(oa.get(cache[0, place[0], 0], D, value, place[1]),
                                  oa.get(before[0, source[0], 0], D, value, source[1]))
    assert (cache != before).sum() <= 2 * 2 * (D // 2 + oa.scale_stride(D))
