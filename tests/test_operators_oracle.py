"""Hand-worked values of the oracle of the routing and matrix-product operators."""

import numpy as np

from oracle import operators_oracle as P


def test_softmax_routes_and_renormalised_weights():
    ids, w = P.route_experts(np.log(np.array([[1.0, 4.0, 3.0, 2.0]])), 2, renorm=False)
    assert ids.tolist() == [[1, 2]]
    np.testing.assert_allclose(w, [[0.4, 0.3]], rtol=1e-15)
    _, w = P.route_experts(np.log(np.array([[1.0, 4.0, 3.0, 2.0]])), 2, scale=3.5)
    np.testing.assert_allclose(w, [[2.0, 1.5]], rtol=1e-15)


def test_bias_steers_the_selection_not_the_weight():
    l = np.array([[0.0, 0.0, -np.log(3.0)]])                       # sigmoid: 1/2, 1/2, 1/4
    ids, w = P.route_experts(l, 1, score="sigmoid", renorm=False)
    assert ids.tolist() == [[0]]                                   # a tie goes to the smaller id
    ids, w = P.route_experts(l, 2, score="sigmoid", select_bias=[0.0, 0.1, 1.0], renorm=False)
    assert ids.tolist() == [[2, 1]]
    np.testing.assert_allclose(w, [[0.25, 0.5]], rtol=1e-15)


def test_groups_by_largest_and_by_two_largest():
    p = np.array([[0.9, 0.1, 0.6, 0.6, 0.9, 0.1]])
    l = np.log(p / (1 - p))
    best, _ = P.route_experts(l, 1, score="sigmoid", groups=3, keep_groups=1)
    assert best.tolist() == [[0]]
    two, _ = P.route_experts(l, 1, score="sigmoid", groups=3, keep_groups=1, group_top2=True)
    assert two.tolist() == [[2]]                                   # 1.2 against 1.0 and 1.0
    two, _ = P.route_experts(l, 2, score="sigmoid", groups=3, keep_groups=2, group_top2=True)
    assert two.tolist() == [[0, 2]]                                # the equal groups 0 and 2: the smaller stays


def test_masked_rows():
    l = np.full((2, 4), -np.inf)
    l[1, 3] = -5.0
    ids, w = P.route_experts(l, 2)
    assert ids.tolist() == [[0, 1], [3, 0]]
    np.testing.assert_array_equal(w, [[0, 0], [1, 0]])
    l[1, 3] = -np.finfo(np.float32).max                             # the type's lowest value is no mask
    ids, w = P.route_experts(l, 2)
    assert ids.tolist()[1] == [3, 0] and w[1].tolist() == [1, 0]
    ids, w = P.route_experts(l, 2, groups=2, keep_groups=1)
    assert ids.tolist() == [[0, 1], [3, 2]]


def test_activations():
    z = np.array([-2.0, 0.0, 1.0])
    np.testing.assert_allclose(P.activate("silu", z), [-2 / (1 + np.e ** 2), 0, 1 / (1 + np.e ** -1)], rtol=1e-14)
    np.testing.assert_allclose(P.activate("gelu", z), [-2 * 0.022750131948179195, 0, 0.8413447460685429], rtol=1e-14)
    np.testing.assert_allclose(P.activate("gelu_tanh", z), [-0.04540230591222, 0, 0.84119199060827], rtol=1e-12)
    y, _, _ = P.linear([[1.0, 2.0]], [[1.0, 1.0], [2.0, 0.0]], bias=[0.5, -1.0], act="relu", gated=True, residual=[[10.0]])
    assert y.tolist() == [[13.5]]
