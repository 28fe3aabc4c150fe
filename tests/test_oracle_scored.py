"""Pins of the scored-routing oracle: the softmax rules of the routing oracle, hand-worked groups, differences."""
import numpy as np
import pytest

import oracle
import oracle.scored as O


def test_plain_softmax_equals_the_routing_oracle():
    rng = np.random.default_rng(0)
    x, w = rng.standard_normal((40, 16)), rng.standard_normal((12, 16))
    for renorm, mode in ((True, 0), (False, 1)):
        r, ref = O.route(x, w, 3, renorm=renorm), oracle.routing.route(x, w, 3, 0, mode)
        np.testing.assert_array_equal(r["idx"], ref["idx"])
        np.testing.assert_allclose(r["gate"], ref["gate"], rtol=1e-12)


def test_a_bias_of_minus_infinity_is_a_hard_mask():
    rng = np.random.default_rng(1)
    x, w = rng.standard_normal((40, 16)), rng.standard_normal((8, 16))
    m = np.array([1, 0, 1, 1, 0, 1, 0, 1], np.uint8)
    r = O.route(x, w, 2, bias=np.where(m, 0.0, -np.inf))
    ref = oracle.routing.route(x, w, 2, 1, 0, mask=m)
    np.testing.assert_array_equal(r["idx"], ref["idx"])
    r = O.route(x, w, 3, bias=np.where(np.arange(8) == 5, 0.0, -np.inf))
    assert (r["idx"] == [5, -1, -1]).all() and (r["gate"] == [1, 0, 0]).all() and r["load"][5] == 40


def test_groups_by_hand():
    z = np.array([[3.0, 0.0, 2.0, 2.0, 2.5, -9.0]])  # groups (3, 0), (2, 2), (2.5, -9)
    w = np.eye(6)
    kw = dict(score="sigmoid", n_group=3, renorm=False)
    assert O.route(z, w, 2, topk_group=1, group_top=1, **kw)["idx"].tolist() == [[0, 1]]
    assert O.route(z, w, 2, topk_group=1, group_top=2, **kw)["idx"].tolist() == [[2, 3]]  # .88 + .88 beats .95 + .5
    assert O.route(z, w, 3, topk_group=2, group_top=1, **kw)["idx"].tolist() == [[0, 4, 1]]
    assert O.route(z, w, 1, topk_group=1, group_top=1, bias=np.array([0, 0, 0, .2, 0, 0]), **kw)["idx"].tolist() == [[3]]


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_gradient_is_the_central_difference(score, renorm):
    rng = np.random.default_rng(2)
    T, d, E, K = 5, 7, 6, 3
    x, w, dg = rng.standard_normal((T, d)), rng.standard_normal((E, d)), rng.standard_normal((T, K))
    idx = O.route(x, w, K, score, renorm=renorm)["idx"]
    idx[1, 2] = -1
    dx, dw = O.gradient(x, w, idx, dg, score, renorm, 1.7)
    f = lambda x, w: (O.gates(x, w, idx, score, renorm, 1.7) * dg).sum()  # noqa: E731
    h = 1e-6
    for a, g in ((x, dx), (w, dw)):
        for i in np.ndindex(a.shape):
            keep = a[i]
            a[i] = keep + h
            up = f(x, w)
            a[i] = keep - h
            down = f(x, w)
            a[i] = keep
            assert abs((up - down) / (2 * h) - g[i]) < 1e-8
