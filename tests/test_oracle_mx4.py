"""Pins of the mx4 oracle: the grid's rounding against brute force, scales from their definition, invariances."""
import numpy as np

import oracle.mx4 as O


def test_rounding_is_the_nearest_grid_value_with_even_ties():
    a = np.linspace(0, 6, 4801)
    q = O.round_to_grid(a)
    best = np.abs(a[:, None] - O.GRID).min(1)
    np.testing.assert_array_equal(np.abs(a - q), best)
    ties = {0.25: 0.0, 0.75: 1.0, 1.25: 1.0, 1.75: 2.0, 2.5: 2.0, 3.5: 4.0, 5.0: 4.0}
    for t, v in ties.items():
        assert O.round_to_grid(t) == v
    assert (O.round_to_grid([6.5, 7.999, 1e9]) == 6).all()


def test_block_scale():
    x = np.zeros((3, 64))
    x[0, 3], x[0, 4] = 7.9, 0.26  # floor(log2) = 2: unit 1
    x[1, 0], x[1, 32] = 8.0, 1.0  # unit 2; a block of its own
    x[1, 1], x[1, 33] = 1.1, 0.3
    q = O.quantize(x)
    assert q[0, 3] == 6 and q[0, 4] == 0.5
    assert q[1, 0] == 8 and q[1, 1] == 1 and q[1, 32] == 1 and q[1, 33] == 0.25
    assert (q[2] == 0).all()


def test_power_of_two_scaling_and_sign_commute_with_rounding():
    x = np.random.default_rng(0).standard_normal((20, 100))
    np.testing.assert_array_equal(O.quantize(x * 2.0 ** 30), O.quantize(x) * 2.0 ** 30)
    np.testing.assert_array_equal(O.quantize(-x), -O.quantize(x))
    np.testing.assert_array_equal(O.quantize(O.quantize(x)), O.quantize(x))
    assert np.abs(O.quantize(x) - x).max() <= np.abs(x).max() / 4  # 8 -> 6 at worst


def test_a_non_finite_value_spoils_its_block_only():
    x = np.ones((2, 64))
    x[0, 40], x[1, 1] = np.inf, np.nan
    assert np.isnan(O.quantize(x)).tolist() == [[False] * 32 + [True] * 32, [True] * 32 + [False] * 32]


def test_slack_covers_moved_inputs():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 64))
    d = 1e-2 * np.abs(x) + 1e-3
    room = O.slack(x, d)
    for _ in range(50):
        y = x + rng.uniform(-1, 1, x.shape) * d
        assert (np.abs(O.quantize(y) - O.quantize(x)) <= room + 1e-12).all()
    assert (O.slack(x, np.zeros_like(x)) == 0).all()


def test_layer_with_exactly_representable_parts():
    rng = np.random.default_rng(2)
    w1, w3 = (rng.choice(O.GRID, (32, 32)) for _ in range(2))
    w2 = rng.choice(O.GRID, (32, 32))
    w1[:, 0] = w3[:, 0] = w2[:, 0] = 4  # unit 1 in every row
    x = np.zeros((2, 32))
    x[0, 0] = 4.0
    y, room = O.moe_layer(x, [[0, -1], [-1, -1]], [[0.5, 9.0], [1.0, 1.0]], [(w1, w3, w2)])
    h = 16 / (1 + np.exp(-16.0)) * 16  # every hidden value alike: the top of the grid is 1.5 * 128 .. 256
    np.testing.assert_allclose(y[0], 0.5 * O.round_to_grid(h / 32) * 32 * w2.sum(1))
    assert (y[1] == 0).all() and (room[1] == 0).all()
