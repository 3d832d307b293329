"""Pins of the norm + rotary oracle: closed forms and the defining property of the rotation."""
import numpy as np

from oracle import rope


def test_position_zero_changes_nothing_and_a_quarter_turn_swaps():
    x = np.arange(1.0, 9.0).reshape(1, 1, 8)
    f = np.array([1.0, 0.5])
    np.testing.assert_array_equal(rope.rotate(x, [0], f), x)
    y = rope.rotate(np.ones((1, 1, 2)) * [[3.0, 4.0]], [1], np.array([np.pi / 2]))
    np.testing.assert_allclose(y[0, 0], [-4.0, 3.0], atol=1e-12)


def test_products_depend_on_the_distance_alone():
    rng = np.random.default_rng(1)
    f = 10000.0 ** (-np.arange(0, 32, 2) / 32)
    q, k = rng.normal(size=(1, 1, 64)), rng.normal(size=(1, 1, 64))
    for il in (False, True):
        d = [float((rope.rotate(q, [p + 7], f, il) * rope.rotate(k, [p], f, il)).sum()) for p in (0, 13, 100000)]
        np.testing.assert_allclose(d, d[0], atol=1e-9)


def test_both_pairings_are_one_permutation_of_each_other():
    rng = np.random.default_rng(2)
    f = 10000.0 ** (-np.arange(0, 16, 2) / 16)
    x = rng.normal(size=(2, 3, 16))
    perm = np.concatenate([np.arange(0, 16, 2), np.arange(1, 16, 2)])
    np.testing.assert_allclose(rope.rotate(x[..., perm], [1, 5, 9], f), rope.rotate(x, [1, 5, 9], f, True)[..., perm])


def test_norm_has_unit_mean_square_and_the_weight_scales_it():
    x = np.random.default_rng(3).normal(size=(4, 64)) * 7
    y = rope.norm_heads(x, np.ones(64), 0.0)
    np.testing.assert_allclose((y * y).mean(-1), 1.0)
    np.testing.assert_allclose(rope.norm_heads(x, np.full(64, 2.0), 0.0), 2 * y)
    np.testing.assert_array_equal(rope.norm_heads(np.zeros((1, 64)), np.ones(64), 1e-6), 0.0)
