"""The oracle of the norm, of the position rotation and of 4-bit weights, pinned by facts that do not come from it."""

import numpy as np
import pytest

import workloads as wl
from oracle import e4m3, fp4, norm, rope


def bits(x):
    return wl.bf16_bits_from_f32(np.asarray(x, np.float32))


def test_norm_of_a_constant_row_is_its_weight():
    w = np.array([0.5, 1.0, -2.0, 3.0], np.float32)
    y = norm.rms_norm(norm.residual_sum(bits([[7.0] * 4])), bits(w), 1e-30)
    np.testing.assert_allclose(y[0], w, rtol=1e-12)


def test_norm_by_hand():
    # mean square 12.5, eps 3.5: divided by 4
    y = norm.rms_norm(norm.residual_sum(bits([[1.0, 4.0]]), bits([[2.0, 0.0]])), bits([2.0, 1.0]), 3.5)
    np.testing.assert_array_equal(y, [[1.5, 1.0]])
    assert norm.row_scale(y)[0] == 1.5 / 448
    assert norm.row_scale(np.zeros((1, 2)))[0] == 2.0 ** -100


def test_norm_does_not_see_the_scale_of_a_row():
    x = np.random.default_rng(0).standard_normal((3, 64)).astype(np.float32)
    h = norm.residual_sum(bits(x))
    a, b = norm.rms_norm(h, bits(np.ones(64)), 1e-12), norm.rms_norm(h * 2.0 ** 20, bits(np.ones(64)), 1e-12)
    np.testing.assert_allclose(a, b, rtol=1e-10)


def test_norm_rows_that_are_not_finite():
    x = np.ones((3, 8), np.float32)
    x[1, 3], x[2, 0] = np.inf, np.nan
    y = norm.rms_norm(norm.residual_sum(bits(x)), bits(np.ones(8)), 1e-5)
    assert np.isfinite(y[0]).all() and np.isnan(y[1:]).all()
    assert norm.row_scale(y)[1] == 2.0 ** -100


@pytest.mark.parametrize("neighbours", [False, True])
def test_rotation_is_one_and_adds_up(neighbours):
    rng = np.random.default_rng(1)
    x = rng.standard_normal((4, 2, 24))
    f = 10000.0 ** (-np.arange(8) / 8)
    at = np.array([0, 1, 77, 131071])
    y = rope.rotate(x, at, f, neighbours)
    np.testing.assert_array_equal(y[0], x[0])                                   # position 0
    np.testing.assert_array_equal(y[..., 16:], x[..., 16:])                     # channels behind R
    np.testing.assert_allclose(np.linalg.norm(y, axis=-1), np.linalg.norm(x, axis=-1), rtol=1e-12)
    np.testing.assert_allclose(rope.rotate(y, 5 - at, f, neighbours), rope.rotate(x, np.full(4, 5), f, neighbours), atol=1e-10)
    # q . k depends on the distance of their positions alone
    q, k = rng.standard_normal((1, 1, 16)), rng.standard_normal((1, 1, 16))
    dot = lambda i, j: (rope.rotate(q, [i], f, neighbours) * rope.rotate(k, [j], f, neighbours)).sum()
    np.testing.assert_allclose(dot(1000, 990), dot(10, 0), atol=1e-10)


def test_rotation_pairs():
    x = np.arange(1.0, 5.0).reshape(1, 1, 4)
    quarter = np.array([np.pi / 2, 0.0])
    np.testing.assert_allclose(rope.rotate(x, [1], quarter, False)[0, 0], [-3, 2, 1, 4], atol=1e-12)
    np.testing.assert_allclose(rope.rotate(x, [1], quarter, True)[0, 0], [-2, 1, 3, 4], atol=1e-12)
    np.testing.assert_array_equal(rope.pair_sums(x, 4, False)[0, 0], [4, 6, 4, 6])
    np.testing.assert_array_equal(rope.pair_sums(x, 2, True)[0, 0], [3, 3, 0, 0])


def test_fp4_grid_and_ties():
    assert list(fp4.decode_table()[:8]) == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    assert list(fp4.encode(ties)) == [0, 2, 2, 4, 4, 6, 6]
    assert list(fp4.encode(np.array([0.26, 0.74, 5.01, 7.0, 1e9, -0.0, -6.0]))) == [1, 1, 7, 7, 7, 8, 15]


def test_fp4_exponents():
    """The largest magnitude of a group lands on 4 or 6: below 7/4 of its power of two on that power's scale, from there on
    the next one's."""
    x = np.zeros((1, 32 * 6), np.float32)
    x[0, 5], x[0, 40], x[0, 70], x[0, 100], x[0, 130] = 4.0, 6.96875, 7.0, 1.0, -3.0 * 2.0 ** -60
    assert list(fp4.group_exponents(bits(x))[0]) == [0, 0, 1, -2, -61, -100]
    codes, scales = fp4.quantize(bits(x))
    back = fp4.decode(codes, scales)
    assert back[0, 5] == 4 and back[0, 40] == 6 and back[0, 70] == 8 and back[0, 100] == 1
    assert back[0, 130] == -3.0 * 2.0 ** -60
    assert codes[0, 2] == (6 << 4) and codes[0, 20] == 7       # odd columns in the high half, even ones in the low


def test_fp4_values_are_within_half_a_step():
    x = wl.linear_weights(16, 256, 3)
    v = wl.f32_from_bf16_bits(x).astype(np.float64)
    codes, scales = fp4.quantize(x)
    s = np.repeat(2.0 ** (scales.astype(np.float64) - 127), 32, 1)
    step = np.where(np.abs(v) < 2 * s, 0.5, np.where(np.abs(v) < 4 * s, 1.0, 2.0)) * s
    assert (np.abs(fp4.decode(codes, scales) - v) <= step / 2).all()


def test_fp4_linear_by_hand():
    a = np.zeros((2, 64), np.uint8)
    a[0, 1], a[0, 33], a[1, 0] = e4m3.encode(np.float32([2.0, -1.5, 0.0]))[[0, 1, 2]]
    w = np.zeros((1, 32), np.uint8)
    w[0, 0], w[0, 16] = 0x70, 0x30                                              # columns 1 and 33: 6 and 1.5
    y = fp4.gemm(a, np.float32([0.5, 1.0]), fp4.decode(w, np.uint8([[127, 129]])))
    np.testing.assert_array_equal(y, [[0.5 * (2 * 6 - 1.5 * 1.5 * 4)], [0.0]])
