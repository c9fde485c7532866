"""The fp64 oracle of norm and rotation: complex arithmetic, products that depend on the distance alone, norms, far positions."""
import cmath

import numpy as np
import pytest

from oracle import rope


@pytest.mark.parametrize("pairing", ["halves", "neighbours"])
def test_pairs_turn_as_complex_numbers(pairing):
    rng = np.random.default_rng(0)
    x, rad = rng.standard_normal((3, 2, 12)), np.array([0.9, 0.05, 2.5])
    got = rope.norm_rotate(x, [0, 7, 1001], rad, pairing)
    for t, p in enumerate([0, 7, 1001]):
        for h in range(2):
            for i in range(3):
                a, b = (i, i + 3) if pairing == "halves" else (2 * i, 2 * i + 1)
                z = complex(x[t, h, a], x[t, h, b]) * cmath.exp(1j * p * rad[i])
                assert abs(got[t, h, a] - z.real) < 1e-12 and abs(got[t, h, b] - z.imag) < 1e-12
    assert np.array_equal(got[:, :, 6:], x[:, :, 6:]) and np.array_equal(got[0], x[0])


def test_products_depend_on_the_distance():
    rng = np.random.default_rng(1)
    rad = 10000.0 ** (-np.arange(0, 16, 2) / 16)
    q, k = rng.standard_normal((1, 1, 16)), rng.standard_normal((1, 1, 16))

    def product(i, j):
        return float((rope.norm_rotate(q, [i], rad, "halves") * rope.norm_rotate(k, [j], rad, "halves")).sum())

    assert abs(product(5, 2) - product(100003, 100000)) < 1e-11 and abs(product(5, 2) - product(2 ** 31 - 1, 2 ** 31 - 4)) < 1e-11


def test_norm():
    x, w = np.arange(1.0, 9.0).reshape(1, 1, 8), np.arange(8.0)
    got = rope.norm_rotate(x, [3], [], "halves", w, 0.5)
    assert np.allclose(got, x / np.sqrt(25.5 + 0.5) * w, rtol=1e-15)
    assert np.allclose((rope.norm_rotate(x, [3], [], "halves", np.ones(8)) ** 2).mean(), 1.0)


def test_far_angles_are_exact():
    # pi as a float64 is 1.2246e-16 short of pi: over an even number of half turns the angle is what is missing
    assert np.isclose(rope.angles([2 ** 30], [np.pi])[0, 0], 2 * np.pi - 2 ** 30 * 1.2246467991473532e-16, rtol=1e-14)
    assert rope.angles([0], [np.pi])[0, 0] == 0.0
