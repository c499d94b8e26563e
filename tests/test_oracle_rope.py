"""The oracle of norms and rotation against closed forms."""
import numpy as np
import pytest

from oracle import rope


def test_norm_by_hand():
    x = np.array([[3.0, 4.0, 0.0, 0.0]])
    got = rope.norm(x, np.array([1.0, 2.0, 1.0, 1.0]), 0.0)
    assert np.allclose(got.astype(float), [[1.2, 3.2, 0, 0]], atol=1e-15)  # mean square 25 / 4
    assert rope.norm(x, None, 1.0) is not None and np.array_equal(rope.norm(x, None, 1.0), x)
    assert np.allclose(rope.norm(x, np.ones(4), 2.75).astype(float), x / 3.0)  # the eps is inside the root


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_product_of_complex_numbers(interleaved):
    r = np.random.default_rng(1)
    y, pairs = r.standard_normal((5, 3, 16)), 6
    ang = rope.angles(r.integers(0, 50, (1, 5)), 0.7 ** np.arange(pairs))
    z = rope.rotate(y, ang, interleaved, 1.0)
    a, b = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if interleaved else (slice(0, pairs), slice(pairs, 2 * pairs))
    want = (y[..., a] + 1j * y[..., b]) * np.exp(1j * ang.astype(float))[:, None]
    assert np.allclose(z[..., a].astype(float), want.real) and np.allclose(z[..., b].astype(float), want.imag)
    assert np.array_equal(z[..., 2 * pairs:], y[..., 2 * pairs:])


def test_products_of_rotated_rows_depend_on_the_distance_alone():
    r = np.random.default_rng(2)
    q, k = r.standard_normal((2, 1, 1, 8))
    f = 0.3 ** np.arange(4)

    def score(i, j):
        return float((rope.rotate(q, rope.angles([[i]], f), False, 1.0) * rope.rotate(k, rope.angles([[j]], f), False, 1.0)).sum())

    assert np.isclose(score(9, 4), score(105, 100), atol=1e-12) and not np.isclose(score(9, 4), score(9, 5), atol=1e-3)


def test_axes_turn_their_own_pairs():
    f, axis = np.array([1.0, 0.5, 0.25]), [2, 0, 1]
    assert np.allclose(rope.angles([[1], [10], [100]], f, axis).astype(float), [[100.0, 0.5, 2.5]])


def test_planted_mistakes_are_seen():
    r = np.random.default_rng(3)
    y, ang = r.standard_normal((2, 1, 8)), rope.angles([[1, 2]], 0.5 ** np.arange(4))
    z = rope.rotate(y, ang, False, 1.0)
    for wrong in (rope.rotate(y, -ang, False, 1.0), rope.rotate(y, ang, True, 1.0), rope.rotate(y, ang[:, ::-1], False, 1.0),
                  rope.rotate(y, ang, False, 1.1)):
        assert np.abs((z - wrong).astype(float)).max() > 1e-2
