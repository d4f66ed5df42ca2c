"""The oracle's rotation and masks against their properties (CPU only)."""
import numpy as np
import pytest

from oracle import paged as ref


@pytest.mark.parametrize("layout", ["halves", "neighbours"])
def test_rotation_keeps_products_of_equal_distances(layout):
    """Turned queries and keys: their product depends on the positions' difference alone."""
    rng = np.random.default_rng(0)
    freq, axis = 100.0 ** (-np.arange(4) / 4), [0, 0, 1, 1]
    q, k = rng.standard_normal((2, 1, 1, 10))
    dot = []
    for shift in (0, 5, -300):
        p = np.array([[7], [-3]]) + shift
        r = np.array([[2], [11]]) + shift
        dot.append((ref.rotate(q, p, freq, axis, layout) * ref.rotate(k, r, freq, axis, layout)).sum())
    np.testing.assert_allclose(dot, dot[0], rtol=0, atol=1e-12)
    y = ref.rotate(q, np.zeros((2, 1)), freq, axis, layout)
    np.testing.assert_array_equal(y, q)
    np.testing.assert_array_equal(ref.rotate(q, np.ones((2, 1)), freq, axis, layout)[..., 8:], q[..., 8:])


def test_rotation_of_one_pair_is_a_turn():
    x = np.zeros((1, 1, 8))
    x[0, 0, 0] = 1.0
    y = ref.rotate(x, [[1]], [np.pi / 2], [0], "halves")
    np.testing.assert_allclose(y[0, 0], [0, 1, 0, 0, 0, 0, 0, 0], atol=1e-15)
    y = ref.rotate(x, [[1]], [np.pi / 2, 0, 0, 0], [0] * 4, "halves")
    np.testing.assert_allclose(y[0, 0], [0, 0, 0, 0, 1, 0, 0, 0], atol=1e-15)


def test_window_masks():
    w = ref.window([0, 5, -1, 99], 8, 3, 1)
    assert w.astype(int).tolist() == [[1, 0, 0, 0, 0, 0, 0, 0], [1, 0, 0, 1, 1, 1, 0, 0], [0] * 8, [1] + [0] * 7]
    assert ref.window([7], 8, 2 ** 31 - 1, 0).all() and not ref.window([-2 ** 31], 8, 2 ** 31 - 1, 8).any()


def test_tree_masks():
    m = np.array([[1, 0], [0b101, 1]], np.uint32)
    t = ref.tree(m, 40, 4)
    assert t[0].nonzero()[0].tolist() == [0, 1, 2, 3, 4]
    assert t[1].nonzero()[0].tolist() == [0, 1, 2, 3, 4, 6, 36]
    assert ref.tree(m[:1], 3, -5)[0].tolist() == [True, False, False]
    assert ref.tree(m, 2, 9).all()
