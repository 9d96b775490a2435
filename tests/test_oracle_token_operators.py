"""Pins of the float64 embedding, cross-entropy and clipping: known results, gradients against differences."""
import numpy as np
import pytest

from oracle import clipping, cross_entropy, embedding


def test_embedding_of_known_tokens():
    table = np.array([[1.0, 2.0], [3.0, 4.0], [5.0, 6.0]])
    assert np.array_equal(embedding.forward([2, -1, 0, 3], table, 0.5), [[2.5, 3.0], [0, 0], [0.5, 1.0], [0, 0]])
    dy = np.array([[1.0, 10.0], [2.0, 20.0], [4.0, 40.0], [8.0, 80.0]])
    assert np.array_equal(embedding.backward(dy, [1, -1, 1, 0], 3, 2.0), [[16, 160], [10, 100], [0, 0]])


def test_embedding_gradient_is_its_difference():
    """The lookup is linear in the table: a difference is exact but for rounding (eps / h of sums of 12 numbers)."""
    rng = np.random.default_rng(0)
    table, tokens = rng.standard_normal((5, 3)), np.array([4, 0, 4, -7, 2, 5, 4, 0, 4])
    dy = rng.standard_normal((len(tokens), 3))
    grad = embedding.backward(dy, tokens, 5, 1.7)
    for i in np.ndindex(table.shape):
        up, down = table.copy(), table.copy()
        up[i] += 0.5
        down[i] -= 0.5
        slope = np.sum(dy * (embedding.forward(tokens, up, 1.7) - embedding.forward(tokens, down, 1.7)))
        assert abs(slope - grad[i]) < 1e-13


def test_cross_entropy_of_known_rows():
    loss, d = cross_entropy.cross_entropy([[0.0, 0.0], [np.log(3.0), 0.0], [5.0, 9.0], [-np.inf, 2.0]], [0, 1, -1, 1], 2.0)
    assert np.allclose(loss, [np.log(2.0), np.log(4.0), 0.0, 0.0])
    assert np.allclose(d, 2.0 * np.array([[-0.5, 0.5], [0.75, -0.75], [0, 0], [0, 0]]))
    loss, d = cross_entropy.cross_entropy([[60.0, 0.0, 0.0], [-np.inf, 1.0, 1.0]], [0, 0])
    assert loss[0] == pytest.approx(2 * np.exp(-60.0), rel=1e-14) and d[0, 0] == pytest.approx(-2 * np.exp(-60.0), rel=1e-14)
    assert loss[1] == np.inf and np.array_equal(d[1], [-1.0, 0.5, 0.5])
    assert all(np.isnan(cross_entropy.cross_entropy([row], [0])[0][0]) for row in ([np.nan, 0.0], [np.inf, 0.0], [-np.inf, -np.inf]))


def test_cross_entropy_gradient_is_its_difference():
    rng = np.random.default_rng(1)
    x, labels = 2.0 * rng.standard_normal((4, 6)), np.array([0, 5, 6, 3])
    _, d = cross_entropy.cross_entropy(x, labels, 0.3)
    assert np.allclose(d.sum(axis=1), 0.0, atol=1e-15)
    h = 1e-5
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += h
        down[i] -= h
        slope = 0.3 * (cross_entropy.cross_entropy(up, labels)[0].sum() - cross_entropy.cross_entropy(down, labels)[0].sum()) / (2 * h)
        assert abs(slope - d[i]) < 1e-9     # h^2 / 6 times a third derivative below 1, and eps / h times sums of about 10


def test_clipping():
    t = [np.array([3.0, 0.0]), None, np.array([[4.0]])]
    assert clipping.norm_and_factor(t, 2.5) == (5.0, 0.5) and clipping.norm_and_factor(t, 5.0) == (5.0, 1.0)
    assert clipping.norm_and_factor([np.zeros(3)], 0.0) == (0.0, 1.0)
    assert clipping.norm_and_factor([np.array([np.inf, 1.0])], 1.0) == (np.inf, 0.0)
    assert np.isnan(clipping.norm_and_factor([np.array([np.nan, np.inf])], 1.0)).all()
