"""Pins of the float64 layer norm and AdamW: gradients against differences, the moments' codes against their rules."""
import numpy as np
import pytest

from oracle import adamw, layer_norm


def test_layer_norm_of_known_rows():
    x = np.array([[1.0, 3.0, 1.0, 3.0], [5.0, 5.0, 5.0, 5.0]])
    y, mean, rstd = layer_norm.forward(x, epsilon=0.25)
    assert np.array_equal(mean, [2.0, 5.0]) and np.allclose(rstd, [1.25 ** -0.5, 2.0])
    assert np.allclose(y[0], np.array([-1, 1, -1, 1]) * 1.25 ** -0.5) and np.array_equal(y[1], np.zeros(4))
    y, _, _ = layer_norm.forward(x, np.array([1.0, 2.0, 3.0, 4.0]), np.full(4, 7.0), epsilon=0.25)
    assert np.array_equal(y[1], np.full(4, 7.0)) and np.isclose(y[0, 3], 7.0 + 4.0 * 1.25 ** -0.5)


@pytest.mark.parametrize("N,D", [(1, 1), (1, 5), (4, 2), (3, 17)])
def test_layer_norm_gradients_are_differences(N, D):
    rng = np.random.default_rng(N * 100 + D)
    x, w, b, dy = rng.standard_normal((N, D)), rng.standard_normal(D), rng.standard_normal(D), rng.standard_normal((N, D))

    def f(x, w, b):
        return float(np.sum(layer_norm.forward(x, w, b)[0] * dy))

    _, mean, rstd = layer_norm.forward(x, w, b)
    h = 1e-6
    for at, grad in zip((0, 1, 2), layer_norm.backward(dy, x, mean, rstd, w)):
        args = [x, w, b]
        for i in np.ndindex(args[at].shape):
            up, down = [a.copy() for a in args], [a.copy() for a in args]
            up[at][i] += h
            down[at][i] -= h
            # rounding eps / h and, for one column, where f is constant, nothing else; the third derivative is of order
            # rstd^3 <= (1e-5)^(-3/2), times h^2
            assert abs((f(*up) - f(*down)) / (2 * h) - grad[i]) < 1e-7 * max(1.0, rstd.max() ** 3) * max(1.0, np.abs(dy).sum())


def test_adamw_of_a_constant_gradient():
    """With unbiased moments a constant gradient gives steps of lr sign(g) from the first one on."""
    p, m, v = np.array([1.0, -2.0]), np.zeros(2), np.zeros(2)
    g = np.array([0.5, -4.0])
    for t in range(1, 6):
        p, m, v = adamw.step(p, g, m, v, t, lr=0.1, epsilon=0.0)
        assert np.allclose(p, np.array([1.0, -2.0]) - 0.1 * t * np.sign(g))
    q, _, _ = adamw.step(np.ones(2), np.zeros(2), np.zeros(2), np.zeros(2), 1, lr=0.1, decay=0.5)
    assert np.allclose(q, 0.95)


def test_codes_are_fixed_points_and_monotone():
    rng = np.random.default_rng(3)
    for scale in (1.0, 1e-30, 1e20):
        m = rng.standard_normal(256) * np.exp2(rng.uniform(-20, 0, 256)) * scale
        v = (rng.standard_normal(256) * np.exp2(rng.uniform(-20, 0, 256)) * scale) ** 2
        for which, a in ((adamw.coded_m, m), (adamw.coded_v, v)):
            held = which(a)
            assert np.array_equal(which(held), held)
            order = np.argsort(a)
            assert np.all(np.diff(held[order]) >= 0)
        big = np.abs(m) > np.abs(m).max() * 2.0 ** -14
        assert np.all(np.abs(adamw.coded_m(m) - m)[big] <= np.abs(m)[big] / 16)
        assert np.all(np.abs(np.sqrt(adamw.coded_v(v)) - np.sqrt(v)) <= np.sqrt(v) / 16)
        assert len(np.unique(np.abs(adamw.coded_m(m)))) <= 128 and len(np.unique(adamw.coded_v(v))) <= 255


def test_values_fit_bfloat16():
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(4)
    for which, a in ((adamw.coded_m, rng.standard_normal(256)), (adamw.coded_v, rng.standard_normal(256) ** 2)):
        held = torch.from_numpy(which(a, adamw.share(256, 9)))
        assert torch.equal(held.to(torch.bfloat16).double(), held)


def test_shares_visit_the_unit_interval_evenly():
    """Over n steps the share of an element stays below any x about x n times (discrepancy of order log n)."""
    shares = np.array([adamw.share(3, t, 1000) for t in range(1, 1001)])
    for x in (0.1, 0.25, 0.5, 0.9):
        assert np.all(np.abs((shares < x).sum(axis=0) - 1000 * x) <= 8)


def test_small_changes_add_up():
    """v under a constant gradient: to nearest it stays, with the shares it reaches g^2."""
    v = np.full(256, 1.0)
    near = v.copy()
    for t in range(1, 8001):
        v = adamw.coded_v(0.999 * v + 0.001 * 4.0, adamw.share(256, t))
        near = adamw.coded_v(0.999 * near + 0.001 * 4.0)
    assert np.array_equal(near, np.full(256, 1.0))
    assert abs(v.mean() - 4.0) < 0.2   # the codes around the root 2 are an eighth and a quarter apart


def test_codes_stand_for_numbers_of_fp32():
    """The largest numbers that fp32 holds are held as numbers, whatever share of a step is added."""
    top = float(np.finfo(np.float32).max)
    for a in (np.array([top, 1.0, 0.0]), np.array([1.9 * 2.0 ** 126, 2.0 ** 126])):
        for share in (0.0, 0.5, 1.0 - 2.0 ** -20):
            m, v = adamw.coded_m(-a, share), adamw.coded_v(a, share)
            assert np.all(np.abs(m) <= 1.875 * 2.0 ** 127) and np.all(v <= (1.875 * 2.0 ** 63) ** 2)
            assert np.all(np.abs(m[:1] + a[0]) <= a[0] / 8) and np.all(np.abs(np.sqrt(v[:1]) - np.sqrt(a[0])) <= np.sqrt(a[0]) / 8)
