"""Pins of the float64 network with layer norms: its gradients against differences of its objective."""
import numpy as np
import pytest

from oracle.network import LAYERNORM, PNORM, TANH, NGSGDNetwork


def network(nonlin, renorm=False, method="online"):
    rng = np.random.default_rng(11)
    dims = [8, 12, 15, 7]
    din = [8] + [d // 3 if n & ~LAYERNORM == PNORM else d for d, n in zip(dims[1:3], nonlin)]
    weights = [0.6 * rng.standard_normal((dims[l + 1], din[l] + 1)) for l in range(3)]
    net = NGSGDNetwork(dims, nonlin, weights, pnorm_group=3, rank_in=2, rank_out=2, renorm=renorm, method=method)
    for l in range(2):
        net.gain[l] = 1.0 + 0.3 * rng.standard_normal(din[l + 1])
        net.shift[l] = 0.3 * rng.standard_normal(din[l + 1])
    return net, rng.standard_normal((9, 8)), rng.integers(0, 7, 9)


@pytest.mark.parametrize("nonlin,renorm", [([TANH | LAYERNORM, TANH], False), ([TANH, PNORM | LAYERNORM], False),
                                           ([PNORM | LAYERNORM, TANH | LAYERNORM], True)])
def test_gradients_are_differences(nonlin, renorm):
    net, x, y = network(nonlin, renorm)
    grads = net.gradients(x, y)
    norms = dict(net.norm_gradients)
    assert sorted(norms) == [l for l, n in enumerate(nonlin) if n & LAYERNORM]
    h = 1e-6
    places = [(net.W[l], grads[l]) for l in range(3)]
    places += [(p[l], norms[l][k]) for l in norms for k, p in ((0, net.gain), (1, net.shift))]
    for p, g in places:
        assert p.shape == g.shape
        for i in np.ndindex(p.shape):
            keep = p[i]
            p[i] = keep + h
            up = net.objective(x, y)
            p[i] = keep - h
            down = net.objective(x, y)
            p[i] = keep
            assert abs((up - down) / (2 * h) - g[i]) < 1e-6 * max(1.0, abs(g[i]))


def test_layer_norms_are_updated_upwards():
    net, x, y = network([TANH | LAYERNORM, TANH | LAYERNORM])
    gain, shift = [g.copy() for g in net.gain], [s.copy() for s in net.shift]
    net.step(x, y, 0.01)
    for l in range(2):
        for before, after, g in ((gain[l], net.gain[l], net.norm_gradients[l][0]), (shift[l], net.shift[l], net.norm_gradients[l][1])):
            assert np.allclose(after - before, 0.01 * np.sign(g), rtol=1e-4)     # the first step of AdamW


def test_adamw_moves_every_matrix():
    net, x, y = network([TANH | LAYERNORM, TANH], method="adamw")
    net.adamw["decay"] = 0.5
    before = [w.copy() for w in net.W]
    obj = net.step(x, y, 0.01)
    for w, b, d in zip(net.W, before, net.last["delta"]):
        assert np.allclose(w, b * (1 - 0.005) + 0.01 * np.sign(d), atol=1e-6)
    for _ in range(20):
        last = net.step(x, y, 0.01)
    assert last > obj
