"""GPU parity: networks with layer norms and with AdamW as their method, through the C ABI, against the float64 oracle.

Bar: 1e-4 relative Frobenius error per gradient on the same inputs, as for the other networks; the weights of each step are taken
from the oracle, so that steps do not add their rounding up.
"""
import numpy as np
import pytest

import workloads
from oracle import adamw as oracle_adamw
from oracle.network import LAYERNORM, NGSGDNetwork

pytestmark = pytest.mark.gpu

TOL = 1.0e-4
TANH, PNORM = workloads.TANH, workloads.PNORM


def rel(a, b):
    a, b = np.asarray(a, np.float64), np.asarray(b, np.float64)
    return float(np.linalg.norm(a - b) / max(np.linalg.norm(b), 1e-300))


def cuda(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()


class Pair:
    def __init__(self, ngsgd, dims, nonlin, rows, method="online", renorm=False, group=5, ranks=(4, 8), max_change=0.0, seed=0, **gpu):
        import torch
        self.torch, self.ngsgd, self.rng = torch, ngsgd, np.random.default_rng(500 + seed)
        self.dims, self.nonlin, self.rows = dims, nonlin, rows
        din, in_dims = dims[0], []
        for l in range(len(dims) - 1):
            in_dims.append(din)
            if l < len(nonlin):
                din = dims[l + 1] // group if nonlin[l] & ~LAYERNORM == PNORM else dims[l + 1]
        self.in_dims = in_dims
        weights = [np.concatenate([self.rng.standard_normal((dims[l + 1], d)) / np.sqrt(d), 0.1 * self.rng.standard_normal((dims[l + 1], 1))], 1)
                   for l, d in enumerate(in_dims)]
        weights = [w.astype(np.float32).astype(np.float64) for w in weights]
        self.ora = NGSGDNetwork(dims, nonlin, weights, group, *ranks, renorm=renorm, max_change_per_sample=max_change,
                                method="adamw" if method == "adamw8" else method)
        self.gpu = ngsgd.Network(dims, nonlin, rows, group, *ranks, renorm=renorm, max_change_per_sample=max_change, method=method, **gpu)
        self.norms = [l for l, n in enumerate(nonlin) if n & LAYERNORM]
        for l in self.norms:
            w, b = self.gpu.get_norm(l)
            assert bool((w == 1).all()) and bool((b == 0).all())
            self.ora.gain[l] = (1.0 + 0.2 * self.rng.standard_normal(in_dims[l + 1])).astype(np.float32).astype(np.float64)
            self.ora.shift[l] = (0.2 * self.rng.standard_normal(in_dims[l + 1])).astype(np.float32).astype(np.float64)
        self.give_weights()

    def give_weights(self):
        for l, w in enumerate(self.ora.W):
            self.gpu.set_params(l, cuda(self.torch, w))
        for l in self.norms:
            self.gpu.set_norm(l, cuda(self.torch, self.ora.gain[l]), cuda(self.torch, self.ora.shift[l]))

    def minibatch(self, rows=None):
        rows = self.rows if rows is None else rows
        x = self.rng.standard_normal((rows, self.dims[0])).astype(np.float32)
        y = self.rng.integers(0, self.dims[-1], rows).astype(np.int32)
        return x, y

    def step(self, lr, rows=None):
        torch = self.torch
        x, y = self.minibatch(rows)
        before = [w.copy() for w in self.ora.W], {l: (self.ora.gain[l].copy(), self.ora.shift[l].copy()) for l in self.norms}
        objective = self.ora.step(x.astype(np.float64), y, lr)
        out = self.gpu.step(cuda(torch, x), torch.from_numpy(y).cuda(), lr)
        torch.cuda.synchronize()
        assert abs(float(out.item()) - objective) / len(y) < 1e-4
        for l in range(len(self.dims) - 1):
            assert rel(self.gpu.last_gradient(l).cpu().numpy(), self.ora.last["delta"][l]) < TOL, l
        for l in self.norms:
            for got, want in zip(self.gpu.last_norm_gradient(l), self.ora.norm_gradients[l]):
                assert rel(got.cpu().numpy(), want) < TOL, l
        # What moved.  Natural gradients: by lr times a gradient, and weights near 1 are rounded to fp32 (u against lr times some 0.1: 1e-3).
        # AdamW's first steps are lr times little more than the gradient's sign: with gradients off by TOL of their root mean square, a
        # share of 0.8 TOL of normally distributed ones is smaller than that and may move the other way, by 2 lr: 2 sqrt(0.8 TOL) = 1.8e-2.
        for l, w in enumerate(self.ora.W):
            tol = 2e-2 if self.ora.method == "adamw" else 2e-3
            assert rel(self.gpu.get_params(l).double().cpu().numpy() - before[0][l], w - before[0][l]) < tol, l
        for l in self.norms:
            for got, want, b in zip(self.gpu.get_norm(l), (self.ora.gain[l], self.ora.shift[l]), before[1][l]):
                assert rel(got.double().cpu().numpy() - b, want - b) < 2e-2, l
        self.give_weights()


NETS = [([24, 40, 48, 20], [TANH | LAYERNORM, TANH | LAYERNORM], 64), ([24, 200, 33, 20], [PNORM | LAYERNORM, TANH], 70),
        ([40, 300, 1030, 515, 203], [TANH, TANH | LAYERNORM, PNORM | LAYERNORM], 129), ([16, 2100, 30], [TANH | LAYERNORM], 33),
        ([16, 3000, 600], [PNORM | LAYERNORM], 40)]


@pytest.mark.parametrize("method", ["online", "simple", "adamw"])
@pytest.mark.parametrize("dims,nonlin,rows", NETS)
def test_steps_match_the_oracle(ngsgd, dims, nonlin, rows, method):
    """Split and whole backward products, every row kernel, mixed layers."""
    p = Pair(ngsgd, dims, nonlin, rows, method)
    for t in range(3):
        p.step(1e-3)


@pytest.mark.parametrize("dims,nonlin,rows", [([16, 30, 200, 700, 400, 300], [PNORM | LAYERNORM] + [TANH | LAYERNORM] * 3, 40),
                                              ([16, 2080, 9000, 600], [TANH | LAYERNORM] * 2, 33), ([16, 17000, 600], [TANH | LAYERNORM], 5)])
def test_every_width_of_row(ngsgd, dims, nonlin, rows):
    """Rows of 6, 200, 700, 400 numbers (parts of a wavefront), 2080 and 9000 (workgroups), most behind split products, and 17000 (from memory)."""
    p = Pair(ngsgd, dims, nonlin, rows, method="adamw")
    for t in range(2):
        p.step(1e-3)


@pytest.mark.parametrize("side_streams", [1, 3])
def test_past_the_always_update_phase(ngsgd, side_streams):
    p = Pair(ngsgd, [24, 200, 60, 50], [PNORM | LAYERNORM, TANH | LAYERNORM], 64, renorm=True, max_change=0.075, side_streams=side_streams)
    for t in range(14):
        p.step(1e-3)


def test_minibatches_of_other_sizes(ngsgd):
    p = Pair(ngsgd, [24, 200, 60, 50], [PNORM | LAYERNORM, TANH | LAYERNORM], 300, method="adamw")
    for rows in (300, 1, 2, 17, 299):
        p.step(1e-3, rows)


def test_numbers_of_adamw(ngsgd):
    p = Pair(ngsgd, [24, 60, 50], [TANH | LAYERNORM], 64, method="adamw")
    p.gpu.set_adamw(rate=0.5, betas=(0.8, 0.95), epsilon=1e-3, weight_decay=0.25)
    p.ora.adamw = dict(beta1=0.8, beta2=0.95, epsilon=1e-3, decay=0.25, rate=0.5)
    for t in range(4):
        p.step(1e-2)
    p.gpu.set_adamw()                     # forgets the moments
    p.ora.adamw = dict(beta1=0.9, beta2=0.999, epsilon=1e-8, decay=0.0, rate=1.0)
    p.ora.reset_adamw()
    for t in range(2):
        p.step(1e-3)


def test_moments_in_8_bits(ngsgd):
    """The step from the network's own gradients.  Codes are by the element's place among the padded rows; the gradient that is read back may
    differ in its last bit from the one that was used, which moves one code in 10^5 by a step, an eighth of the element's own."""
    import torch
    p = Pair(ngsgd, [24, 65, 50], [TANH | LAYERNORM], 64, method="adamw8")
    lr = 1e-3
    lds = [-(-(d + 1) // 32) * 32 for d in p.in_dims]
    rows = [d for d in p.dims[1:]]

    def flat(parts):        # as the network lays its weight matrices out
        out = [np.pad(a, ((0, 0), (0, ld - a.shape[1]))).reshape(-1) for a, ld in zip(parts, lds)]
        return np.concatenate(out)

    size = sum(r * ld for r, ld in zip(rows, lds))
    padded = -(-size // 256) * 256
    m, v = np.zeros(padded), np.zeros(padded)
    for t in range(1, 4):
        x, y = p.minibatch()
        before = flat([p.gpu.get_params(l).double().cpu().numpy() for l in range(2)])
        p.gpu.step(cuda(torch, x), torch.from_numpy(y).cuda(), lr)
        g = flat([-p.gpu.last_gradient(l).double().cpu().numpy() for l in range(2)])
        after = flat([p.gpu.get_params(l).double().cpu().numpy() for l in range(2)])
        want, m1, v1 = oracle_adamw.step(before, g, m[:size], v[:size], t, lr)
        d = np.abs(after - want)
        assert d.max() <= 0.2 * lr and np.sqrt(np.mean(d ** 2)) <= 2e-3 * lr
        m = oracle_adamw.coded(oracle_adamw.coded_m, np.pad(m1, (0, padded - size)), t)
        v = oracle_adamw.coded(oracle_adamw.coded_v, np.pad(v1, (0, padded - size)), t)


@pytest.mark.parametrize("method", ["adamw", "adamw8", "online"])
def test_captured_steps(ngsgd, method):
    """A captured step, replayed with new minibatches between eager work, against the same steps issued one by one."""
    import torch
    nets = [Pair(ngsgd, [24, 200, 60, 50], [PNORM | LAYERNORM, TANH | LAYERNORM], 64, method=method) for _ in range(2)]
    a, b = nets[0].gpu, nets[1].gpu
    data = [(cuda(torch, x), torch.from_numpy(y).cuda()) for x, y in (nets[0].minibatch() for _ in range(17))]
    x, y = (t.clone() for t in data[0])
    for k in range(11):      # past the steps that update every factor: t = 11 updates none
        a.step(*data[k], 1e-3)
        b.step(*data[k], 1e-3)
    a.join()
    b.join()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step(x, y, 1e-3)
        b.join()
    if method == "online":   # the host's counter of steps moved with the capture; the factors are those of step 11 in every replay
        x.copy_(data[11][0])
        y.copy_(data[11][1])
        graph.replay()
        a.step(*data[11], 1e-3)
        a.join()
        torch.cuda.synchronize()
        pairs = [(p.get_params(l), q.get_params(l)) for p, q in ((a, b),) for l in range(3)]
        pairs += [pq for l in range(2) for pq in zip(a.get_norm(l), b.get_norm(l))]
        assert all(rel(p.cpu().numpy(), q.cpu().numpy()) < 1e-6 for p, q in pairs)
        return
    for k in range(11, 17):
        x.copy_(data[k][0])
        y.copy_(data[k][1])
        graph.replay()
        torch.ones(1000, device="cuda").sum().item()
        a.step(*data[k], 1e-3)
        torch.cuda.synchronize()
        for l in range(3):
            assert torch.equal(a.get_params(l), b.get_params(l)), (k, l)
        for l in range(2):
            assert all(torch.equal(p, q) for p, q in zip(a.get_norm(l), b.get_norm(l))), (k, l)


@pytest.mark.parametrize("method", ["online", "adamw"])
def test_average_of_replicas(ngsgd, method):
    """Layer norms are averaged with the weights; with a reset AdamW starts anew.  Each replica on a stream of its own."""
    import torch
    pairs = [Pair(ngsgd, [24, 200, 60, 50], [PNORM | LAYERNORM, TANH | LAYERNORM], 64, method=method, seed=s) for s in range(3)]
    streams = [torch.cuda.Stream() for _ in pairs]
    torch.cuda.synchronize()
    for reset in (False, True):
        batches = []
        for p, s in zip(pairs, streams):
            for _ in range(2):
                x, y = p.minibatch()
                batches.append((cuda(torch, x), torch.from_numpy(y).cuda()))
                s.wait_stream(torch.cuda.current_stream())
                p.gpu.step(*batches[-1], 1e-3, stream=s)
        torch.cuda.synchronize()
        before = [[p.gpu.get_params(l).double() for l in range(3)] + [v.double() for l in range(2) for v in p.gpu.get_norm(l)] for p in pairs]
        ngsgd.average([p.gpu for p in pairs], reset_preconditioners=reset)
        torch.cuda.synchronize()
        for p in pairs:
            after = [p.gpu.get_params(l) for l in range(3)] + [v for l in range(2) for v in p.gpu.get_norm(l)]
            for k, got in enumerate(after):
                assert rel(got.cpu().numpy(), sum(b[k] for b in before).cpu().numpy() / 3) < 1e-6
    # the moments are gone: a step of lr in every direction
    p = pairs[0]
    x, y = p.minibatch()
    before = [v.clone() for l in range(2) for v in p.gpu.get_norm(l)]
    p.gpu.step(cuda(torch, x), torch.from_numpy(y).cuda(), 1e-3)
    for old, new, g in zip(before, [v for l in range(2) for v in p.gpu.get_norm(l)], [v for l in range(2) for v in p.gpu.last_norm_gradient(l)]):
        moved = (new.double() - old.double()).cpu().numpy()
        big = g.abs().cpu().numpy() > 1e-4
        assert np.allclose(moved[big], 1e-3 * np.sign(g.cpu().numpy()[big]), rtol=2e-3)


def test_another_rule_for_everything_else_stays(ngsgd):
    """A network without layer norms steps as it did: its weights do not depend on whether another network has them."""
    import torch
    plain = [Pair(ngsgd, [24, 60, 50], [TANH], 64) for _ in range(2)]
    other = Pair(ngsgd, [24, 60, 50], [TANH | LAYERNORM], 64)
    for _ in range(3):
        x, y = plain[0].minibatch()
        args = cuda(torch, x), torch.from_numpy(y).cuda(), 1e-3
        plain[0].gpu.step(*args)
        other.gpu.step(*args)
        plain[1].gpu.step(*args)
    torch.cuda.synchronize()
    for l in range(2):
        assert rel(plain[0].gpu.get_params(l).cpu().numpy(), plain[1].gpu.get_params(l).cpu().numpy()) < 1e-6


def test_refusals(ngsgd):
    import torch
    plain = ngsgd.Network([24, 60, 50], [TANH], 64, rank_in=4, rank_out=8)
    normed = ngsgd.Network([24, 60, 50], [TANH | LAYERNORM], 64, rank_in=4, rank_out=8)
    v = torch.zeros(60, device="cuda")
    for bad in (lambda: plain.get_norm(0), lambda: plain.set_norm(0, v), lambda: plain.set_adamw(), lambda: normed.get_norm(1), lambda: normed.get_norm(-1),
                lambda: normed.last_norm_gradient(0), lambda: normed.set_adamw(epsilon=0.0), lambda: normed.set_adamw(betas=(1.0, 0.9)),
                lambda: normed.set_adamw(rate=float("inf")), lambda: normed.set_adamw(weight_decay=float("nan")),
                lambda: ngsgd.Network([24, 60, 50], [TANH], 64, rank_in=4, rank_out=8, method="adamw", max_change_per_sample=0.1),
                lambda: ngsgd.Network([24, 60, 50], [LAYERNORM + 2], 64, rank_in=4, rank_out=8),
                lambda: ngsgd.average([plain, normed])):
        with pytest.raises(ngsgd.NgsgdError):
            bad()
    with pytest.raises(ValueError):
        normed.set_norm(0, v[:59])
    x, y = torch.zeros(64, 24, device="cuda"), torch.zeros(64, dtype=torch.int32, device="cuda")
    for lr in (float("nan"), float("inf"), 1e30):
        with pytest.raises(ngsgd.NgsgdError):
            normed.step(x, y, lr)
    w, b = normed.get_norm(0)
    assert bool((w == 1).all()) and bool((b == 0).all())
