"""Embedding, layer norm, cross-entropy, gradient norm and AdamW together, as a program that trains a model of tokens calls them, against the float64
definitions.

The model: tokens -> embedding (table E) -> layer norm (w, b) -> product with the same table (x = y E^T) -> cross-entropy of the next token.
The table's gradient is that of the product, with the embedding's added to it.
"""
import numpy as np
import pytest

from oracle import adamw, clipping, cross_entropy, embedding, layer_norm

pytestmark = pytest.mark.gpu

LR, BOUND = 1e-2, 0.5


def rel(a, b):
    a, b = np.asarray(a, np.float64), np.asarray(b, np.float64)
    return float(np.linalg.norm(a - b) / max(np.linalg.norm(b), 1e-300))


def batch(rng, N, V):
    t = rng.integers(0, V, N + 1)
    tokens, labels = t[:-1].copy(), t[1:].copy()
    tokens[-(N // 5):], labels[-(N // 5) - 1:] = -1, -1          # the batch's padding
    return tokens, labels


class Program:
    def __init__(self, ngsgd, N, V, D, seed=0):
        import torch
        rng = np.random.default_rng(seed)
        self.torch, self.N = torch, N
        self.E = torch.from_numpy(0.3 * rng.standard_normal((V, D))).float().cuda()
        self.w, self.b = torch.ones(D, device="cuda"), torch.zeros(D, device="cuda")
        self.tokens, self.labels = (torch.zeros(N, dtype=torch.int64, device="cuda") for _ in range(2))
        self.scale = torch.ones(1, device="cuda")
        self.embed = ngsgd.Embedding(N, V, D, scale=float(np.sqrt(D)))
        self.ln, self.ce = ngsgd.LayerNorm(N, D), ngsgd.CrossEntropy(N, V)
        self.opt = ngsgd.AdamW([self.E, self.w, self.b], weight_decay=[0.01, 0.0, 0.0])
        self.clip = ngsgd.GradientNorm([self.E, self.w, self.b])

    def give(self, tokens, labels):
        torch = self.torch
        self.tokens.copy_(torch.from_numpy(tokens))
        self.labels.copy_(torch.from_numpy(labels))
        self.scale.fill_(1.0 / max(1, int((labels >= 0).sum())))

    def step(self):
        x = self.embed.forward(self.tokens, self.E)
        y, mean, rstd = self.ln.forward(x, self.w, self.b)
        logits = y @ self.E.t()
        loss, d = self.ce.gradient(logits, self.labels, scale=self.scale, dlogits=logits)
        dE = d.t() @ y
        dx, dw, db = self.ln.backward(d @ self.E, x, mean, rstd, self.w)
        self.embed.backward(dx, self.tokens, dtable=dE, accumulate=True)
        norm, factor = self.clip.norm([dE, dw, db], BOUND)
        self.opt.step([dE, dw, db], LR, grad_scale=factor)
        return loss, dE, dw, db, norm, factor

    def values(self):
        return [p.double().cpu().numpy() for p in (self.E, self.w, self.b)]


def expected(E, w, b, tokens, labels, V, D):
    root = float(np.float32(np.sqrt(D)))
    x = embedding.forward(tokens, E, root)
    y, mean, rstd = layer_norm.forward(x, w, b)
    loss, d = cross_entropy.cross_entropy(y @ E.T, labels, 1.0 / max(1, int((labels >= 0).sum())))
    dx, dw, db = layer_norm.backward(d @ E, x, mean, rstd, w)
    return loss, d.T @ y + embedding.backward(dx, tokens, V, root), dw, db


@pytest.mark.parametrize("N,V,D", [(40, 30, 24), (200, 1000, 65), (9000, 50, 16)])
def test_steps_follow_the_definitions(ngsgd, N, V, D):
    """Losses and gradients to 1e-4: products in fp32 of at most N = 9000 terms with N u = 5e-4 as the worst and their root as the usual error, behind a layer
    norm whose rows of padding (all zero) have a rstd of 300.  The norm and the factor from those gradients to fp32's rounding, the step from them to
    AdamW's (24 u of 10 lr a step, 4 u of the parameters)."""
    p, rng, u = Program(ngsgd, N, V, D), np.random.default_rng(1), 2.0 ** -24
    moments = [(np.zeros(v.shape), np.zeros(v.shape)) for v in p.values()]
    for t in range(1, 6):
        tokens, labels = batch(rng, N, V)
        p.give(tokens, labels)
        before = p.values()
        got = [a.double().cpu().numpy() for a in p.step()]
        want = expected(*before, tokens, labels, V, D)
        for g, e in zip(got[:4], want):
            assert rel(g, e) < 1e-4
        norm, factor = clipping.norm_and_factor(got[1:4], BOUND)
        assert abs(got[4][0] - norm) <= 2 * u * norm and abs(got[5][0] - factor) <= 2 * u * factor
        for k, (now, old, g, decay) in enumerate(zip(p.values(), before, got[1:4], (0.01, 0.0, 0.0))):
            step, m, v = adamw.step(old, g, *moments[k], t, float(np.float32(LR)), decay=float(np.float32(decay)), scale=float(np.float32(factor)))
            moments[k] = (m, v)
            assert np.all(np.abs(now - step) <= 4 * u * np.abs(old) + 24 * u * t * 10 * LR)


def test_captured_as_a_whole(ngsgd):
    """All calls of a step in one graph, replayed with new batches between eager work, equal the same calls one by one, bit for bit."""
    import torch
    rng = np.random.default_rng(2)
    N, V, D = 300, 90, 48
    a, b = (Program(ngsgd, N, V, D) for _ in range(2))
    first = batch(rng, N, V)
    for p in (a, b):
        p.give(*first)
        p.step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = b.step()
    for _ in range(5):
        now = batch(rng, N, V)
        a.give(*now)
        b.give(*now)
        want = a.step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(want, outs))
        assert all(np.array_equal(x, y) for x, y in zip(a.values(), b.values()))
    assert a.opt.steps() == b.opt.steps() == 6


def test_two_programs_on_two_streams(ngsgd):
    import torch
    rng = np.random.default_rng(3)
    N, V, D = 2000, 300, 64
    want = Program(ngsgd, N, V, D)
    both = [Program(ngsgd, N, V, D) for _ in range(2)]
    now = batch(rng, N, V)
    for p in [want] + both:
        p.give(*now)
    for _ in range(4):
        want.step()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in both]
    for _ in range(4):
        for p, s in zip(both, streams):
            with torch.cuda.stream(s):
                p.step()
    torch.cuda.synchronize()
    for p in both:
        assert all(np.array_equal(x, y) for x, y in zip(p.values(), want.values()))
