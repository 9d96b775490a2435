"""Layer norm and AdamW together, as a program with a network of its own calls them, against the float64 definitions.

The model: rows x -> layer norm (w, b) -> product with a matrix V -> squared distance to a target, summed.  The gradient of V is
preconditioned by nothing here; w, b and V are one AdamW's tensors.
"""
import numpy as np
import pytest

from oracle import adamw, layer_norm

pytestmark = pytest.mark.gpu


def rel(a, b):
    a, b = np.asarray(a, np.float64), np.asarray(b, np.float64)
    return float(np.linalg.norm(a - b) / max(np.linalg.norm(b), 1e-300))


class Program:
    def __init__(self, ngsgd, N, D, H, bits, dtype="float32", master=False, seed=0):
        import torch
        rng = np.random.default_rng(seed)
        self.torch, self.N, self.D, self.H = torch, N, D, H
        self.dtype = getattr(torch, dtype)
        self.V = torch.from_numpy(0.1 * rng.standard_normal((D, H))).to(self.dtype).cuda()
        self.w = torch.ones(D, dtype=self.dtype, device="cuda")
        self.b = torch.zeros(D, dtype=self.dtype, device="cuda")
        self.x = torch.from_numpy(rng.standard_normal((N, D)) + 0.5).to(self.dtype).cuda()
        self.target = torch.from_numpy(rng.standard_normal((N, H))).cuda()
        self.ln = ngsgd.LayerNorm(N, D)
        self.opt = ngsgd.AdamW([self.V, self.w, self.b], weight_decay=[0.01, 0.0, 0.0], grad_dtype=torch.float32, state_bits=bits, master=master)

    def gradients(self):
        torch = self.torch
        y, mean, rstd = self.ln.forward(self.x, self.w, self.b)
        d = 2.0 * (y.double() @ self.V.double() - self.target)
        dy = (d @ self.V.double().t()).to(self.dtype)
        _, dw, db = self.ln.backward(dy, self.x, mean, rstd, self.w, needs=(False, True, True))
        return (y.double().t() @ d).float(), dw.float(), db.float(), d

    def step(self, lr):
        grads = self.gradients()
        self.opt.step(grads[:3], lr)
        return grads

    def values(self):
        return [p.double().cpu().numpy() for p in (self.V, self.w, self.b)]


@pytest.mark.parametrize("N,D,H", [(33, 100, 7), (64, 1030, 16), (7, 5, 3)])
def test_steps_follow_the_definitions(ngsgd, N, D, H):
    """Gradients to 1e-5 (sums of up to 64 rows in fp32: 64 u, and the layer norm's own), then the step from those gradients to fp32's
    rounding of the parameters (4 u) and of the step (24 u of lr, and no more than lr / (1 - beta1) = 10 lr long)."""
    p = Program(ngsgd, N, D, H, 32)
    x, target = p.x.double().cpu().numpy(), p.target.cpu().numpy()
    moments = [(np.zeros(v.shape), np.zeros(v.shape)) for v in p.values()]
    lr, u = float(np.float32(1e-2)), 2.0 ** -24
    for t in range(1, 9):
        before = p.values()
        V, w, b = before
        y, mean, rstd = layer_norm.forward(x, w, b)
        d = 2.0 * (y @ V - target)
        _, dw, db = layer_norm.backward(d @ V.T, x, mean, rstd, w)
        got = p.step(1e-2)
        for g, want in zip(got, (y.T @ d, dw, db)):
            assert rel(g.cpu().numpy(), want) < 1e-5
        for k, (now, old, g, decay) in enumerate(zip(p.values(), before, got, (0.01, 0.0, 0.0))):
            want, m, v = adamw.step(old, g.double().cpu().numpy(), *moments[k], t, lr, decay=float(np.float32(decay)))
            moments[k] = (m, v)
            assert np.all(np.abs(now - want) <= 4 * u * np.abs(old) + 24 * u * t * 10 * lr)


@pytest.mark.parametrize("bits,dtype,master", [(32, "float32", False), (8, "float32", False), (8, "bfloat16", True)])
def test_captured_as_a_whole(ngsgd, bits, dtype, master):
    """Forward, backward and step in one graph, replayed between eager work, equal the same calls one by one, bit for bit."""
    import torch
    a, b = (Program(ngsgd, 64, 300, 8, bits, dtype, master) for _ in range(2))
    dy = torch.randn(64, 300, device="cuda").to(a.dtype)

    def calls(p):
        y, mean, rstd = p.ln.forward(p.x, p.w, p.b)
        _, dw, db = p.ln.backward(dy, p.x, mean, rstd, p.w, needs=(False, True, True))
        p.opt.step([None, dw.float(), db.float()], 1e-2)

    for p in (a, b):
        calls(p)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(b)
    for _ in range(5):
        dy.normal_()
        calls(a)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a.w, b.w) and torch.equal(a.b, b.b) and all(torch.equal(p, q) for p, q in zip(a.opt.state(), b.opt.state()))
    assert a.opt.steps() == b.opt.steps() == 6


def test_two_programs_on_two_streams(ngsgd):
    """Two objects, each on a stream of its own, at the same time."""
    import torch
    want = Program(ngsgd, 64, 700, 8, 8)
    both = [Program(ngsgd, 64, 700, 8, 8) for _ in range(2)]
    for _ in range(6):
        want.step(1e-2)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in both]
    for _ in range(6):
        for p, s in zip(both, streams):
            with torch.cuda.stream(s):
                p.step(1e-2)
    torch.cuda.synchronize()
    for p in both:
        assert all(np.array_equal(x, y) for x, y in zip(p.values(), want.values()))


def test_objects_that_are_gone_before_their_work(ngsgd):
    """Calls on another stream than the objects were made on, the objects deleted before that stream gets to them: their workspaces are
    nobody else's until then."""
    import torch
    N, D = 4000, 2000
    torch.manual_seed(5)
    x, dy = torch.randn(N, D, device="cuda"), torch.randn(N, D, device="cuda")
    w = torch.ones(D, device="cuda")
    y, mean, rstd = ngsgd.LayerNorm(N, D).forward(x, w)
    want = ngsgd.LayerNorm(N, D).backward(dy, x, mean, rstd, w)
    start = torch.randn(300000, device="cuda")
    grad = torch.randn(300000, device="cuda")
    moved = start.clone()
    ngsgd.AdamW([moved], state_bits=8).step([grad], 0.1)
    s = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device="cuda")
    for given in (True, False):
        ln, p = ngsgd.LayerNorm(N, D), start.clone()
        opt = ngsgd.AdamW([p], state_bits=8)
        sizes = [ln.workspace.numel(), opt.workspace.numel()]
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for _ in range(30):          # some milliseconds before its turn
                big = big @ big * 1e-3
            if not given:
                got = ln.backward(dy, x, mean, rstd, w)
                opt.step([grad], 0.1)
        if given:
            got = ln.backward(dy, x, mean, rstd, w, stream=s)
            opt.step([grad], 0.1, stream=s)
        del ln, opt
        taken = [torch.zeros(n, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(3)]   # (a table of zeros is one without work)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(p, moved)
        del taken
