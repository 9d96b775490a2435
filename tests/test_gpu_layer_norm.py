"""GPU parity: layer norm and its gradients through the C ABI against the float64 definition.

Tolerances.  u = 2^-24 is half a step of fp32, u_t of the output's type; a number computed from K additions in fp32 is off by at most
K u times the sum of the magnitudes (a chain is at most D / 64 additions in a lane, or in a thread, and 24 behind it), and
each product, quotient or root adds u of its result.  K(D) = D / 64 + 24.
  mean: K u mean|x|.  rstd: the variance is off by K + 4 u of itself, and by the square of the mean's error, which rstd sees
  as half of that.  y = xhat w + b: xhat is off by rstd (error of the mean) + |xhat| (error of rstd + 3 u).
  dx = rstd (g - c1 - xhat c2): c1 and c2 are off by (K + 4) u of the mean magnitudes, the rest by 6 u of each term.
  dw, db: N + 8 additions at most, each term off by 4 u.
"""
import numpy as np
import pytest

from oracle import layer_norm as oracle

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
COMBOS = [("float32", "float32"), ("bfloat16", "float32"), ("bfloat16", "bfloat16"), ("float16", "float32"), ("float16", "float16")]


def half_step(torch, dtype):
    return torch.finfo(dtype).eps / 2


def tiny(torch, dtype):
    """Half a step among the smallest numbers of a type."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def inputs(torch, N, D, dtype, wtype, pad=0, seed=0, offset=0.0):
    rng = np.random.default_rng(1000 * N + D + seed)

    def rows(a):
        wide = torch.full((N, D + pad), 77.0, dtype=dtype, device="cuda")
        wide[:, :D] = torch.from_numpy(a).to(dtype).cuda()
        return wide[:, :D]

    x = rows(rng.standard_normal((N, D)) * rng.uniform(0.2, 3.0, (N, 1)) + rng.standard_normal((N, 1)) + offset)
    dy = rows(rng.standard_normal((N, D)))
    w = torch.from_numpy(1.0 + 0.3 * rng.standard_normal(D)).to(wtype).cuda()
    b = torch.from_numpy(0.3 * rng.standard_normal(D)).to(wtype).cuda()
    return x, dy, w, b


def f64(t):
    return t.detach().double().cpu().numpy()


def check_forward(torch, x, w, b, eps, y, mean, rstd):
    D = x.shape[-1]
    K = D / 64 + 24
    X = f64(x)
    want, m, r = oracle.forward(X, None if w is None else f64(w), None if b is None else f64(b), eps)
    W = np.ones(D) if w is None else f64(w)
    e_mean = K * U * np.abs(X).mean(axis=1) + U * np.abs(m)
    assert np.all(np.abs(f64(mean) - m) <= e_mean)
    e_rstd = r * ((K + 8) * U + 0.5 * (e_mean * r) ** 2)
    assert np.all(np.abs(f64(rstd) - r) <= e_rstd)
    xhat = np.abs((X - m[:, None]) * r[:, None])
    e_y = np.abs(W) * (r[:, None] * e_mean[:, None] + xhat * (e_rstd / r + 3 * U)[:, None]) + 3 * U * np.abs(want) + U * np.abs(W) * xhat
    u = half_step(torch, y.dtype)
    assert np.all(np.abs(f64(y) - want) <= e_y * (1 + 2 * u) + u * np.abs(want) + tiny(torch, y.dtype))


def check_backward(torch, dy, x, mean, rstd, w, dx, dw, db):
    N, D = x.shape
    K = D / 64 + 24
    DY, X, m, r = f64(dy), f64(x), f64(mean)[:, None], f64(rstd)[:, None]
    W = np.ones(D) if w is None else f64(w)
    want, want_dw, want_db = oracle.backward(DY, X, f64(mean), f64(rstd), None if w is None else W)
    xhat, g = np.abs((X - m) * r), np.abs(DY * W)
    if dx is not None:
        c1, c2 = g.mean(axis=1, keepdims=True), (g * xhat).mean(axis=1, keepdims=True)
        e = r * ((K + 10) * U * (c1 + xhat * c2) + 8 * U * g)
        u = half_step(torch, dx.dtype)
        assert np.all(np.abs(f64(dx) - want) <= e * (1 + 2 * u) + u * np.abs(want) + tiny(torch, dx.dtype))
    for got, ref, terms in ((dw, want_dw, np.abs(DY) * xhat), (db, want_db, np.abs(DY))):
        if got is not None:
            u = half_step(torch, got.dtype)
            e = (N + 12) * U * terms.sum(axis=0)
            assert np.all(np.abs(f64(got) - ref) <= e * (1 + 2 * u) + u * np.abs(ref) + tiny(torch, got.dtype))


def both(torch, ngsgd, x, dy, w, b, eps=1e-5):
    ln = ngsgd.LayerNorm(x.shape[0], x.shape[1], eps)
    y, mean, rstd = ln.forward(x, w, b)
    check_forward(torch, x, w, b, eps, y, mean, rstd)
    grads = ln.backward(dy, x, mean, rstd, w)
    check_backward(torch, dy, x, mean, rstd, w, *grads)
    return ln, (y, mean, rstd), grads


WIDTHS = [1, 2, 3, 7, 8, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 300, 511, 512, 513, 516, 1000, 1001, 1023, 1024, 1025, 1032, 2000, 2047, 2048,
          2049, 2056, 3000, 4095, 4096, 4097, 4104, 5000, 8191, 8192, 8193, 8200, 12000, 16383, 16384, 16385, 16392, 20001, 40000]


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("types", COMBOS, ids="-".join)
def test_widths(ngsgd, D, types):
    """Widths at and around every power of two, rows that start on no common boundary, few rows."""
    import torch
    dtype, wtype = (getattr(torch, t) for t in types)
    x, dy, w, b = inputs(torch, 5, D, dtype, wtype)
    both(torch, ngsgd, x, dy, w, b)


@pytest.mark.parametrize("N,D", [(1, 1), (1, 300), (2, 2048), (3, 8), (9, 100), (17, 512), (31, 513), (64, 128), (65, 1000), (93, 230), (129, 2048), (300, 77),
                                 (512, 300), (511, 1030), (2049, 24), (4001, 40), (3000, 264), (1025, 4100), (777, 8200)])
@pytest.mark.parametrize("types", [COMBOS[0], COMBOS[1], COMBOS[4]], ids="-".join)
def test_rows(ngsgd, N, D, types):
    """Row counts at and around what a workgroup and a grid take; several rows per workgroup."""
    import torch
    dtype, wtype = (getattr(torch, t) for t in types)
    both(torch, ngsgd, *inputs(torch, N, D, dtype, wtype))


@pytest.mark.parametrize("N,D,pad", [(9, 64, 1), (33, 100, 28), (50, 511, 1), (7, 1000, 24), (40, 2048, 8), (12, 4099, 5), (5, 16384, 3), (5, 20000, 16)])
@pytest.mark.parametrize("types", [COMBOS[0], COMBOS[2], COMBOS[3]], ids="-".join)
def test_rows_inside_a_wider_buffer(ngsgd, N, D, pad, types):
    """Leading dimensions of every alignment, another one for each matrix; what lies between the rows stays as it was."""
    import torch
    dtype, wtype = (getattr(torch, t) for t in types)
    x, dy, w, b = inputs(torch, N, D, dtype, wtype, pad)
    both(torch, ngsgd, x, dy, w, b)
    ln = ngsgd.LayerNorm(N, D)
    wide_y = torch.full((N, D + 2 * pad), 5.0, dtype=dtype, device="cuda")
    wide_dx = torch.full((N, D + 3 * pad), 6.0, dtype=dtype, device="cuda")
    y, mean, rstd = ln.forward(x, w, b, out=wide_y[:, :D])
    check_forward(torch, x, w, b, 1e-5, y, mean, rstd)
    check_backward(torch, dy, x, mean, rstd, w, *ln.backward(dy, x, mean, rstd, w, dx=wide_dx[:, :D]))
    assert bool((wide_y[:, D:] == 5.0).all()) and bool((wide_dx[:, D:] == 6.0).all())
    assert bool((x.untyped_storage().nbytes() == N * (D + pad) * x.element_size()))
    for t in (x, dy):
        base = torch.as_strided(t, (N, D + pad), (D + pad, 1))
        assert bool((base[:, D:] == 77.0).all())


@pytest.mark.parametrize("D", [5, 256, 1000, 3000, 20000])
def test_shifted_starts(ngsgd, D):
    """Matrices and vectors that start one element behind an aligned address."""
    import torch
    N, dtype = 6, torch.bfloat16
    x, dy, w, b = inputs(torch, N, D, dtype, dtype)

    def shifted(t):
        flat = torch.zeros(t.numel() + 1, dtype=t.dtype, device="cuda")
        flat[1:] = t.reshape(-1)
        return flat[1:].view(t.shape)

    both(torch, ngsgd, shifted(x), shifted(dy), shifted(w), shifted(b))


@pytest.mark.parametrize("D", [3, 128, 700, 2048, 9000, 17000])
def test_without_weight_or_bias(ngsgd, D):
    import torch
    x, dy, w, b = inputs(torch, 11, D, torch.float32, torch.float32)
    ln = ngsgd.LayerNorm(11, D, 1e-3)
    for ww, bb in ((None, None), (w, None), (None, b)):
        y, mean, rstd = ln.forward(x, ww, bb)
        check_forward(torch, x, ww, bb, 1e-3, y, mean, rstd)
    check_backward(torch, dy, x, mean, rstd, None, *ln.backward(dy, x, mean, rstd))
    full = ln.backward(dy, x, mean, rstd, w)
    for needs in ((True, False, False), (False, True, False), (False, False, True), (False, True, True), (True, False, True)):
        part = ln.backward(dy, x, mean, rstd, w, needs=needs)
        for need, p, f in zip(needs, part, full):
            assert (p is None) if not need else torch.equal(p, f)


@pytest.mark.parametrize("D", [1, 8, 300, 1024, 4097, 30000])
def test_in_place(ngsgd, D):
    import torch
    x, dy, w, b = inputs(torch, 13, D, torch.float32, torch.float32)
    ln, (y, mean, rstd), (dx, dw, db) = both(torch, ngsgd, x, dy, w, b)
    d = dy.clone()
    dx2, dw2, db2 = ln.backward(d, x, mean, rstd, w, dx=d)
    assert dx2 is d and torch.equal(d, dx) and torch.equal(dw2, dw) and torch.equal(db2, db)
    x2 = x.clone()
    y2, _, _ = ln.forward(x2, w, b, out=x2)
    assert y2 is x2 and torch.equal(x2, y)


def test_a_mean_far_from_zero(ngsgd):
    """The variance comes from differences to the mean: a mean of 1000 standard deviations costs no more than its own rounding."""
    import torch
    for D in (64, 1000, 8192, 20000):
        x, dy, w, b = inputs(torch, 4, D, torch.float32, torch.float32, offset=3000.0)
        both(torch, ngsgd, x, dy, w, b)


@pytest.mark.parametrize("D", [1, 6, 512, 2050, 20000])
def test_constant_rows_and_epsilon(ngsgd, D):
    import torch
    x = torch.full((3, D), 2.5, device="cuda")
    w, b = torch.full((D,), 3.0, device="cuda"), torch.full((D,), -1.0, device="cuda")
    y, mean, rstd = ngsgd.LayerNorm(3, D, 0.25).forward(x, w, b)
    assert torch.equal(y, b.expand(3, D)) and torch.equal(mean, x[:, 0]) and bool((rstd == 2.0).all())
    y, mean, rstd = ngsgd.LayerNorm(3, D, 0.0).forward(x, w, b)
    assert bool(y.isnan().all()) and bool(rstd.isinf().all())


@pytest.mark.parametrize("D", [40, 1024, 3000, 20000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_bad_numbers_stay_in_their_row(ngsgd, D, bad):
    import torch
    x, dy, w, b = inputs(torch, 9, D, torch.bfloat16, torch.float32)
    ln, (y, mean, rstd), (dx, dw, db) = both(torch, ngsgd, x, dy, w, b)
    x2 = x.clone()
    x2[4, D - 1] = bad
    y2, m2, r2 = ln.forward(x2, w, b)
    rows = [0, 1, 2, 3, 5, 6, 7, 8]
    assert bool(y2[4].isnan().all()) and torch.equal(y2[rows], y[rows]) and torch.equal(m2[rows], mean[rows]) and torch.equal(r2[rows], rstd[rows])
    d2 = dy.clone()
    d2[4, 0] = bad
    dx2, dw2, db2 = ln.backward(d2, x, mean, rstd, w)
    assert not bool(dx2[4].isfinite().any()) and torch.equal(dx2[rows], dx[rows])
    assert not bool(dw2[0].isfinite()) and not bool(db2[0].isfinite()) and torch.equal(dw2[1:], dw[1:]) and torch.equal(db2[1:], db[1:])


def test_no_rows(ngsgd):
    import torch
    ln = ngsgd.LayerNorm(4, 100)
    x = torch.zeros(0, 100, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(100, dtype=torch.bfloat16, device="cuda")
    y, mean, rstd = ln.forward(x, w, w)
    assert y.shape == (0, 100) and mean.shape == (0,)
    ln.workspace.fill_(255)          # NaN, were it read
    dx, dw, db = ln.backward(x, x, mean, rstd, w)
    assert dx.shape == (0, 100) and bool((dw == 0).all()) and bool((db == 0).all())


def test_fewer_rows_than_the_workspace_is_for(ngsgd):
    import torch
    ln = ngsgd.LayerNorm(500, 260)
    for N in (500, 3, 77, 499):
        x, dy, w, b = inputs(torch, N, 260, torch.float32, torch.float32)
        y, mean, rstd = ln.forward(x, w, b)
        check_forward(torch, x, w, b, 1e-5, y, mean, rstd)
        check_backward(torch, dy, x, mean, rstd, w, *ln.backward(dy, x, mean, rstd, w))


def test_more_than_two_dimensions(ngsgd):
    import torch
    x, dy, w, b = inputs(torch, 24, 96, torch.float16, torch.float32)
    ln = ngsgd.LayerNorm(24, 96)
    y, mean, rstd = ln.forward(x, w, b)
    y3, mean3, rstd3 = ln.forward(x.view(2, 3, 4, 96), w, b)
    assert y3.shape == (2, 3, 4, 96) and torch.equal(y3.view(24, 96), y) and torch.equal(mean3, mean)
    dx, dw, db = ln.backward(dy, x, mean, rstd, w)
    dx3, dw3, db3 = ln.backward(dy.view(2, 3, 4, 96), x.view(2, 3, 4, 96), mean, rstd, w)
    assert torch.equal(dx3.view(24, 96), dx) and torch.equal(dw3, dw) and torch.equal(db3, db)
    y1, _, _ = ln.forward(x[0], w, b)
    assert y1.shape == (96,) and torch.equal(y1, y[0])


def test_repeated_calls_give_the_same_bits(ngsgd):
    import torch
    for N, D in ((1000, 70), (700, 1500), (300, 9000)):
        x, dy, w, b = inputs(torch, N, D, torch.bfloat16, torch.float32)
        ln, first, grads = both(torch, ngsgd, x, dy, w, b)
        for _ in range(3):
            ln.workspace.fill_(255)
            assert all(torch.equal(p, q) for p, q in zip(ln.forward(x, w, b), first))
            assert all(torch.equal(p, q) for p, q in zip(ln.backward(dy, x, first[1], first[2], w), grads))


def test_gradients_are_differences(ngsgd):
    """sum(dy y) moved by a small step in each input, in fp32 through the kernels: against the kernels' own gradients.  The difference quotient
    over 2h is off by the rounding of y, which its sum in 64 bits sees as (K + 40) u |dy| (|y| + 1) / h at most, and by the third
    derivative, of order h^2 rstd^3."""
    import torch
    N, D, h = 3, 12, 2.0 ** -7
    x, dy, w, b = inputs(torch, N, D, torch.float32, torch.float32)
    x = x.clone()
    ln, (y, mean, rstd), (dx, dw, db) = both(torch, ngsgd, x, dy, w, b, 0.1)

    def f(x, w, b):
        return float((ln.forward(x, w, b)[0].double() * dy.double()).sum())

    r = float(rstd.max())
    rounding = 64 * U * float((dy.abs() * (y.abs() + 1)).sum()) / h * max(1.0, 1.0 + float(mean.abs().max()) * r)
    curved = 30 * h * h * max(1.0, r ** 3) * float(dy.abs().sum()) * float(w.abs().max())
    for at, grad in ((0, dx), (1, dw), (2, db)):
        for i in np.ndindex(tuple(grad.shape)):
            up, down = [t.clone() for t in (x, w, b)], [t.clone() for t in (x, w, b)]
            up[at][i] += h
            down[at][i] -= h
            width = float(up[at][i].double() - down[at][i].double())
            assert abs((f(*up) - f(*down)) / width - float(grad[i])) <= rounding + curved


def test_on_another_stream(ngsgd):
    import torch
    x, dy, w, b = inputs(torch, 200, 600, torch.bfloat16, torch.float32)
    ln, want, grads = both(torch, ngsgd, x, dy, w, b)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = ln.forward(x, w, b, stream=s)
    got_grads = ln.backward(dy, x, got[1], got[2], w, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(p, q) for p, q in zip(got + got_grads, want + grads))


def test_captured_calls(ngsgd):
    """Two graphs that share an object's workspace, replayed in turn with new inputs and eager calls between the replays."""
    import torch
    sizes = [(300, 700), (40, 2600)]
    made = []
    for N, D in sizes:
        x, dy, w, b = inputs(torch, N, D, torch.float32, torch.float32)
        made.append([ngsgd.LayerNorm(N, D), x.clone(), dy.clone(), w, b])
    shared = max((m[0].workspace for m in made), key=lambda t: t.numel())
    for m in made:
        m[0].workspace, m[0].workspace_bytes = shared, shared.numel()
    graphs = []
    for ln, x, dy, w, b in made:
        ln.forward(x, w, b)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            y, mean, rstd = ln.forward(x, w, b)
            out = (y, mean, rstd) + ln.backward(dy, x, mean, rstd, w)
        graphs.append((g, out))
    for k in range(4):
        for (ln, x, dy, w, b), (g, out) in zip(made, graphs):
            new_x, new_dy, _, _ = inputs(torch, *x.shape, torch.float32, torch.float32, seed=10 + k)
            x.copy_(new_x)
            dy.copy_(new_dy)
            g.replay()
            got = [t.clone() for t in out]
            eager = ln.forward(x, w, b)
            want = eager + ln.backward(dy, x, eager[1], eager[2], w)
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("D", [100, 3000, 20000])
def test_offsets_beyond_32_bits(ngsgd, D):
    """Rows more than 2^30 elements apart: the third one starts behind 2^31."""
    import torch
    N, apart = 3, 2 ** 30 + 40
    x, dy, w, b = inputs(torch, N, D, torch.bfloat16, torch.float32)
    ln, (y, mean, rstd), (dx, dw, db) = both(torch, ngsgd, x, dy, w, b)

    def far(t=None):
        rows = torch.empty(N * apart, dtype=torch.bfloat16, device="cuda").as_strided((N, D), (apart, 1))
        return rows if t is None else rows.copy_(t)

    fx, fdy, fy = far(x), far(dy), far()
    y2, mean2, rstd2 = ln.forward(fx, w, b, out=fy)
    dx2, dw2, db2 = ln.backward(fdy, fx, mean, rstd, w, dx=fy)
    assert torch.equal(mean2, mean) and torch.equal(rstd2, rstd) and torch.equal(dw2, dw) and torch.equal(db2, db)
    assert torch.equal(dx2, dx)
    ln.forward(fx, w, b, out=fy)
    assert torch.equal(fy, y)
    torch.cuda.empty_cache()


def test_rows_that_are_not_given_stay(ngsgd):
    import torch
    for D in (64, 1000, 3000, 20000):
        x, dy, w, b = inputs(torch, 9, D, torch.float32, torch.float32)
        y, dx = (torch.full((9, D), 4.0, device="cuda") for _ in range(2))
        mean, rstd = (torch.full((9,), 5.0, device="cuda") for _ in range(2))
        ln = ngsgd.LayerNorm(9, D)
        ln.forward(x[:7], w, b, out=y[:7], mean=mean[:7], rstd=rstd[:7])
        ln.backward(dy[:7], x[:7], mean[:7], rstd[:7], w, dx=dx[:7])
        assert bool((y[7:] == 4.0).all()) and bool((dx[7:] == 4.0).all()) and bool((mean[7:] == 5.0).all()) and bool((rstd[7:] == 5.0).all())
        assert bool((y[:7] != 4.0).any(dim=1).all()) and bool((dx[:7] != 4.0).any(dim=1).all())


def test_refusals(ngsgd):
    import torch
    ln = ngsgd.LayerNorm(8, 64)
    x = torch.zeros(8, 64, device="cuda")
    v = torch.ones(64, device="cuda")
    mean = torch.zeros(8, device="cuda")
    for bad in (lambda: ln.forward(torch.zeros(9, 64, device="cuda")), lambda: ln.forward(torch.zeros(8, 63, device="cuda")),
                lambda: ln.forward(x.double()), lambda: ln.forward(x.t().contiguous().t()), lambda: ln.forward(x, v.bfloat16()),
                lambda: ln.forward(x.bfloat16(), v.half()), lambda: ln.forward(x, v, v.bfloat16()), lambda: ln.forward(x, v[:63]),
                lambda: ln.forward(x, v, out=x[:7]), lambda: ln.forward(x, v, out=x.half()), lambda: ln.forward(x, v, mean=mean[:7]),
                lambda: ln.forward(x, v, rstd=mean.double()), lambda: ln.forward(x, v.cpu()), lambda: ln.forward(x.cpu()),
                lambda: ln.backward(x[:7], x, mean, mean), lambda: ln.backward(x, x, mean[:7], mean), lambda: ln.backward(x, x, mean, mean, v, dbias=v.half()),
                lambda: ln.backward(x.half(), x, mean, mean)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(ngsgd.NgsgdError):
        ln.forward(torch.zeros(1, 64, device="cuda").expand(8, 64))      # rows that overlap
    with pytest.raises(ngsgd.NgsgdError):
        ln.backward(x, x, mean, mean, v, needs=(False, False, False))


def check_large(torch, x, dy, w, b, out, grads, eps=1e-5):
    """Some 90 rows (fewer of very wide ones) and the last ones; all of the sums over the rows, in 64 bits on the GPU."""
    N, D = x.shape
    count = min(90, max(3, (1 << 22) // D))
    rows = sorted(set(range(0, N, -(-N // count))) | set(range(max(0, N - count // 3), N)))
    check_forward(torch, x[rows], w, b, eps, *(t[rows] for t in out))
    _, mean, rstd = out
    check_backward(torch, dy[rows], x[rows], mean[rows], rstd[rows], w, grads[0][rows], None, None)
    terms = x.double()
    terms -= mean.double()[:, None]
    terms *= rstd.double()[:, None]
    for got in (grads[1], grads[2]):
        d = dy.double()
        if got is grads[1]:
            d *= terms
        want = d.sum(dim=0)
        u = half_step(torch, got.dtype)
        e = (N + 12) * U * d.abs_().sum(dim=0)
        assert bool(((got.double() - want).abs() <= e * (1 + 2 * u) + u * want.abs() + tiny(torch, got.dtype)).all())


@pytest.mark.parametrize("N,D", [(24584, 7), (24583, 24), (49159, 100), (12293, 200), (24577, 133), (6149, 300), (12297, 512), (6151, 600), (18439, 1001),
                                 (8198, 100), (16411, 65), (4099, 250), (8195, 129), (4101, 1500), (8200, 2049), (2051, 16390), (4100, 16385),
                                 (3400, 20000), (65, 1100003)])
@pytest.mark.parametrize("types", [COMBOS[0], COMBOS[2]], ids="-".join)
def test_more_rows_than_a_grid(ngsgd, N, D, types):
    """A second and third round of rows, the last one not full, of every shape, forward (1536 wavefronts' grids) and backward (640); rows from memory in
    more than 2048 workgroups, and as many groups of their sums as the workspace's bound leaves (3400 x 20000, 65 x 1100003)."""
    import torch
    dtype, wtype = (getattr(torch, t) for t in types)
    g = torch.Generator(device="cuda")
    g.manual_seed(N + D)
    x = torch.randn(N, D, generator=g, device="cuda")
    x *= torch.rand(N, 1, generator=g, device="cuda") * 2.0 + 0.25
    x += torch.randn(N, 1, generator=g, device="cuda")
    x = x.to(dtype)
    dy = torch.randn(N, D, generator=g, device="cuda").to(dtype)
    w = (1.0 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(wtype)
    b = (0.3 * torch.randn(D, generator=g, device="cuda")).to(wtype)
    ln = ngsgd.LayerNorm(N, D)
    out = ln.forward(x, w, b)
    grads = ln.backward(dy, x, out[1], out[2], w)
    check_large(torch, x, dy, w, b, out, grads)
    # in place, and with nothing but the sums, the same bits
    d, y = dy.clone(), x.clone()
    assert torch.equal(ln.forward(y, w, b, out=y)[0], out[0])
    assert torch.equal(ln.backward(d, x, out[1], out[2], w, dx=d)[0], grads[0])
    assert all(torch.equal(p, q) for p, q in zip(ln.backward(dy, x, out[1], out[2], w, needs=(False, True, True))[1:], grads[1:]))


def test_each_gradient_is_its_difference(ngsgd):
    """As above with bounds near the kernels' own, entry by entry.  f = sum(dy y) is summed in 64 bits and only what moves is counted: a row
    for an element of x, a column for one of w or b.
    Rounding: 2 e / 2h with the error e of y as at the top; w and b leave xhat as it is, and y is off by u of |xhat w| and u of |y|.
    Curvature: h^2 / 6 times the third derivative, which is 0 in w and b.  For x, |xhat| <= sqrt(D) gives |r'| <= r^2 D^(-1/2), |r''| <= 4 r^3 / D and
    |r'''| <= 24 r^4 D^(-3/2), and so |xhat'''| <= 3 |r''| + |xhat r''' / r| <= 36 r^3 / D."""
    import torch
    N, D, h = 4, 12, 2.0 ** -8
    rng = np.random.default_rng(77)
    # rows of deviation near 1 and a mean below 1
    x = torch.from_numpy(rng.standard_normal((N, D)) + rng.uniform(-1, 1, (N, 1))).float().cuda()
    _, dy, w, b = inputs(torch, N, D, torch.float32, torch.float32)
    ln, (y, mean, rstd), grads = both(torch, ngsgd, x, dy, w, b, 0.1)
    Y, DY, W, X, r = np.abs(f64(y)), np.abs(f64(dy)), np.abs(f64(w)), f64(x), f64(rstd)
    xhat = np.abs((X - f64(mean)[:, None]) * r[:, None])
    K = D / 64 + 24
    e_y = U * (W * (K * r * np.abs(X).mean(axis=1))[:, None] + W * xhat * (K + 12) + 4 * Y)
    row = (DY * e_y).sum(axis=1) / h + h * h * 6 / D * r ** 3 * (DY * W).sum(axis=1)
    column = (DY * 2 * U * (W * xhat + Y + h * (xhat + 1))).sum(axis=0) / h
    bounds = np.repeat(row[:, None], D, axis=1), column, column
    for at, (grad, bound) in enumerate(zip(grads, bounds)):
        grad = f64(grad)
        assert np.median(bound / np.abs(grad)) < 0.05       # (zeros, or another entry's, would not pass)
        for i in np.ndindex(grad.shape):
            moved = [[t.clone() for t in (x, w, b)] for _ in range(2)]
            moved[0][at][i] += h
            moved[1][at][i] -= h
            up, down = (f64(ln.forward(*m)[0]) for m in moved)
            width = float(moved[0][at][i].double() - moved[1][at][i].double())
            # the gradients' own bounds, of some 40 u, are far below these
            assert abs((f64(dy) * (up - down)).sum() / width - grad[i]) <= bound[i]


@pytest.mark.parametrize("D", [3, 6, 24, 200, 300, 1000, 1500, 4099, 9000, 16384, 20001])
def test_rows_far_from_zero(ngsgd, D):
    """Equal numbers give the bias, and rows of a deviation of 1e-2 around 3000 lose no more of their digits than rows around 0.

    The first mean is off by delta, K u mean|x| at most.  The differences to it (u of each) are summed, which gives delta to (K + 2) u of their mean
    magnitude, and it is taken off them (u of each).  The variance is the mean of their squares less delta^2: off by (2 K + 6) u of
    variance + 2 delta^2.  The rest as at the top."""
    import torch
    N, K, eps = 5, D / 64 + 24, 1e-5
    rng = np.random.default_rng(D)
    x = torch.from_numpy(3000.0 + 1e-2 * rng.standard_normal((N, D)) + rng.standard_normal((N, 1))).float().cuda()
    x[3] = 3000.1
    x[4] = -0.7
    _, _, w, b = inputs(torch, N, D, torch.float32, torch.float32)
    y, mean, rstd = ngsgd.LayerNorm(N, D, eps).forward(x, w, b)
    X, W = f64(x), np.abs(f64(w))
    want, m, r = oracle.forward(X, f64(w), f64(b), eps)
    d, m, r = np.abs(X - m[:, None]), m[:, None], r[:, None]
    var, delta = (d * d).mean(axis=1, keepdims=True), K * U * np.abs(X).mean(axis=1, keepdims=True)
    e_d = U * (d + delta) + (K + 2) * U * (d.mean(axis=1, keepdims=True) + delta) + U * d
    e_r = (2 * K + 6) * U * (var + 2 * delta ** 2) / (2 * (var + eps)) + 4 * U
    assert np.all(np.abs(f64(rstd)[:, None] - r) <= e_r * r)
    assert np.all(np.abs(f64(mean)[:, None] - m) <= U * np.abs(m) + (K + 2) * U * (d.mean(axis=1, keepdims=True) + delta))
    assert np.all(np.abs(f64(y) - want) <= W * (r * e_d + d * r * (e_r + 4 * U)) + 3 * U * np.abs(want))


@pytest.mark.parametrize("D", [5, 200, 1000, 3000, 20000])
def test_statistics_of_infinite_rows(ngsgd, D):
    """The mean of a row with one infinity is that; of one with both it is NaN, as with a NaN.  A variance above what fp32 holds: rstd 0, y the bias."""
    import torch
    x = torch.randn(5, D, device="cuda")
    x[0, 1], x[1, D - 1], x[3, 2] = float("inf"), float("-inf"), float("nan")
    x[2, 0], x[2, D - 1] = float("inf"), float("-inf")
    x[4, 0], x[4, D - 1] = 1e30, -1e30
    w, b = torch.full((D,), 2.0, device="cuda"), torch.randn(D, device="cuda")
    y, mean, rstd = ngsgd.LayerNorm(5, D).forward(x, w, b)
    assert mean[:2].tolist() == [float("inf"), float("-inf")] and bool(mean[2:4].isnan().all()) and bool(mean[4].isfinite())
    assert bool(y[:4].isnan().all()) and bool(rstd[:4].isnan().all())
    assert float(rstd[4]) == 0.0 and torch.equal(y[4], b)


@pytest.mark.parametrize("N,D", [(100, 5), (24600, 20), (50, 200), (6200, 600), (3000, 1500), (2100, 5000), (2100, 16400)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows_far_from_zero_among_others(ngsgd, N, D, dtype):
    """A row's numbers are its own: the same bits whether the rows beside it are far from zero or near, or there are none."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(N + D)
    x = torch.randn(N, D, generator=g, device="cuda")
    far = torch.rand(N, generator=g, device="cuda") < 0.3
    x[far] += 64.0 * (1 + torch.arange(int(far.sum()), device="cuda") % 7)[:, None]
    x[far.nonzero()[::5, 0]] = 100.5
    x = x.to(getattr(torch, dtype))
    b = torch.randn(D, generator=g, device="cuda").to(x.dtype)
    ln = ngsgd.LayerNorm(N, D)
    out = ln.forward(x, None, b)
    for part in (far, ~far):
        assert all(torch.equal(whole[part], alone) for whole, alone in zip(out, ln.forward(x[part], None, b)))
    # equal numbers: what the first mean is off by, K u 100.5 at most, is taken off up to K + 3 u of itself
    equal, K, B = far.nonzero()[::5, 0], D / 64 + 24, b.double()
    bound = out[2][equal].double()[:, None] * (K * U * 100.5) * (K + 3) * U + (half_step(torch, x.dtype) + U) * B.abs()
    assert bool(((out[0][equal].double() - B).abs() <= bound).all())
    check_forward(torch, x[:64], None, b, 1e-5, *(t[:64] for t in out))
