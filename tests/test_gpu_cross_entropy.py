"""GPU parity: the cross-entropy and its gradient through the C ABI against the float64 definition.

Tolerances.  u = 2^-24 is half a step of fp32, u_t of the output's type.  v = x - m is off by u |v|, and so is exp(v), relative to itself, with 6 u more of the
function's own; a sum of positive terms adds K u, K(V) = V / 64 + 24 additions in a chain at most.  So S and S + e are off by
  E = sum e_j (|v_j| + 6) u / sum e_j + K u
relative to themselves.  The loss: log's argument E, 4 u of the logarithm, u of x_y - m and of their sum; where the label is the largest,
E + 4 u of log1p(S).  The gradient: (|v_j| + 6) u of e_j, E of the quotient, 4 u of its products, then u_t.  A result below 2^-126 may be zero.
"""
import numpy as np
import pytest

from oracle.cross_entropy import cross_entropy as oracle

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = ["float32", "bfloat16", "float16"]
INDEX = ["int32", "int64"]


def f64(t):
    return t.detach().double().cpu().numpy()


def matrix(torch, a, dtype, pad=0, shift=0):
    """Rows inside a wider buffer of 77s that starts `shift` elements behind an aligned address."""
    n, d = a.shape
    flat = torch.full((n * (d + pad) + shift,), 77.0, dtype=dtype, device="cuda")
    wide = flat[shift:].view(n, d + pad)
    wide[:, :d] = torch.from_numpy(a).to(dtype).cuda()
    return wide[:, :d]


def between_rows(m, pad):
    n, d = m.shape
    return m.as_strided((n, d + pad), (d + pad, 1), m.storage_offset())[:, d:]


def make_labels(torch, rng, N, V, index, ignored=0.15):
    y = rng.integers(0, V, N)
    outside = [-1, V, -100, -2 ** 31, 2 ** 31 - 1] + ([2 ** 32, -2 ** 63, 2 ** 63 - 1] if index == "int64" else [])
    where = rng.random(N) < ignored
    y[where] = rng.choice(outside, where.sum())
    return torch.from_numpy(y).to(getattr(torch, index)).cuda(), y


def logits_of(rng, N, V, y, sure=8.0):
    x = 2.0 * rng.standard_normal((N, V))
    there = (y >= 0) & (y < V)
    x[np.arange(N)[there], y[there]] += sure * rng.random(there.sum())
    return x


def check(torch, x, y, scale, loss, d=None):
    X = f64(x)
    N, V = X.shape
    K = V / 64 + 24
    scale = float(np.float32(scale))
    want, grad = oracle(X, y, scale)
    there = (y >= 0) & (y < V)
    at = np.where(there, y, 0)
    with np.errstate(invalid="ignore"):
        v = np.abs(X - X.max(axis=1, keepdims=True))
        e = np.exp(-v)
        weight = np.where(e > 0, e * (np.where(np.isfinite(v), v, 0) + 6), 0)
        E = U * (weight.sum(axis=1) / e.sum(axis=1) + K)
        own = np.take_along_axis(v, at[:, None], 1)[:, 0]
        others = e.copy()
        np.put_along_axis(others, at[:, None], 0.0, 1)
        others_E = U * (np.where(others > 0, weight, 0).sum(axis=1) / np.maximum(others.sum(axis=1), 1e-300) + K)
        log_term = np.log(e.sum(axis=1))
        bound = np.where(own == 0, (others_E + 4 * U) * np.abs(want), E + 4 * U * np.abs(log_term) + 2 * U * (own + np.abs(want))) + 2.0 ** -125
    got = f64(loss).reshape(-1)
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine], equal_nan=True)
    off, most = np.abs(got[fine] - want[fine]), bound[fine]
    assert np.all(off <= most), float(np.max(off / most))
    assert np.all(got[~there] == 0)
    if d is None:
        return
    h = torch.finfo(d.dtype).eps / 2 if d.dtype != torch.float32 else 0.0
    tiny = torch.finfo(d.dtype).smallest_normal * torch.finfo(d.dtype).eps / 2
    with np.errstate(invalid="ignore"):
        rel = (np.where(np.isfinite(v), v, 0) + 10) * U + E[:, None]
        np.put_along_axis(rel, at[:, None], (others_E + E + 4 * U)[:, None], 1)
    G = f64(d)
    fine = np.isfinite(grad)
    assert np.array_equal(np.isnan(G), np.isnan(grad)) and np.array_equal(G[~fine], grad[~fine], equal_nan=True)
    off, most = np.abs(G[fine] - grad[fine]), ((rel * (1 + h) + h) * np.abs(grad) + tiny + (1 + abs(scale)) * 2.0 ** -125)[fine]
    assert np.all(off <= most), float(np.max(off / most))
    assert np.all(G[~there] == 0)


WIDTHS = [1, 2, 3, 4, 7, 8, 9, 31, 50, 63, 64, 65, 127, 128, 255, 256, 257, 511, 512, 513, 1000, 1024, 1025, 2047, 2048, 2049, 4095, 4096, 4097, 5000, 8191,
          8192, 8193, 16384, 16385, 20011, 32768, 32769, 65536, 65537, 100003, 131072, 131073]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", WIDTHS)
def test_widths(ngsgd, V, dtype):
    """Every number of classes at its borders, few rows and many, aligned or not, in place and not."""
    import torch
    dtype = getattr(torch, dtype)
    for N, pad, shift in ((5, 0, 0), (3, 3, 1), (1, 8, 8), (400 if V <= 1100 else 67 if V <= 9000 else 9, 1, 0)):
        rng = np.random.default_rng(V + N)
        labels, y = make_labels(torch, rng, N, V, INDEX[V % 2])
        x = matrix(torch, logits_of(rng, N, V, y), dtype, pad, shift)
        ce = ngsgd.CrossEntropy(N, V)
        d = matrix(torch, np.zeros((N, V)), dtype, pad, shift)
        loss, _ = ce.gradient(x, labels, scale=0.7, dlogits=d)
        check(torch, x, y, 0.7, loss, d)
        alone = ce.forward(x, labels)
        check(torch, x, y, 1.0, alone)
        assert torch.equal(alone, loss)
        again, dense = ce.gradient(x, labels, scale=0.7)
        assert dense.is_contiguous() and torch.equal(dense, d) and torch.equal(again, loss)
        ce.gradient(x, labels, scale=0.7, dlogits=x)
        assert torch.equal(x, d)
        if pad:
            assert bool((between_rows(d, pad) == 77).all()) and bool((between_rows(x, pad) == 77).all())


@pytest.mark.parametrize("N", [1, 2, 4, 15, 16, 17, 63, 64, 100, 255, 256, 257, 300, 511, 512, 513, 1030])
@pytest.mark.parametrize("V", [50, 3001, 40001])
def test_rows(ngsgd, N, V):
    import torch
    dtype = torch.bfloat16 if V > 3001 else torch.float32
    rng = np.random.default_rng(N)
    labels, y = make_labels(torch, rng, N, V, INDEX[N % 2])
    x = matrix(torch, logits_of(rng, N, V, y), dtype)
    loss, d = ngsgd.CrossEntropy(N, V).gradient(x, labels, scale=2.0)
    check(torch, x, y, 2.0, loss, d)


@pytest.mark.parametrize("V,dtype", [(32769, "float16"), (65536, "bfloat16"), (65537, "float16"), (100003, "bfloat16"), (131072, "bfloat16"), (131073, "float16"),
                                     (150001, "bfloat16"), (32769, "float32"), (65536, "float32"), (65537, "float32"), (90001, "float32")])
def test_wide_rows_of_a_workgroup(ngsgd, V, dtype):
    """As many rows as are not cut into parts: held in registers, and wider than those.  Among them rows that are decided, masked, empty or not numbers."""
    import torch
    dtype = getattr(torch, dtype)
    rng = np.random.default_rng(V)
    N, low = 130, float(torch.finfo(dtype).min)
    labels, y = make_labels(torch, rng, N, V, "int64")
    y[:10] = rng.integers(0, V, 10)
    y[3], y[4] = V - 1, 0
    labels[:10] = torch.from_numpy(y[:10])
    x = logits_of(rng, N, V, y)
    x[0, y[0]] = 50.0
    x[1] = -np.inf
    x[2, ::2] = -np.inf
    x[2, y[2]] = 1.0
    x[3, V // 2], x[4, V - 1] = np.nan, np.inf
    x[5] = low
    x[6, np.arange(V) != y[6]] = low
    x[7, y[7]] = -np.inf
    pad = V % 2 + 1
    x = matrix(torch, x, dtype, pad, 1)
    ce = ngsgd.CrossEntropy(N, V)
    loss, d = ce.gradient(x, labels, scale=1.5)
    check(torch, x, y, 1.5, loss, d)
    assert bool(loss[[1, 3, 4]].isnan().all()) and float(loss[5]) == pytest.approx(np.log(V), rel=1e-6) and float(loss[0]) > 0
    assert torch.equal(torch.nan_to_num(ce.forward(x, labels), nan=-5.0), torch.nan_to_num(loss, nan=-5.0))
    kept = x.clone()
    again, _ = ce.gradient(x, labels, scale=1.5, dlogits=x)
    assert torch.equal(x.nan_to_num(), d.nan_to_num()) and torch.equal(again.nan_to_num(), loss.nan_to_num())
    assert bool((between_rows(x, pad) == 77).all())
    few = ngsgd.CrossEntropy(20, V).gradient(kept[:20], labels[:20], scale=1.5)          # the same rows in parts
    check(torch, kept[:20], y[:20], 1.5, *few)


def test_very_wide_rows(ngsgd):
    import torch
    rng = np.random.default_rng(4)
    for N, V in ((1, 3_000_001), (2, 2_500_000)):
        labels, y = make_labels(torch, rng, N, V, "int64", ignored=0.0)
        x = matrix(torch, logits_of(rng, N, V, y), torch.bfloat16)
        loss, d = ngsgd.CrossEntropy(N, V).gradient(x, labels)
        check(torch, x, y, 1.0, loss, d)


def test_many_rows(ngsgd):
    import torch
    rng = np.random.default_rng(1)
    for N, V in ((200003, 11), (2 ** 21 + 100, 3)):      # the second one: more than a launch takes
        labels, y = make_labels(torch, rng, N, V, "int32")
        x = matrix(torch, logits_of(rng, N, V, y), torch.float32)
        loss, d = ngsgd.CrossEntropy(N, V).gradient(x, labels)
        check(torch, x, y, 1.0, loss, d)


@pytest.mark.parametrize("V", [9, 300, 5000, 40000, 140000])
def test_decided_rows_keep_their_digits(ngsgd, V):
    """A label far above the rest: the loss and the label's gradient are as small as what the others leave, to fp32's relative precision (check's bound is
    relative there)."""
    import torch
    rng = np.random.default_rng(2)
    N = 12
    y = rng.integers(0, V, N)
    x = rng.standard_normal((N, V))
    x[np.arange(N), y] = 6.0 + 5.0 * np.arange(N)
    x = matrix(torch, x, torch.float32)
    loss, d = ngsgd.CrossEntropy(N, V).gradient(x, torch.from_numpy(y).cuda())
    check(torch, x, y, 1.0, loss, d)
    assert float(loss.min()) > 0 and float(loss.min()) < 1e-20


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [6, 300, 5001, 33000, 140001])
def test_large_equal_and_masked_logits(ngsgd, V, dtype):
    import torch
    torch_type = getattr(torch, dtype)
    rng = np.random.default_rng(3)
    low = float(torch.finfo(torch_type).min)
    x = 2.0 * rng.standard_normal((9, V))
    y = rng.integers(0, V, 9)
    x[0] += 3e4                                        # far from zero
    x[1] -= 3e4
    x[2] = 1.5                                         # all equal
    x[3, np.arange(V) != y[3]] = -np.inf               # the label alone is there
    x[4, ::2] = -np.inf
    x[4, y[4]] = 1.0
    x[5, y[5]] = -np.inf                               # the label is not there
    x[6, 1::2] = low                                   # masked with the type's lowest value
    x[6, y[6]] = 0.0
    x[7] = low                                         # nothing but that
    x[8] = -low                                        # nothing but the type's largest
    x = matrix(torch, x, torch_type)
    loss, d = ngsgd.CrossEntropy(9, V).gradient(x, torch.from_numpy(y).cuda())
    check(torch, x, y, 1.0, loss, d)
    assert float(loss[3]) == 0 and not bool(d[3].any()) and float(loss[5]) == float("inf")
    assert float(loss[7]) == pytest.approx(np.log(V), rel=1e-6) and float(loss[8]) == pytest.approx(np.log(V), rel=1e-6)


@pytest.mark.parametrize("V", [5, 100, 3000, 20000, 70000, 140000])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_bad_rows_are_nan_and_alone(ngsgd, V, bad):
    """A NaN or +infinity anywhere, or -infinity everywhere, makes its own row NaN; a row that does not count is zero whatever it holds."""
    import torch
    rng = np.random.default_rng(5)
    N = 7
    y = rng.integers(0, V, N)
    y[4] = -1
    x = matrix(torch, rng.standard_normal((N, V)), torch.float32)
    ce, labels = ngsgd.CrossEntropy(N, V), torch.from_numpy(y).cuda()
    clean = ce.gradient(x, labels)
    if bad == -float("inf"):
        x[1], x[4] = bad, bad
        hit = [1]
    else:
        x[1, V - 1], x[2, 0], x[3, int(y[3])], x[4] = bad, bad, bad, bad
        x[5, V // 2] = bad
        hit = [1, 2, 3, 5]
    loss, d = ce.gradient(x, labels)
    assert bool(loss[hit].isnan().all()) and bool(d[hit].isnan().all())
    rest = [i for i in range(N) if i not in hit]
    assert torch.equal(loss[rest], clean[0][rest]) and torch.equal(d[rest], clean[1][rest])
    assert torch.equal(torch.nan_to_num(ce.forward(x, labels), nan=-5.0), torch.nan_to_num(loss, nan=-5.0))


def test_scales(ngsgd):
    import torch
    rng = np.random.default_rng(6)
    for N, V in ((33, 100), (20, 9000), (3, 150000)):
        labels, y = make_labels(torch, rng, N, V, "int64")
        x = matrix(torch, logits_of(rng, N, V, y), torch.float32)
        ce = ngsgd.CrossEntropy(N, V)
        for scale in (0.0, -2.5, 1.0 / 3.0, 65536.0):
            loss, d = ce.gradient(x, labels, scale=scale)
            check(torch, x, y, scale, loss, d)
            there = torch.tensor([scale], device="cuda")
            other = ce.gradient(x, labels, scale=there)
            assert torch.equal(other[0], loss) and torch.equal(other[1], d)


def test_no_rows_none_that_counts_and_one_class(ngsgd):
    import torch
    ce = ngsgd.CrossEntropy(4, 10)
    loss, d = ce.gradient(torch.zeros(0, 10, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda"))
    assert loss.shape == (0,) and d.shape == (0, 10)
    loss, d = ce.gradient(torch.full((4, 10), float("nan"), device="cuda"), torch.full((4,), -100, device="cuda"))
    assert not bool(loss.any()) and not bool(d.any())
    loss, d = ngsgd.CrossEntropy(3, 1).gradient(torch.tensor([[3.0], [-9e9], [0.0]], device="cuda"), torch.tensor([0, 0, 1], device="cuda"))
    assert not bool(loss.any()) and not bool(d.any())


def test_fewer_rows_than_the_workspace_is_for(ngsgd):
    import torch
    rng = np.random.default_rng(7)
    for V in (60, 50000, 140000):
        ce = ngsgd.CrossEntropy(300, V)
        for N in (300 if V == 60 else 40, 1, 17, 5):
            labels, y = make_labels(torch, rng, N, V, "int32")
            x = matrix(torch, logits_of(rng, N, V, y), torch.bfloat16)
            loss, d = ce.gradient(x, labels)
            check(torch, x, y, 1.0, loss, d)


def test_more_than_two_dimensions(ngsgd):
    import torch
    rng = np.random.default_rng(8)
    labels, y = make_labels(torch, rng, 24, 77, "int64")
    x = matrix(torch, logits_of(rng, 24, 77, y), torch.float16)
    ce = ngsgd.CrossEntropy(24, 77)
    loss, d = ce.gradient(x, labels)
    more = ce.gradient(x.reshape(2, 3, 4, 77), labels.view(2, 3, 4))
    assert more[0].shape == (2, 3, 4) and torch.equal(more[0].view(24), loss) and torch.equal(more[1].view(24, 77), d)
    one = ce.gradient(x[0], labels[0])
    assert one[0].shape == () and torch.equal(one[0], loss[0]) and torch.equal(one[1], d[0])


def test_repeated_calls_give_the_same_bits(ngsgd):
    import torch
    rng = np.random.default_rng(9)
    for N, V in ((5, 130000), (64, 9000), (700, 333)):
        labels, y = make_labels(torch, rng, N, V, "int32")
        x = matrix(torch, logits_of(rng, N, V, y), torch.float32)
        ce = ngsgd.CrossEntropy(N, V)
        first = ce.gradient(x, labels)
        for _ in range(4):
            again = ce.gradient(x, labels)
            assert torch.equal(again[0], first[0]) and torch.equal(again[1], first[1])


@pytest.mark.parametrize("V", [6, 700, 34000])
def test_gradient_is_its_difference(ngsgd, V):
    """Along random directions e of length 1 per row: (L(x + h e) - L(x - h e)) / 2h against <dL, e>.  The losses of a row are off by 40 u of themselves and of
    the logits' spread (below 16 here), over h; the third derivative along e is below 1: h^2 / 6."""
    import torch
    rng = np.random.default_rng(10)
    N, h = 6, 1e-2
    labels, y = make_labels(torch, rng, N, V, "int64", ignored=0.0)
    x = torch.from_numpy(logits_of(rng, N, V, y)).float().cuda()
    ce = ngsgd.CrossEntropy(N, V)
    _, d = ce.gradient(x, labels)
    for k in range(4):
        e = rng.standard_normal((N, V))
        e[np.arange(N), y] += 3.0 * np.sqrt(V)
        e = torch.from_numpy(e / np.linalg.norm(e, axis=1, keepdims=True)).cuda()
        up, down = (x.double() + h * e).float(), (x.double() - h * e).float()
        slope = (ce.forward(up, labels).double() - ce.forward(down, labels).double())
        along = ((up.double() - down.double()) * d.double()).sum(1)
        K = V / 64 + 24
        assert np.all(np.abs(f64(slope - along)) <= 2 * (K + 40) * 16 * U + 2 * h * h * h / 6)


def test_on_another_stream(ngsgd):
    import torch
    rng = np.random.default_rng(11)
    for N, V in ((300, 5000), (6, 150000)):
        labels, y = make_labels(torch, rng, N, V, "int32")
        x = matrix(torch, logits_of(rng, N, V, y), torch.float32)
        ce = ngsgd.CrossEntropy(N, V)
        want = ce.gradient(x, labels)
        both, streams = [ngsgd.CrossEntropy(N, V) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        outs = [[op.gradient(x, labels, stream=q) for op, q in zip(both, streams)] for _ in range(5)]
        torch.cuda.synchronize()
        assert all(torch.equal(o[0], want[0]) and torch.equal(o[1], want[1]) for pair in outs for o in pair)


@pytest.mark.parametrize("N,V", [(40, 100), (300, 5000), (5, 150000), (20, 70000)])
def test_captured_calls(ngsgd, N, V):
    """Replayed with other logits, labels and scales than were captured, with eager work between; two graphs share the workspace."""
    import torch
    rng = np.random.default_rng(12)
    ce = ngsgd.CrossEntropy(N, V)
    x = torch.randn(N, V, device="cuda")
    labels, _ = make_labels(torch, rng, N, V, "int64")
    scale = torch.ones(1, device="cuda")
    ce.gradient(x, labels)
    torch.cuda.synchronize()
    first, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(first):
        loss, d = ce.gradient(x, labels, scale=scale)
    with torch.cuda.graph(second):
        alone = ce.forward(x, labels)
    for k in range(4):
        now, y = make_labels(torch, rng, N, V, "int64")
        labels.copy_(now)
        x.normal_().mul_(1.0 + k)
        scale.fill_(0.5 + k)
        first.replay()
        second.replay()
        torch.cuda.synchronize()
        want = ce.gradient(x, now, scale=0.5 + k)
        assert torch.equal(loss, want[0]) and torch.equal(d, want[1]) and torch.equal(alone, want[0])
        check(torch, x, y, 0.5 + k, loss, d)


def test_an_object_that_is_gone_before_its_work(ngsgd):
    import torch
    rng = np.random.default_rng(13)
    N, V = 6, 150000
    labels, y = make_labels(torch, rng, N, V, "int32")
    x = torch.randn(N, V, device="cuda")
    want = ngsgd.CrossEntropy(N, V).gradient(x, labels)
    s, big = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda")
    for given in (True, False):
        ce = ngsgd.CrossEntropy(N, V)
        size = ce.workspace.numel()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for _ in range(30):
                big = big @ big * 1e-3
            if not given:
                got = ce.gradient(x, labels)
        if given:
            got = ce.gradient(x, labels, stream=s)
        del ce
        taken = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _ in range(3)]
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        del taken


def test_offsets_beyond_32_bits(ngsgd):
    """Logits of more than 2^31 elements, most rows of which do not count; the last rows."""
    import torch
    N, V = 70001, 32768
    x = torch.zeros(N, V, dtype=torch.bfloat16, device="cuda")
    labels = torch.full((N,), -1, dtype=torch.int32, device="cuda")
    labels[N - 1], labels[N - 2], labels[0] = V - 1, 0, 5
    x[N - 1, V - 1], x[N - 2, 1] = 20.0, 30.0
    ce = ngsgd.CrossEntropy(N, V)
    loss, d = ce.gradient(x, labels, dlogits=x)
    assert float(loss[0]) == pytest.approx(np.log(V), rel=1e-6) and float(loss[N - 2]) == pytest.approx(30.0, rel=1e-6)
    assert float(loss[N - 1]) == pytest.approx(np.log1p((V - 1) * np.exp(-20.0)), rel=1e-5) and int((loss != 0).sum()) == 3
    assert float(d[N - 2, 0]) == -1 and float(d[N - 2, 1]) == 1 and float(d[0, 5]) == -1 and not bool(d[1:N - 2].any())


def test_rows_behind_the_last_stay(ngsgd):
    import torch
    for N, V in ((5, 40), (5, 150000)):
        x, d = torch.randn(N, V, device="cuda"), torch.full((N + 3, V), 9.0, device="cuda")
        loss = torch.full((N + 3,), 9.0, device="cuda")
        ngsgd.CrossEntropy(N, V).gradient(x, torch.zeros(N, dtype=torch.int64, device="cuda"), loss=loss[:N], dlogits=d[:N])
        assert bool((loss[N:] == 9).all()) and bool((d[N:] == 9).all())


def test_refusals(ngsgd):
    import torch
    ce = ngsgd.CrossEntropy(8, 10)
    x, labels = torch.zeros(8, 10, device="cuda"), torch.zeros(8, dtype=torch.int64, device="cuda")
    for call in [lambda: ce.forward(x, labels.cpu()), lambda: ce.forward(x, labels.short()), lambda: ce.forward(x, labels.float()), lambda: ce.forward(x[:7], labels),
                 lambda: ce.forward(x[:, :9], labels), lambda: ce.forward(x.double(), labels), lambda: ce.forward(x.cpu(), labels), lambda: ce.forward(x.t().contiguous().t(), labels),
                 lambda: ce.forward(x, labels.view(2, 4)), lambda: ce.forward(x, torch.zeros(16, dtype=torch.int64, device="cuda")[::2]),
                 lambda: ce.forward(torch.zeros(9, 10, device="cuda"), torch.zeros(9, dtype=torch.int64, device="cuda")),
                 lambda: ce.forward(x, labels, loss=torch.zeros(7, device="cuda")), lambda: ce.forward(x, labels, loss=torch.zeros(8, device="cuda").half()),
                 lambda: ce.gradient(x, labels, dlogits=x.half()), lambda: ce.gradient(x, labels, dlogits=x[:7]), lambda: ce.gradient(x, labels, dlogits=x.cpu()),
                 lambda: ce.gradient(x, labels, scale=torch.ones(2, device="cuda")), lambda: ce.gradient(x, labels, scale=torch.ones(1)),
                 lambda: ce.gradient(x, labels, scale=torch.ones(1, device="cuda").double())]:
        with pytest.raises(ValueError):
            call()
    for bad in ((-1, 10), (8, 0), (8, -3)):
        with pytest.raises(ngsgd.NgsgdError):
            ngsgd.CrossEntropy(*bad)


MASKS = [1e9, 2.0 ** 30, 2.0 ** 30 + 128, 2.0 ** 31, 1e10, 1e12, 1e20, 1e30, 1e38]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])      # (fp16 has no such numbers)
@pytest.mark.parametrize("N,V", [(63, 6), (63, 300), (63, 5001), (63, 33000), (63, 70001), (63, 140001), (130, 70001), (130, 140001)])
def test_large_finite_logits(ngsgd, N, V, dtype):
    """Masks that are finite and not the type's lowest value, and classes far above the rest: rows of 16 lanes to a workgroup, in parts, and wider than the registers."""
    import torch
    torch_type = getattr(torch, dtype)
    rng = np.random.default_rng(14)
    y = rng.integers(0, V, N)
    x = 2.0 * rng.standard_normal((N, V))
    for k, mask in enumerate(MASKS):
        i = 7 * k
        others = np.arange(V) != y[i]
        x[i, others] = -mask                           # the label alone is left
        x[i + 1, V // 4:V // 4 + max(1, V // 2)] = -mask      # a range of classes
        x[i + 1, y[i + 1]] = 1.0
        x[i + 2, rng.random(V) < 0.5] = -mask          # half of them
        x[i + 2, y[i + 2]] = 1.0
        x[i + 3] = -mask                               # all of them
        x[i + 4, y[i + 4]] = -mask                     # the label
        x[i + 5, (y[i + 5] + 1) % V] = mask            # another class far above
        x[i + 6, y[i + 6]] = mask                      # the label far above
    x = matrix(torch, x, torch_type, 1, 1)
    ce, labels = ngsgd.CrossEntropy(N, V), torch.from_numpy(y).cuda()
    loss, d = ce.gradient(x, labels, scale=0.5)
    assert bool(loss.isfinite().all()) and bool(d.isfinite().all())
    check(torch, x, y, 0.5, loss, d)
    assert torch.equal(ce.forward(x, labels), loss)
    for k in range(len(MASKS)):
        i = 7 * k
        assert float(loss[i]) == 0 and not bool(d[i].any()) and float(loss[i + 6]) == 0 and not bool(d[i + 6].any())
        assert float(loss[i + 3]) == pytest.approx(np.log(V), rel=1e-6)
    ce.gradient(x, labels, scale=0.5, dlogits=x)
    assert torch.equal(x, d)


def columns_at_borders(rng, V, E, parts):
    """Both sides of the borders of pieces of E columns (the first one's, the last ones', those between a row's threads and rounds, between the rest and
    what is held of a wide row, between parts), and some others."""
    pieces = (V - 1) // E + 1 if V >= E else V
    share = -(-pieces // parts)
    at = {0, 1, 2, 3, E, V // 2, V // 3, V - E, V - 2 * E}
    for threads in (16, 64, 256, 512, 1024):
        at |= {threads * E * k for k in (1, 2, 3, 4, 7, 8, 15)}
    at |= {share * E * k for k in range(1, parts)} | {(pieces - 12 * 1024) * E, (pieces - 1) * E, (pieces - 2) * E}
    at = {b + s for b in at for s in (-1, 0)} | {V - 1 - k for k in range(2 * E)} | set(rng.integers(0, V, 20).tolist())
    return np.array(sorted(c for c in at if 0 <= c < V))


def count_columns(torch, ngsgd, V, dtype, at, N):
    """Rows of zeros but for one column each.

    16 at the label: its loss is log1p((V - 1) e^-16).  The others are 1 each in units of their own largest, whole numbers that fp32 adds exactly, so the loss counts the
    columns: off by 16 u of itself (an exponential 3 u, a product, the label's power 2 u, a division 3 u, log1p 4 u; and 2^-40 of the argument), where one
    column makes 1 / V.  16 elsewhere: a column that is left out makes the loss log V, one that is taken twice adds log 2 to it."""
    p = np.exp(-16.0)
    E, half = (4, 0.0) if dtype == torch.float32 else (8, torch.finfo(dtype).eps / 2)
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2
    total = 1 + (V - 1) * p
    ce = ngsgd.CrossEntropy(N, V)
    for first in range(0, len(at), N):
        c = np.resize(at[first:first + N], N)
        rows, columns = torch.arange(N, device="cuda"), torch.from_numpy(c).cuda()
        x = torch.zeros(N, V, dtype=dtype, device="cuda")
        x[rows, columns] = 16.0
        loss, d = ce.gradient(x, columns)
        want = float(np.log1p((V - 1) * p))
        assert bool(((loss.double() - want).abs() <= 16 * U * want).all()), (V, first, float(((loss.double() - want) / max(want, 1e-30)).abs().max()))
        label, d[rows, columns] = d[rows, columns].double(), float("nan")
        assert bool(((label + (V - 1) * p / total).abs() <= (32 * U + half) * (V - 1) * p + tiny).all())
        there = d.isfinite().sum(1)
        assert bool((there == V - 1).all())
        assert bool((((d.double() - p / total).abs() <= (40 * U + half) * p + tiny) | d.isnan()).all())
        if V == 1:
            continue
        labels = torch.from_numpy((c + 1 + V // 3) % V).cuda()
        labels[labels == columns] = (columns[labels == columns] + 1) % V
        loss, d = ce.gradient(x, labels)
        # (K u of a sum of K additions, an eighth of log 2 at most here)
        assert bool(((loss.double() - 16 - np.log(total)).abs() <= (V / 64 + 60) * U + 16 * 4 * U).all()), (V, first)
        assert bool(((d[rows, columns].double() - 1 / total).abs() <= (V / 64 + 60) * U + half).all())
        assert bool((d[rows, labels].double() + 1).abs().max() <= 2 * p + half)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [*WIDTHS, 140001, 250001])
def test_every_column_counts_once(ngsgd, V, dtype):
    """Many rows, and few ones, which are cut into parts where they are wide."""
    import torch
    dtype = getattr(torch, dtype)
    E = 4 if dtype == torch.float32 else 8
    rng = np.random.default_rng(V)
    for N in (130, 100, 5) if V > 4096 * E else (130,):
        parts = 1 if N >= 128 else min(64, -(-1024 // N), -(-V // E) // 512)
        count_columns(torch, ngsgd, V, dtype, columns_at_borders(rng, V, E, max(1, parts)), N)


def test_every_column_of_narrow_rows(ngsgd):
    import torch
    for V, dtype in ((5, torch.float32), (37, torch.float16), (64, torch.bfloat16), (129, torch.bfloat16), (515, torch.float32), (1025, torch.float16)):
        count_columns(torch, ngsgd, V, dtype, np.arange(V), V)


@pytest.mark.parametrize("N,V", [(1, 3_000_001), (2, 2_500_000), (130, 2_000_003)])
def test_columns_of_very_wide_rows(ngsgd, N, V):
    """A piece of 8 columns that is left out or taken twice makes 8 / V = 2.7e-6 at least, where 16 u = 9.5e-7 are allowed."""
    import torch
    rng = np.random.default_rng(V)
    pieces = -(-V // 8)
    at = np.concatenate([[0, 7, 8, V - 1, V - 8, V - 9, V // 2, (pieces - 12288) * 8 - 1, (pieces - 12288) * 8], rng.integers(0, V, 3)])
    count_columns(torch, ngsgd, V, torch.bfloat16, at, N)
