"""GPU parity: the embedding and its gradient through the C ABI against the float64 definition.

Tolerances.  u = 2^-24 is half a step of fp32, u_t of the output's type.  A looked-up row is one product: u of it, then u_t.  A sum of n rows in
fp32, in whatever order, is off by at most n u times the sum of the magnitudes; the scale adds u of the result, an addition to what is there
another u, and the output's type u_t.
"""
import numpy as np
import pytest

from oracle import embedding as oracle

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
COMBOS = [("float32", "float32"), ("bfloat16", "float32"), ("bfloat16", "bfloat16"), ("float16", "float32"), ("float16", "float16")]   # rows, table
INDEX = ["int32", "int64"]


def f64(t):
    return t.detach().double().cpu().numpy()


def half_step(torch, dtype):
    return torch.finfo(dtype).eps / 2 if dtype != torch.float32 else 0.0


def tiny(torch, dtype):
    """Half a step among the smallest numbers of a type."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def matrix(torch, a, dtype, pad=0, shift=0):
    """Rows inside a wider buffer of 77s that starts `shift` elements behind an aligned address."""
    n, d = a.shape
    flat = torch.full((n * (d + pad) + shift,), 77.0, dtype=dtype, device="cuda")
    wide = flat[shift:].view(n, d + pad)
    wide[:, :d] = torch.from_numpy(a).to(dtype).cuda()
    return wide[:, :d]


def make_tokens(torch, rng, count, vocabulary, index, law="zipf", padded=0.1):
    if law == "zipf":
        p = 1.0 / np.arange(1, vocabulary + 1) ** 1.1
        t = rng.choice(vocabulary, count, p=p / p.sum())
    elif law == "uniform":
        t = rng.integers(0, vocabulary, count)
    else:                              # one of them
        t = np.full(count, vocabulary - 1 if law == "last" else 0)
    t = t.astype(np.int64)
    outside = [-1, vocabulary, -2 ** 31, 2 ** 31 - 1] + ([2 ** 32, -2 ** 63, 2 ** 63 - 1, 2 ** 32 + 1] if index == "int64" else [])
    where = rng.random(count) < padded
    t[where] = rng.choice(outside, where.sum())
    return torch.from_numpy(t).to(getattr(torch, index)).cuda(), t


def check_forward(torch, tokens, table, scale, y):
    want = oracle.forward(tokens, f64(table), float(np.float32(scale)))
    h = half_step(torch, y.dtype)
    assert np.all(np.abs(f64(y) - want) <= (U + h * (1 + U)) * np.abs(want) + tiny(torch, y.dtype))


def check_backward(torch, dy, tokens, V, scale, got, before=None):
    scale, dy = float(np.float32(scale)), f64(dy)
    named = (tokens >= 0) & (tokens < V)
    total, sizes = (torch.zeros(V, dy.shape[1], dtype=torch.float64).index_add_(0, torch.from_numpy(tokens[named]), torch.from_numpy(a[named])).numpy() * f
                    for a, f in ((dy, scale), (np.abs(dy), abs(scale))))
    if len(tokens) <= 4096:
        assert np.allclose(total, oracle.backward(dy, tokens, V, scale), rtol=1e-12, atol=1e-12)
    counts = np.bincount(tokens[named], minlength=V)[:, None]
    bound = (counts + 1) * U * (1 + 1e-3) * sizes
    if before is not None:
        total = total + before
        bound = bound + U * np.abs(total)
    h = half_step(torch, got.dtype)
    g = f64(got)
    assert np.all(np.abs(g - total) <= bound * (1 + h) + h * np.abs(total) + tiny(torch, got.dtype))
    quiet = (counts == 0)[:, 0]
    assert np.array_equal(g[quiet], np.zeros_like(g[quiet]) if before is None else before[quiet])


@pytest.mark.parametrize("types", COMBOS, ids="-".join)
@pytest.mark.parametrize("D", [1, 2, 3, 4, 7, 8, 9, 15, 16, 63, 64, 65, 128, 500, 512, 513, 1024, 1030, 2047, 2048, 2049, 5000])
def test_widths(ngsgd, D, types):
    import torch
    dtype, ttype = (getattr(torch, t) for t in types)
    rng = np.random.default_rng(D)
    N, V = 101, 37
    tokens, t = make_tokens(torch, rng, N, V, INDEX[D % 2])
    e = ngsgd.Embedding(N, V, D, scale=1.7)
    for pad, shift in ((0, 0), (3, 1), (8, 8)):
        table = matrix(torch, rng.standard_normal((V, D)), ttype, pad, shift)
        y = matrix(torch, np.zeros((N, D)), dtype, pad, shift)
        check_forward(torch, t, table, 1.7, e.forward(tokens, table, out=y))
        dense = e.forward(tokens, table, dtype=dtype)
        assert dense.is_contiguous() and torch.equal(dense, y)
        dy = matrix(torch, rng.standard_normal((N, D)), dtype, pad, shift)
        into = matrix(torch, rng.standard_normal((V, D)), ttype, pad, shift)
        before = f64(into)
        e.backward(dy, tokens, dtable=into, accumulate=True)
        check_backward(torch, dy, t, V, 1.7, into, before)
        e.backward(dy, tokens, dtable=into)
        check_backward(torch, dy, t, V, 1.7, into)
        assert torch.equal(e.backward(dy, tokens, dtype=ttype), into)
        if pad:                        # what is between the rows stays
            for m in (y, into):
                wide = m.as_strided((m.shape[0], D + pad), (D + pad, 1), m.storage_offset())
                assert bool((wide[:, D:] == 77).all())


@pytest.mark.parametrize("law", ["zipf", "uniform", "first", "last"])
@pytest.mark.parametrize("N,V", [(1, 1), (1, 1000), (2, 1), (3, 70000), (15, 4), (16, 5000), (63, 64), (64, 2), (65, 300), (127, 1), (128, 7), (129, 9),
                                 (1000, 50), (1024, 255), (1025, 256), (2048, 257), (4095, 3), (4096, 4096), (4097, 65535), (8192, 65536), (8193, 65537),
                                 (5120, 33), (5121, 900), (10007, 1), (16384, 100), (31745, 2), (32767, 40000), (32768, 5), (32769, 12000), (20011, 511), (30000, 131073), (65537, 1023), (100003, 3000)])
def test_counts(ngsgd, N, V, law):
    """From one token to many, every kind of vocabulary: spread, equal, all one."""
    import torch
    rng = np.random.default_rng(N + V)
    index, D = INDEX[N % 2], 8 + N % 3
    e = ngsgd.Embedding(N, V, D, scale=0.5)
    table = matrix(torch, rng.standard_normal((V, D)), torch.float32)
    for padded in (0.0, 0.2):
        tokens, t = make_tokens(torch, rng, N, V, index, law, padded)
        if N <= 4097:
            check_forward(torch, t, table, 0.5, e.forward(tokens, table))
        dy = matrix(torch, rng.standard_normal((N, D)), torch.bfloat16)
        check_backward(torch, dy, t, V, 0.5, e.backward(dy, tokens, dtype=torch.float32))


@pytest.mark.parametrize("N,V,D", [(262144, 5000, 8), (262145, 131072, 8), (300007, 70, 12), (1000003, 2 ** 20 + 1, 5), (20000, 3, 8), (9000, 2 ** 21 + 5, 4),
                                   (129, 600011, 8), (128, 600011, 8), (500, 1500007, 3)])
def test_many_tokens_and_large_tables(ngsgd, N, V, D):
    """More tiles than a workgroup adds up itself; digits of one to three passes; wavefronts that clear 64 rows and more."""
    import torch
    rng = np.random.default_rng(N)
    e = ngsgd.Embedding(N, V, D)
    for law in ("zipf", "uniform", "last"):
        tokens, t = make_tokens(torch, rng, N, V, "int64", law, 0.05)
        dy = matrix(torch, rng.standard_normal((N, D)), torch.float32)
        check_backward(torch, dy, t, V, 1.0, e.backward(dy, tokens))


@pytest.mark.parametrize("N,D,types", [(3000, 8192, ("float32", "float32")), (4099, 4097, ("bfloat16", "float32")), (2100, 8192, ("bfloat16", "bfloat16")),
                                       (5003, 5001, ("float16", "float32")), (16411, 1024, ("bfloat16", "bfloat16")), (40000, 257, ("float32", "float32"))])
def test_lookups_of_large_rows(ngsgd, N, D, types):
    """Rows in slabs, and outputs that are written past the caches."""
    import torch
    rng = np.random.default_rng(D)
    V = 333
    dtype, ttype = (getattr(torch, t) for t in types)
    e = ngsgd.Embedding(N, V, D, scale=0.3)
    tokens, t = make_tokens(torch, rng, N, V, "int32")
    for pad in (0, 3):
        table = matrix(torch, rng.standard_normal((V, D)), ttype, pad, pad)
        y = e.forward(tokens, table, dtype=dtype)
        named = torch.from_numpy((t >= 0) & (t < V)).cuda()
        want = table.double()[torch.where(named, tokens.long(), 0)] * float(np.float32(0.3)) * named[:, None]
        h = half_step(torch, dtype)
        assert bool(((y.double() - want).abs() <= (U + h * (1 + U)) * want.abs() + tiny(torch, dtype)).all())


@pytest.mark.parametrize("N,V,D", [(5000, 700, 1000), (4096, 40, 2050), (60000, 900, 129), (9000, 20000, 77), (33000, 5, 260)])
@pytest.mark.parametrize("types", COMBOS, ids="-".join)
def test_long_sums(ngsgd, N, V, D, types):
    """Tokens that are named hundreds and thousands of times, in every type."""
    import torch
    dtype, ttype = (getattr(torch, t) for t in types)
    rng = np.random.default_rng(N + D)
    tokens, t = make_tokens(torch, rng, N, V, "int32", padded=0.03)
    dy = matrix(torch, rng.standard_normal((N, D)) + 0.3, dtype)
    e = ngsgd.Embedding(N, V, D)
    check_backward(torch, dy, t, V, 1.0, e.backward(dy, tokens, dtype=ttype))
    into = matrix(torch, rng.standard_normal((V, D)), ttype)
    before = f64(into)
    e.backward(dy, tokens, dtable=into, accumulate=True)
    check_backward(torch, dy, t, V, 1.0, into, before)


def test_nothing_but_padding(ngsgd):
    import torch
    for N in (1, 100, 9000):
        e = ngsgd.Embedding(N, 50, 12)
        tokens = torch.full((N,), -1, device="cuda")
        table, dy = torch.full((50, 12), float("nan"), device="cuda"), torch.full((N, 12), float("nan"), device="cuda")
        assert bool((e.forward(tokens, table) == 0).all())
        assert bool((e.backward(dy, tokens) == 0).all())
        kept = torch.full((50, 12), 3.0, device="cuda")
        assert bool((e.backward(dy, tokens, dtable=kept, accumulate=True) == 3).all())


def test_no_tokens(ngsgd):
    import torch
    e = ngsgd.Embedding(0, 50, 12)
    none = torch.zeros(0, dtype=torch.int64, device="cuda")
    assert e.forward(none, torch.ones(50, 12, device="cuda")).shape == (0, 12)
    assert bool((e.backward(torch.zeros(0, 12, device="cuda"), none) == 0).all())
    kept = torch.full((50, 12), 3.0, device="cuda")
    assert bool((e.backward(torch.zeros(0, 12, device="cuda"), none, dtable=kept, accumulate=True) == 3).all())


def test_fewer_tokens_than_the_workspace_is_for(ngsgd):
    import torch
    rng = np.random.default_rng(3)
    e = ngsgd.Embedding(50000, 300, 20)
    for N in (50000, 1, 4097, 70, 20000, 0, 33):
        tokens, t = make_tokens(torch, rng, N, 300, "int64")
        dy = matrix(torch, rng.standard_normal((N, 20)), torch.float32)
        check_backward(torch, dy, t, 300, 1.0, e.backward(dy, tokens))


def test_bad_numbers_stay_in_their_row(ngsgd):
    """An infinity or NaN among the derivatives reaches its token's row and column alone; of padding, none; rows that no token names may hold anything."""
    import torch
    rng = np.random.default_rng(4)
    N, V, D = 3000, 40, 96
    tokens, t = make_tokens(torch, rng, N, V, "int32", "uniform")
    dy = matrix(torch, rng.standard_normal((N, D)), torch.float32)
    e = ngsgd.Embedding(N, V, D)
    clean = e.backward(dy, tokens)
    at = int(np.flatnonzero(t == 7)[5])
    dy[at, 11], dy[at, 12] = float("nan"), float("inf")
    dy[torch.from_numpy(np.flatnonzero((t < 0) | (t >= V))).cuda()] = float("nan")
    got = e.backward(dy, tokens)
    assert bool(got[7, 11].isnan()) and bool(got[7, 12].isinf())
    got[7, 11:13] = clean[7, 11:13]
    assert torch.equal(got, clean)
    table = matrix(torch, rng.standard_normal((V, D)), torch.float32)
    table[39] = float("nan")
    few = torch.tensor([0, 1, 38], dtype=torch.int32, device="cuda")
    assert bool(ngsgd.Embedding(3, V, D).forward(few, table).isfinite().all())


def test_more_than_one_dimension(ngsgd):
    import torch
    rng = np.random.default_rng(5)
    tokens, t = make_tokens(torch, rng, 60, 30, "int64")
    e = ngsgd.Embedding(60, 30, 24, scale=2.0)
    table = matrix(torch, rng.standard_normal((30, 24)), torch.bfloat16)
    y = e.forward(tokens.view(3, 4, 5), table)
    assert y.shape == (3, 4, 5, 24) and torch.equal(y.view(60, 24), e.forward(tokens, table))
    dy = torch.randn(3, 4, 5, 24, device="cuda").bfloat16()
    check_backward(torch, dy.view(60, 24), t, 30, 2.0, e.backward(dy, tokens.view(3, 4, 5), dtype=torch.float32))
    one = e.forward(tokens[0], table)
    assert one.shape == (24,) and torch.equal(one, y[0, 0, 0])
    assert torch.equal(e.backward(dy[0, 0, 0], tokens[0]), e.backward(dy[0, 0, :1], tokens[:1]))


def test_repeated_calls_give_the_same_bits(ngsgd):
    import torch
    rng = np.random.default_rng(6)
    for N, V, D in ((700, 30, 600), (50000, 1000, 72)):
        tokens, _ = make_tokens(torch, rng, N, V, "int32")
        dy = torch.randn(N, D, device="cuda")
        e = ngsgd.Embedding(N, V, D)
        first = e.backward(dy, tokens)
        for _ in range(4):
            assert torch.equal(e.backward(dy, tokens), first)


def test_gradient_is_its_difference(ngsgd):
    """<dy, y(W + E) - y(W)> = <dW, E>: the lookup is linear.  In fp32: y is off by 2 u of its numbers, dW by the bound above."""
    import torch
    rng = np.random.default_rng(7)
    N, V, D = 500, 60, 50
    tokens, t = make_tokens(torch, rng, N, V, "int64")
    W, E = (torch.from_numpy(rng.standard_normal((V, D))).float().cuda() for _ in range(2))
    dy = torch.from_numpy(rng.standard_normal((N, D))).float().cuda()
    e = ngsgd.Embedding(N, V, D, scale=1.3)
    sum_ = W + E
    left = ((e.forward(tokens, sum_).double() - e.forward(tokens, W).double()) * dy.double()).sum()
    right = (e.backward(dy, tokens).double() * (sum_.double() - W.double())).sum()
    most = float((e.forward(tokens, sum_).double().abs() + e.forward(tokens, W).double().abs()).mul(dy.double().abs()).sum())
    # terms: a y is off by u of itself; a sum of at most N terms by N u (every token's own count is less)
    assert abs(float(left - right)) <= (2 + N) * U * most


def test_on_another_stream(ngsgd):
    import torch
    rng = np.random.default_rng(8)
    N, V, D = 20000, 500, 100
    tokens, t = make_tokens(torch, rng, N, V, "int32")
    table, dy = torch.randn(V, D, device="cuda"), torch.randn(N, D, device="cuda")
    e = ngsgd.Embedding(N, V, D)
    want = e.forward(tokens, table), e.backward(dy, tokens)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = e.forward(tokens, table, stream=s), e.backward(dy, tokens, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # two objects at the same time, each on a stream of its own
    both, streams = [ngsgd.Embedding(N, V, D) for _ in range(2)], [s, torch.cuda.Stream()]
    torch.cuda.synchronize()
    outs = [[op.backward(dy, tokens, stream=q) for op, q in zip(both, streams)] for _ in range(5)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[1]) for pair in outs for o in pair)


@pytest.mark.parametrize("N", [70, 5000, 40000])
def test_captured_calls(ngsgd, N):
    """Replayed with other tokens and rows than were captured, with eager work between; two graphs share the workspace."""
    import torch
    rng = np.random.default_rng(9)
    V, D = 400, 64
    e = ngsgd.Embedding(N, V, D, scale=3.0)
    tokens, _ = make_tokens(torch, rng, N, V, "int64")
    table, dy = torch.randn(V, D, device="cuda"), torch.randn(N, D, device="cuda")
    kept = torch.zeros(V, D, device="cuda")
    e.backward(e.forward(tokens, table), tokens)
    torch.cuda.synchronize()
    first, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(first):
        y = e.forward(tokens, table)
        grad = e.backward(dy, tokens)
    with torch.cuda.graph(second):
        e.backward(dy, tokens, dtable=kept, accumulate=True)
    for k in range(4):
        now, t = make_tokens(torch, rng, N, V, "int64", ["zipf", "first", "uniform", "last"][k])
        tokens.copy_(now)
        dy.normal_()
        kept.fill_(1.0)
        first.replay()
        second.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, e.forward(now, table)) and torch.equal(grad, e.backward(dy, now))
        check_backward(torch, dy, t, V, 3.0, kept, np.ones((V, D)))


def test_an_object_that_is_gone_before_its_work(ngsgd):
    """On another stream than the object was made on: the workspace is nobody else's until that stream is done with it."""
    import torch
    rng = np.random.default_rng(10)
    N, V, D = 30000, 900, 64
    tokens, _ = make_tokens(torch, rng, N, V, "int32")
    dy = torch.randn(N, D, device="cuda")
    want = ngsgd.Embedding(N, V, D).backward(dy, tokens)
    s, big = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda")
    for given in (True, False):
        e = ngsgd.Embedding(N, V, D)
        size = e.workspace.numel()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for _ in range(30):
                big = big @ big * 1e-3
            if not given:
                got = e.backward(dy, tokens)
        if given:
            got = e.backward(dy, tokens, stream=s)
        del e
        taken = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _ in range(3)]
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        del taken


def test_offsets_beyond_32_bits(ngsgd):
    """A table, rows and a gradient of more than 2^31 elements each; the last rows of each."""
    import torch
    V, D = 70001, 32768
    table = torch.zeros(V, D, dtype=torch.bfloat16, device="cuda")
    table[V - 1] = 5.0
    table[65536] = 2.0
    table[1] = 7.0
    tokens = torch.full((V,), -1, dtype=torch.int32, device="cuda")
    tokens[V - 1], tokens[V - 2], tokens[0] = V - 1, 65536, 1
    e = ngsgd.Embedding(V, V, D)
    y = e.forward(tokens, table)
    assert bool((y[V - 1] == 5).all()) and bool((y[V - 2] == 2).all()) and bool((y[0] == 7).all()) and not bool(y[1:V - 2].any())
    del table
    y[V - 1] = 3.0
    y[1:V - 2] = float("nan")
    grad = e.backward(y, tokens)
    assert bool((grad[V - 1] == 3).all()) and bool((grad[65536] == 2).all()) and bool((grad[1] == 7).all())
    grad[V - 1], grad[65536], grad[1] = 0.0, 0.0, 0.0
    assert not bool(grad.any())


def test_rows_behind_the_last_stay(ngsgd):
    import torch
    rng = np.random.default_rng(11)
    N, V, D = 77, 21, 40
    tokens, t = make_tokens(torch, rng, N, V, "int32")
    e = ngsgd.Embedding(N, V, D)
    y, grad = torch.full((N + 5, D), 9.0, device="cuda"), torch.full((V + 5, D), 9.0, device="cuda")
    table = torch.randn(V, D, device="cuda")
    e.forward(tokens, table, out=y[:N])
    e.backward(torch.randn(N, D, device="cuda"), tokens, dtable=grad[:V])
    assert bool((y[N:] == 9).all()) and bool((grad[V:] == 9).all())


def test_refusals(ngsgd):
    import torch
    e = ngsgd.Embedding(8, 10, 16)
    tokens = torch.zeros(8, dtype=torch.int64, device="cuda")
    table, dy = torch.zeros(10, 16, device="cuda"), torch.zeros(8, 16, device="cuda")
    half = table.bfloat16()
    for call in [lambda: e.forward(tokens.cpu(), table), lambda: e.forward(tokens.short(), table), lambda: e.forward(tokens.float(), table),
                 lambda: e.forward(torch.zeros(9, dtype=torch.int64, device="cuda"), table), lambda: e.forward(torch.zeros(16, dtype=torch.int64, device="cuda")[::2], table),
                 lambda: e.forward(tokens, table[:9]), lambda: e.forward(tokens, table[:, :15]), lambda: e.forward(tokens, table.cpu()), lambda: e.forward(tokens, table.double()),
                 lambda: e.forward(tokens, table.t().contiguous().t()), lambda: e.forward(tokens, half, dtype=torch.float32), lambda: e.forward(tokens, half, dtype=torch.float16),
                 lambda: e.forward(tokens, table, out=dy[:7]), lambda: e.forward(tokens, table, out=dy.cpu()), lambda: e.forward(tokens, table, dtype=torch.bfloat16, out=dy),
                 lambda: e.forward(tokens.view(2, 4), table, out=dy),
                 lambda: e.backward(dy[:7], tokens), lambda: e.backward(dy[:, :15], tokens), lambda: e.backward(dy.double(), tokens), lambda: e.backward(dy.cpu(), tokens),
                 lambda: e.backward(dy, tokens, accumulate=True), lambda: e.backward(dy, tokens, dtype=torch.bfloat16), lambda: e.backward(dy, tokens, dtable=table[:9]),
                 lambda: e.backward(dy, tokens, dtable=half), lambda: e.backward(dy, tokens, dtype=torch.float16, dtable=table), lambda: e.backward(dy.view(2, 4, 16), tokens)]:
        with pytest.raises(ValueError):
            call()
    for bad in (float("nan"), float("inf")):
        with pytest.raises(ngsgd.NgsgdError):
            ngsgd.Embedding(8, 10, 16, scale=bad).forward(tokens, table)
    for bad in ((-1, 10, 16), (8, 0, 16), (8, 10, 0)):
        with pytest.raises(ngsgd.NgsgdError):
            ngsgd.Embedding(*bad)
