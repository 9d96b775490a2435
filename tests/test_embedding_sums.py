"""The embedding's gradient, row by row: not one token lost or taken twice, however long its run.

Derivatives are whole numbers from 1 to 8: sums of up to 2^20 of them are below 2^24, so fp32 holds every partial sum exactly, in whatever order, and the
gradient has to be the definition's bit for bit (rounded once where the table has 16 bits).  Derivatives with fractions: a sum is a chain of
additions in its chunk, then of parts by a group of lanes, then of groups two by two; its length times u times the sum of the magnitudes bounds the error.
"""
import numpy as np
import pytest

U = 2.0 ** -24
LAWS = ["zipf", "uniform", "first", "last"]


def make_tokens(rng, count, vocabulary, law, padded):
    if law == "zipf":
        p = 1.0 / np.arange(1, vocabulary + 1) ** 1.1
        t = rng.choice(vocabulary, count, p=p / p.sum())
    elif law == "uniform":
        t = rng.integers(0, vocabulary, count)
    else:
        t = np.full(count, vocabulary - 1 if law == "last" else 0)
    t = t.astype(np.int64)
    where = rng.random(count) < padded
    t[where] = rng.choice([-1, vocabulary], where.sum())
    return t


def sums(torch, dy, tokens, vocabulary):
    """The definition's, in fp64, without the scale."""
    t = torch.from_numpy(tokens)
    named = (t >= 0) & (t < vocabulary)
    return torch.zeros(vocabulary, dy.shape[1], dtype=torch.float64).index_add_(0, t[named], dy.double().cpu()[named])


def longest_chain(count, dim, element_bytes):
    """Additions that one result goes through at most, by the kernels' plan: chunks of sorted tokens for 4096 wavefronts, parts joined by 512 threads."""
    e = 16 // element_bytes if dim >= 16 // element_bytes else 1
    pieces = -(-dim // e)
    lanes = 1
    while lanes < min(pieces, 64):
        lanes *= 2
    units = max(1, 4096 * (64 // lanes) // -(-pieces // 64))
    chunk = 16
    while chunk < 512 and -(-count // chunk) > units:
        chunk *= 2
    groups = 512 // lanes
    return max(128, chunk) + -(-(-(-count // chunk)) // groups) + int(np.log2(groups)) + 2      # (up to 128 tokens: one after the other)


COUNTS = [(1, 3), (2, 1), (63, 2), (64, 64), (65, 1), (127, 3), (128, 1), (129, 1), (130, 9), (1000, 50), (1024, 3), (1025, 256), (2048, 1), (4095, 3), (4096, 1), (4097, 1),
          (4097, 65535), (8192, 100), (8193, 5), (20011, 511), (31745, 2), (32767, 40000), (32768, 1), (32769, 1), (32769, 12000), (65537, 1023), (100003, 3000)]


@pytest.mark.parametrize("law", LAWS)
@pytest.mark.parametrize("N,V", COUNTS)
@pytest.mark.gpu
def test_whole_numbers(ngsgd, N, V, law):
    import torch
    rng = np.random.default_rng(N + V)
    for D, padded in ((8 + N % 3, 0.0), (1, 0.2), (37, 0.1)):
        t = make_tokens(rng, N, V, law, padded)
        tokens = torch.from_numpy(t).cuda()
        dy = torch.from_numpy(rng.integers(1, 9, (N, D))).to(torch.bfloat16).cuda()
        want = (0.5 * sums(torch, dy, t, V)).float().cuda()
        e = ngsgd.Embedding(N, V, D, scale=0.5)
        assert torch.equal(e.backward(dy, tokens, dtype=torch.float32), want)
        assert torch.equal(e.backward(dy, tokens.int()), want.bfloat16())
        assert torch.equal(e.backward(dy.float(), tokens), want)
        into = torch.from_numpy(rng.integers(-99, 99, (V, D))).float().cuda()
        assert torch.equal(e.backward(dy, tokens, dtable=into.clone(), accumulate=True), into + want)


@pytest.mark.parametrize("law", LAWS)
@pytest.mark.parametrize("N,V,D", [(262144, 5000, 8), (262145, 131072, 8), (300007, 70, 12), (1000003, 2 ** 20 + 1, 5), (262144, 1, 64), (9000, 7, 1030), (20011, 300, 773),
                                   (70001, 40, 257), (3000, 5, 4100)])
@pytest.mark.gpu
def test_whole_numbers_in_long_runs(ngsgd, N, V, D, law):
    """Thousands of parts of one run; rows of several slabs."""
    import torch
    rng = np.random.default_rng(N)
    t = make_tokens(rng, N, V, law, 0.05)
    tokens = torch.from_numpy(t).cuda()
    dy = torch.from_numpy(rng.integers(1, 9, (N, D))).float().cuda()
    want = sums(torch, dy, t, V).float().cuda()
    e = ngsgd.Embedding(N, V, D)
    assert torch.equal(e.backward(dy, tokens), want)
    assert torch.equal(e.backward(dy.half(), tokens, dtype=torch.float32), want)
    into = torch.full((V, D), 3.0, device="cuda")
    assert torch.equal(e.backward(dy.half(), tokens, dtable=into, accumulate=True), want + 3)


@pytest.mark.parametrize("N,V,D", [(4096, 1, 16), (32768, 5, 9), (32769, 3, 64), (262144, 5000, 8), (300007, 70, 12), (1000003, 2 ** 20 + 1, 5), (20011, 300, 773)])
@pytest.mark.gpu
def test_fractions_in_long_runs(ngsgd, N, V, D):
    import torch
    rng = np.random.default_rng(N)
    e = ngsgd.Embedding(N, V, D)
    for law in ("zipf", "last"):
        t = make_tokens(rng, N, V, law, 0.05)
        tokens = torch.from_numpy(t).cuda()
        dy = torch.from_numpy(rng.standard_normal((N, D))).float().cuda()
        want, size = sums(torch, dy, t, V), sums(torch, dy.abs(), t, V)
        got = e.backward(dy, tokens).double().cpu()
        assert bool(((got - want).abs() <= longest_chain(N, D, 4) * U * (1 + 1e-3) * size + 2.0 ** -149).all())


def test_a_lost_token_is_seen():
    """On the CPU: the comparisons above refuse a sum without one token of the longest run."""
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(0)
    for N, V, D in ((129, 1, 8), (262144, 1, 64), (1000003, 2 ** 20 + 1, 5)):
        t = make_tokens(rng, N, V, "last", 0.05)
        dy = torch.from_numpy(rng.integers(1, 9, (N, D))).float()
        fewer = t.copy()
        fewer[np.flatnonzero(t == V - 1)[N // 3]] = -1
        assert not torch.equal(sums(torch, dy, t, V), sums(torch, dy, fewer, V))
        assert float(sums(torch, dy, t, V).max()) < 2 ** 24
    # and with fractions, a sum without the longest part
    dy = torch.from_numpy(rng.standard_normal((262144, 8))).float()
    t, fewer = np.zeros(262144, np.int64), np.zeros(262144, np.int64)
    fewer[:512] = -1
    off = (sums(torch, dy, t, 1) - sums(torch, dy, fewer, 1)).abs()
    assert bool((off > longest_chain(262144, 8, 4) * U * sums(torch, dy.abs(), t, 1)).any())
