"""GPU parity: the norm of many gradients and clipping through the C ABI against the float64 definition.

Tolerances.  u = 2^-24.  Squares are summed in 64 bits, so the norm and the factor are off by their rounding to fp32 (u, and 1e-10 of the sums); a
clipped gradient by the factor's u, the product's u and the rounding to its type.
"""
import numpy as np
import pytest

from oracle.clipping import norm_and_factor

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = ["float32", "bfloat16", "float16"]
SIZES = [1, 2, 3, 4, 5, 7, 8, 9, 255, 256, 257, 1000, 2047, 2048, 2049, 4095, 4096, 4097, 10001, 70000]


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def placed(torch, a, dtype, shift=0, behind=0):
    """Inside a buffer of 77s, `shift` elements behind an aligned address."""
    flat = torch.full((len(a) + shift + behind,), 77.0, dtype=dtype, device="cuda")
    flat[shift:shift + len(a)] = torch.from_numpy(np.asarray(a)).to(dtype).cuda()
    return flat[shift:shift + len(a)]


def make(torch, rng, sizes, dtype, scale=1e-2, shift=0, behind=0):
    return [placed(torch, rng.standard_normal(n) * scale, dtype, shift, behind) for n in sizes]


def check(torch, grads, max_norm, norm, factor, out=None):
    want, f = norm_and_factor([f64(g) for g in grads], max_norm)
    if want > float(torch.finfo(torch.float32).max) * (1 + U):       # rounded to fp32, that is infinity
        assert float(norm) == float("inf")
    else:
        assert abs(float(norm) - want) <= (U + 1e-10) * want
    assert abs(float(factor) - f) <= (U + 1e-10) * f
    for g, o in zip(grads, out or []):
        if g is None:
            continue
        info = torch.finfo(o.dtype)
        clipped = f64(g) * f
        assert np.all(np.abs(f64(o) - clipped) <= (2 * U + info.eps / 2) * np.abs(clipped) * (1 + 1e-6) + info.smallest_normal * info.eps / 2)
    return want


@pytest.mark.parametrize("shift", [0, 1, 3])
@pytest.mark.parametrize("dtype", TYPES)
def test_every_size(ngsgd, dtype, shift):
    """Each alone and all together, from one element to many pieces, aligned and not; in place and into others."""
    import torch
    dtype = getattr(torch, dtype)
    rng = np.random.default_rng(shift)
    for sizes in [[n] for n in SIZES] + [SIZES]:
        grads = make(torch, rng, sizes, dtype, shift=shift, behind=5)
        g = ngsgd.GradientNorm(grads)
        expect = norm_and_factor([f64(t) for t in grads], 1.0)[0]
        for max_norm in (0.3 * expect, 2.0 * expect, float("inf")):
            check(torch, grads, max_norm, *g.norm(grads, max_norm))
            out = make(torch, rng, sizes, dtype, shift=(shift + 2) % 4, behind=5)
            check(torch, grads, max_norm, *g.clip(grads, max_norm, out=out), out)
            inside = [placed(torch, f64(t), dtype, shift) for t in grads]
            norm, factor = g.clip(inside, max_norm)
            assert all(torch.equal(a, b) for a, b in zip(inside, out))
            check(torch, grads, max_norm, norm, factor)
            for t, n in zip(out, sizes):
                behind = t.as_strided((n + 5,), (1,), t.storage_offset())[n:]
                assert bool((behind == 77).all())


@pytest.mark.parametrize("count", [1, 2, 127, 128, 129, 255, 256, 257, 1000])
def test_many_tensors(ngsgd, count):
    """More than the arguments of one launch hold, some of them empty or without a gradient."""
    import torch
    rng = np.random.default_rng(count)
    sizes = [0 if k % 11 == 5 else 1 + 37 * k % 600 for k in range(count)]
    grads = make(torch, rng, sizes, torch.float32)
    grads = [None if k % 7 == 3 else t for k, t in enumerate(grads)]
    g = ngsgd.GradientNorm([torch.empty(n, device="cuda") for n in sizes])
    kept = [None if t is None else t.clone() for t in grads]
    expect = norm_and_factor([f64(t) for t in grads], 1.0)[0]
    check(torch, kept, 0.5 * expect, *g.norm(grads, 0.5 * expect))
    norm, factor = g.clip(grads, 0.5 * expect)
    check(torch, kept, 0.5 * expect, norm, factor, grads)


@pytest.mark.parametrize("dtype", TYPES)
def test_large_tensors(ngsgd, dtype):
    """Pieces of more than the least size, of several tensors."""
    import torch
    dtype = getattr(torch, dtype)
    grads = [(1e-3 * torch.randn(n, device="cuda")).to(dtype) for n in (9_000_001, 5, 13_000_000)]
    g = ngsgd.GradientNorm(grads)
    want = float(torch.sqrt(sum(t.double().square().sum() for t in grads)))
    norm, factor = g.norm(grads, 1.0)
    assert abs(float(norm) - want) <= (U + 1e-10) * want and abs(float(factor) - min(1.0, 1.0 / want)) <= (U + 1e-10) / want
    out = [torch.empty_like(t) for t in grads]
    norm, factor = g.clip(grads, 1.0, out=out)
    assert all(torch.equal(o, (t.float() * factor).to(dtype)) for o, t in zip(out, grads))


@pytest.mark.parametrize("sizes", [[4096 * 32], [4096 * 32 + 1], [4096] * 32, [4096] * 33, [1] * 32, [1] * 33, [4097] * 16, [4097] * 17])
def test_one_workgroup_and_more(ngsgd, sizes):
    """32 pieces of 4096 elements are one workgroup's, 33 are not."""
    import torch
    rng = np.random.default_rng(len(sizes))
    for dtype in (torch.float32, torch.bfloat16):
        grads = make(torch, rng, sizes, dtype)
        g = ngsgd.GradientNorm(grads)
        expect = norm_and_factor([f64(t) for t in grads], 1.0)[0]
        out = [torch.empty_like(t) for t in grads]
        for bound in (0.4 * expect, 3.0 * expect):
            check(torch, grads, bound, *g.norm(grads, bound))
            check(torch, grads, bound, *g.clip(grads, bound, out=out), out)


def test_gradients_next_to_each_other(ngsgd):
    """Views of one buffer: clipped in place, and one buffer into another; in another order or over each other it is refused."""
    import torch
    flat, other = torch.randn(3000, device="cuda"), torch.zeros(3000, device="cuda")
    cut = lambda t: [t[:1000], t[1000:1700], t[1700:]]
    g = ngsgd.GradientNorm(cut(flat))
    want = flat.clone()
    norm, factor = g.clip(cut(flat), 5.0, out=cut(other))
    assert torch.equal(flat, want) and torch.equal(other, want * factor)
    g.clip(cut(flat), 5.0)
    assert torch.equal(flat, other)
    one, two = torch.ones(1000, device="cuda"), torch.ones(1000, device="cuda")
    pair = ngsgd.GradientNorm([one, two])
    for grads, out in (([one, one], None), ([one, two], [two, one]), ([one, two], [other[:1000], other[999:1999]])):
        with pytest.raises(ngsgd.NgsgdError):
            pair.clip(grads, 1.0, out=out)
    assert [float(t) for t in pair.norm([one, one], 1.0)] == pytest.approx([2000 ** 0.5, 2000 ** -0.5], rel=1e-7)


def test_squares_beyond_fp32(ngsgd):
    """Numbers whose squares overflow or vanish in fp32; the norm does too where it is above what fp32 holds."""
    import torch
    for scale in (1e30, 3e37, 1e-30, 1e-38):
        grads = [torch.full((1000,), scale, device="cuda"), torch.full((3,), scale, dtype=torch.float32, device="cuda")]
        g = ngsgd.GradientNorm(grads)
        check(torch, grads, scale, *g.norm(grads, scale))
    big = [torch.full((10000,), 3e38, device="cuda")]
    norm, factor = ngsgd.GradientNorm(big).norm(big, 3e38)
    assert float(norm) == float("inf") and float(factor) == pytest.approx(0.01, rel=1e-6)      # formed from the norm in 64 bits


def test_zero_and_bad_numbers(ngsgd):
    import torch
    grads = [torch.zeros(5000, device="cuda"), torch.zeros(3, device="cuda")]
    g = ngsgd.GradientNorm(grads)
    for bound in (0.0, 1.0, float("inf")):
        norm, factor = g.clip(grads, bound)
        assert float(norm) == 0 and float(factor) == 1 and not any(bool(t.any()) for t in grads)
    grads[0][4321] = 2.0
    norm, factor = g.clip(grads, 0.0)
    assert float(norm) == 2 and float(factor) == 0 and not bool(grads[0].any())
    grads[1][2] = float("inf")
    norm, factor = g.norm(grads, 1.0)
    assert float(norm) == float("inf") and float(factor) == 0
    assert [float(t) for t in g.norm(grads)] == [float("inf"), 1.0]
    grads[0][0] = float("nan")
    assert all(bool(t.isnan()) for t in g.norm(grads, 1.0)) and all(bool(t.isnan()) for t in g.norm(grads))
    none = ngsgd.GradientNorm([torch.zeros(0, device="cuda"), torch.zeros(4, device="cuda")])
    assert [float(t) for t in none.clip([torch.zeros(0, device="cuda"), None], 1.0)] == [0.0, 1.0]


def test_in_place_with_a_factor_of_one(ngsgd):
    """Bits stay, those of subnormal numbers and negative zeros too."""
    import torch
    rng = np.random.default_rng(2)
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        grads = make(torch, rng, [3000, 77], dtype)
        grads[0][0], grads[0][1] = -0.0, torch.finfo(dtype).smallest_normal / 4
        kept = [t.clone() for t in grads]
        ints = torch.int32 if dtype == torch.float32 else torch.int16
        ngsgd.GradientNorm(grads).clip(grads, 1e6)
        assert all(torch.equal(a.view(ints), b.view(ints)) for a, b in zip(grads, kept))


def test_shapes_and_another_type_than_the_parameters(ngsgd):
    import torch
    params = [torch.zeros(30, 50, device="cuda"), torch.zeros(50, device="cuda"), torch.zeros((), device="cuda")]
    g = ngsgd.GradientNorm(params, grad_dtype=torch.bfloat16)
    grads = [torch.randn(p.shape, device="cuda").bfloat16() for p in params]
    kept = [t.clone() for t in grads]
    norm, factor = torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    got = g.clip(grads, 3.0, norm=norm, factor=factor)
    assert got[0] is norm and got[1] is factor
    check(torch, kept, 3.0, norm, factor, grads)


def test_repeated_calls_give_the_same_bits(ngsgd):
    import torch
    grads = [torch.randn(n, device="cuda") for n in (3_000_000, 10, 70000)]
    g = ngsgd.GradientNorm(grads)
    first = g.norm(grads, 1.0)
    for _ in range(4):
        assert all(torch.equal(a, b) for a, b in zip(g.norm(grads, 1.0), first))


def test_two_streams_and_objects(ngsgd):
    import torch
    grads = [torch.randn(n, device="cuda") for n in (3_000_000, 10, 70000)]
    want = ngsgd.GradientNorm(grads).norm(grads, 1.0)
    both, streams = [ngsgd.GradientNorm(grads) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = [[op.norm(grads, 1.0, stream=q) for op, q in zip(both, streams)] for _ in range(5)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for pair in outs for o in pair for a, b in zip(o, want))


@pytest.mark.parametrize("sizes", [[300], [5000, 3, 900], [2_000_000, 17], [10] * 300])
def test_captured_calls(ngsgd, sizes):
    """Replayed with other gradients than were captured, with eager work between; two graphs share the workspace."""
    import torch
    grads = [torch.randn(n, device="cuda") for n in sizes]
    out = [torch.empty_like(t) for t in grads]
    g = ngsgd.GradientNorm(grads)
    g.norm(grads, 1.0)
    torch.cuda.synchronize()
    first, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(first):
        norm = g.norm(grads, 1.0)
    with torch.cuda.graph(second):
        clipped = g.clip(grads, 0.5, out=out)
    for k in range(4):
        for t in grads:
            t.normal_().mul_(1.0 + k)
        first.replay()
        second.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(norm, g.norm(grads, 1.0)))
        if sum(sizes) < 1_000_000:
            check(torch, grads, 0.5, *clipped, out)
        other = [torch.empty_like(t) for t in grads]
        g.clip(grads, 0.5, out=other)
        assert all(torch.equal(a, b) for a, b in zip(out, other))


def test_an_object_that_is_gone_before_its_work(ngsgd):
    import torch
    grads = [torch.randn(n, device="cuda") for n in (3_000_000, 70000)]
    want = ngsgd.GradientNorm(grads).norm(grads, 1.0)
    s, big = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda")
    for given in (True, False):
        g = ngsgd.GradientNorm(grads)
        size = g.workspace.numel()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for _ in range(30):
                big = big @ big * 1e-3
            if not given:
                got = g.norm(grads, 1.0)
        if given:
            got = g.norm(grads, 1.0, stream=s)
        del g
        taken = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _ in range(3)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        del taken


def test_offsets_beyond_32_bits(ngsgd):
    import torch
    n = 2 ** 31 + 5000
    big = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    big[n - 1], big[2 ** 31], big[0] = 2.0, 4.0, 4.0
    g = ngsgd.GradientNorm([big])
    norm, factor = g.clip([big], 3.0)
    assert float(norm) == 6 and float(factor) == 0.5
    assert [float(big[i]) for i in (0, 2 ** 31, n - 1)] == [2.0, 2.0, 1.0]


def test_refusals(ngsgd):
    import torch
    grads = [torch.zeros(5, device="cuda"), torch.zeros(7, device="cuda")]
    g = ngsgd.GradientNorm(grads)
    for call in [lambda: g.norm(grads[:1]), lambda: g.norm([grads[1], grads[0]]), lambda: g.norm([grads[0], grads[1].half()]), lambda: g.norm([grads[0], grads[1].cpu()]),
                 lambda: g.norm([grads[0], torch.zeros(14, device="cuda")[::2]]), lambda: g.clip(grads, 1.0, out=grads[:1]), lambda: g.clip(grads, 1.0, out=[grads[0], None]),
                 lambda: g.clip(grads, 1.0, out=[grads[0], grads[0]]), lambda: g.norm(grads, norm=torch.zeros(2, device="cuda")),
                 lambda: g.norm(grads, factor=torch.zeros(1)), lambda: ngsgd.GradientNorm([grads[0], torch.zeros(3)]), lambda: ngsgd.GradientNorm([torch.zeros(3, device="cuda").double()])]:
        with pytest.raises(ValueError):
            call()
    for bad in (-1.0, float("nan")):
        with pytest.raises(ngsgd.NgsgdError):
            g.norm(grads, bad)
        with pytest.raises(ngsgd.NgsgdError):
            g.clip(grads, bad)


def test_no_output_for_an_empty_gradient(ngsgd):
    import torch
    rng = np.random.default_rng(20)
    grads = make(torch, rng, [5, 0, 700], torch.float32, scale=1.0) + [None]
    op = ngsgd.GradientNorm([*grads[:3], grads[0]])
    out = [torch.full_like(grads[0], 9.0), None, torch.full_like(grads[2], 9.0), None]
    norm, factor = op.clip(grads, 0.5, out=out)
    check(torch, [grads[0], grads[2]], 0.5, norm, factor, out=[out[0], out[2]])
