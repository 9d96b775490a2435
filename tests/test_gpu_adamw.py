"""GPU parity: AdamW over many tensors through the C ABI against the float64 definition.

Tolerances, u = 2^-24: m and v are sums of two products of positive parts (4 u of the magnitudes' sum; v's gradient is scaled, then
squared: 6 u), and p of the kept part (3 u) and the step, whose m, v, unbiasing factors, root, quotient and products are
off by 16 u together; epsilon only shrinks that.  Parameters in 16 bits are rounded once more.
Codes of 8 bits are those of a number within these bounds: the coding is monotone, so the held value lies between the
codings of the two bounds (under the block's own exponent, which the reference takes from its own numbers: where a block's
largest number is within the bound of 1.875 2^E both exponents would do, and no seed used here has such a block).
"""
import numpy as np
import pytest

from oracle import adamw as oracle

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = [("float32", "float32"), ("float32", "bfloat16"), ("float32", "float16"), ("bfloat16", "bfloat16"), ("bfloat16", "float32"),
         ("float16", "float16"), ("float16", "float32")]
SIZES = [1, 2, 3, 4, 5, 255, 256, 257, 511, 1000, 4095, 4096, 4097, 10001]


def f64(t):
    return t.detach().double().cpu().numpy().reshape(-1)


class Bench:
    """Tensors with their optimizer, and the float64 copy of everything."""

    def __init__(self, torch, ngsgd, sizes, ptype="float32", gtype="float32", bits=32, master=False, seed=0, shift=0, t=0, **kw):
        self.torch, self.bits, self.kw = torch, bits, kw
        self.rng = np.random.default_rng(100 + seed)
        self.ptype, self.gtype = getattr(torch, ptype), getattr(torch, gtype)
        self.shift, self.sizes = shift, list(sizes)
        self.params = [self.placed(self.rng.standard_normal(n) * 0.1, self.ptype) for n in sizes]
        self.opt = ngsgd.AdamW(self.params, grad_dtype=self.gtype, state_bits=bits, master=master, **kw)
        assert self.opt.elements == sum(-(-n // 256) * 256 for n in sizes)
        if t:
            m, v = np.zeros(self.opt.elements), np.zeros(self.opt.elements)
            for o, n in zip(self.opt.offsets, sizes):
                spread = np.exp2(self.rng.uniform(-12, 0, n))
                m[o:o + n] = 1e-2 * self.rng.standard_normal(n) * spread
                v[o:o + n] = (1e-2 * self.rng.uniform(0.1, 2.0, n) * spread) ** 2
            as32 = [torch.from_numpy(a).float().cuda() for a in (m, v)]
            fp32 = None
            if master:
                fp32 = self.opt.master.clone()
                fp32 += 1e-4 * fp32
            self.opt.set_state(as32[0], as32[1], t, master=fp32)
            if bits == 8:
                held_m, held_v = (f64(a) for a in self.opt.state())
                assert np.array_equal(held_m, oracle.coded(oracle.coded_m, m.astype(np.float32)))
                # the root is rounded to fp32 first (u of itself, 2 u of v): one element in 10^6 is that near to a border
                v = v.astype(np.float32).astype(np.float64)
                low, high = (oracle.coded(oracle.coded_v, v * (1 + s * 2.5 * U)) for s in (-1, 1))
                assert np.all((low <= held_v) & (held_v <= high))
        self.t = t

    def placed(self, a, dtype):
        """On the device, `shift` elements behind an aligned address."""
        flat = self.torch.zeros(len(a) + self.shift, dtype=dtype, device="cuda")
        flat[self.shift:] = self.torch.from_numpy(np.asarray(a)).to(dtype).cuda()
        return flat[self.shift:]

    def gradients(self, scale=1e-2):
        return [self.placed(self.rng.standard_normal(n) * scale, self.gtype) for n in self.sizes]

    def before(self):
        fp32 = self.opt.master
        p = [f64(p) for p in self.params] if fp32 is None else [f64(fp32[o:o + n]) for o, n in zip(self.opt.offsets, self.sizes)]
        m, v = (f64(a) for a in self.opt.state())
        return p, [m[o:o + n] for o, n in zip(self.opt.offsets, self.sizes)], [v[o:o + n] for o, n in zip(self.opt.offsets, self.sizes)]

    def check(self, before, grads, lr, scale=1.0, betas=(0.9, 0.999), epsilon=1e-8):
        """The step that has just run, from the state before it."""
        self.t += 1
        torch, opt = self.torch, self.opt
        m_all, v_all = (f64(a) for a in opt.state())
        for i, n in enumerate(self.sizes):
            o = opt.offsets[i]
            p0, m0, v0 = (b[i] for b in before)
            m_got, v_got, p_got = m_all[o:o + n], v_all[o:o + n], f64(self.params[i])
            pad = -(-n // 256) * 256
            assert np.all(m_all[o + n:o + pad] == 0) and np.all(v_all[o + n:o + pad] == 0)
            if grads[i] is None:
                assert np.array_equal(m_got, m0) and np.array_equal(v_got, v0)
                assert np.array_equal(p_got if opt.master is None else f64(opt.master[o:o + n]), p0)
                continue
            decay, rate = (np.broadcast_to(self.kw.get(k, d), len(self.sizes))[i] for k, d in (("weight_decay", 0.0), ("rate", 1.0)))
            decay, rate = float(np.float32(decay)), float(np.float32(rate))
            g = f64(grads[i])
            p, m, v = oracle.step(p0, g, m0, v0, self.t, lr * rate, betas[0], betas[1], epsilon, decay, scale)
            e_m = 4 * U * (betas[0] * np.abs(m0) + (1 - betas[0]) * np.abs(g * scale))
            e_v = 6 * U * v
            moved = np.abs(p - p0 * (1 - lr * rate * decay))
            # m's error, seen by the step, is that of its terms, not of their sum
            unit = lr * rate / (1 - betas[0] ** self.t) / (np.sqrt(v / (1 - betas[1] ** self.t)) + epsilon)
            e_p = 3 * U * np.abs(p0) + 16 * U * moved + e_m * unit
            if self.bits == 32:
                assert np.all(np.abs(m_got - m) <= e_m) and np.all(np.abs(v_got - v) <= e_v)
            else:
                for at in range(0, n, 256):
                    k = slice(at, min(at + 256, n))
                    shares = oracle.share(len(m[k]), self.t, o + at)
                    low, high = (oracle.coded_m(m[k] + s * e_m[k], shares, m[k]) for s in (-1, 1))
                    low, high = np.minimum(low, high), np.maximum(low, high)
                    # a number whose magnitude is rounded between two codes may be on either side of both
                    assert np.all((low <= m_got[k]) & (m_got[k] <= high))
                    low, high = (oracle.coded_v(np.maximum(v[k] + s * e_v[k], 0), shares, v[k]) for s in (-1, 1))
                    assert np.all((low <= v_got[k]) & (v_got[k] <= high))
                    exact = oracle.coded_m(m[k], shares)
                    assert np.mean(m_got[k] != exact) <= 2 / 256 and np.mean(v_got[k] != oracle.coded_v(v[k], shares)) <= 2 / 256
            if opt.master is None:
                info = torch.finfo(self.ptype)
                extra = info.eps / 2 if self.ptype != torch.float32 else 0.0
                assert np.all(np.abs(p_got - p) <= e_p * (1 + 2 * extra) + extra * np.abs(p) + info.smallest_normal * info.eps / 2)
            else:
                fp32 = opt.master[o:o + n]
                assert np.all(np.abs(f64(fp32) - p) <= e_p) and torch.equal(fp32.to(self.ptype), self.params[i])

    def steps(self, count, lr=1e-3, **call):
        for _ in range(count):
            before, grads = self.before(), self.gradients()
            self.opt.step(grads, lr, **call)
            scale = call.get("grad_scale")
            self.check(before, grads, float(np.float32(lr)) if not self.torch.is_tensor(lr) else float(lr), 1.0 if scale is None else float(scale))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("shift", [0, 1])
def test_every_type_at_every_edge(ngsgd, bits, types, shift):
    """From one element to more than two pieces of work, aligned and not; the first steps and one far into a training."""
    import torch
    for t in (0, 500):
        Bench(torch, ngsgd, SIZES, *types, bits=bits, shift=shift, t=t, weight_decay=0.1).steps(2)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("types", TYPES[3:], ids="-".join)
def test_fp32_copies(ngsgd, bits, types):
    import torch
    for t in (0, 20):
        b = Bench(torch, ngsgd, SIZES, *types, bits=bits, master=True, t=t, weight_decay=0.01)
        b.steps(3)
    # steps below half a step of the 16 bits add up
    b = Bench(torch, ngsgd, [300], *types, bits=bits, master=True)
    first = b.params[0].clone()
    g = [torch.ones(300, dtype=b.gtype, device="cuda")]
    p, m, v = f64(first), np.zeros(300), np.zeros(300)
    for t in range(1, 65):
        b.opt.step(g, 1e-4)
        p, m, v = oracle.step(p, np.ones(300), m, v, t, float(np.float32(1e-4)))
        if bits == 8:
            m, v = (oracle.coded(which, np.pad(a, (0, 212)), t)[:300] for which, a in ((oracle.coded_m, m), (oracle.coded_v, v)))
    assert not torch.equal(first, b.params[0])
    # In 32 bits: 64 steps of 1e-4, each off by 16 u, and 64 roundings of numbers below 1 (0.5 u each, 64 * 0.5 u / 64e-4 = 3e-4).  In 8
    # bits the reference holds codes too, and an element that is coded on the other side of a border (one in 10^6 at a
    # step) moves the mean over 300 by at most 1 / 8 / 300 = 4e-4.
    moved = float((b.opt.master[:300].double() - first.double()).mean())
    assert moved == pytest.approx(float((p - f64(first)).mean()), rel=1e-3)
    if bits == 32:
        assert moved == pytest.approx(-64e-4, rel=1e-3)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_large_tensor_among_small_ones(ngsgd, bits):
    import torch
    Bench(torch, ngsgd, [7, 3_000_001, 900], bits=bits, t=3).steps(1)


@pytest.mark.parametrize("count", [447, 448, 449, 1000])
def test_many_tensors(ngsgd, count):
    """More tensors than the arguments of one launch hold: the step is counted once."""
    import torch
    b = Bench(torch, ngsgd, [1 + 37 * k % 600 for k in range(count)], bits=32)
    b.steps(2)
    assert b.opt.steps() == 2


@pytest.mark.parametrize("bits", [32, 8])
def test_tensors_without_gradient_or_elements(ngsgd, bits):
    import torch
    b = Bench(torch, ngsgd, [300, 0, 5000, 0, 4], bits=bits, t=5)
    for missing in ([2], [0, 4], [0, 2, 4]):
        before, grads = b.before(), b.gradients()
        for i in missing:
            grads[i] = None
        b.opt.step(grads, 1e-3)
        b.check(before, grads, float(np.float32(1e-3)))
    assert b.opt.steps() == 8
    empty = ngsgd.AdamW([torch.zeros(0, device="cuda")], state_bits=bits)
    empty.step([torch.zeros(0, device="cuda")], 0.1)
    assert empty.steps() == 1 and empty.elements == 0
    empty.state(torch.bfloat16)


@pytest.mark.parametrize("bits", [32, 8])
def test_rates_decays_and_factors_on_the_device(ngsgd, bits):
    import torch
    b = Bench(torch, ngsgd, [500, 600, 700], bits=bits, t=9, weight_decay=[0.0, 0.1, 0.5], rate=[1.0, 0.0, 2.5])
    b.steps(1, lr=1e-2)
    b.steps(1, lr=torch.tensor([0.0078125], device="cuda"), grad_scale=torch.tensor([0.375], device="cuda"))
    b.steps(1, grad_scale=-2.0)


def test_other_betas(ngsgd):
    import torch
    b = Bench(torch, ngsgd, [777], betas=(0.0, 0.95), epsilon=1e-6)
    for _ in range(3):
        before, grads = b.before(), b.gradients()
        b.opt.step(grads, 1e-3)
        b.check(before, grads, float(np.float32(1e-3)), betas=(0.0, 0.95), epsilon=float(np.float32(1e-6)))
    b = Bench(torch, ngsgd, [777], betas=(0.0, 0.0), epsilon=0.0)
    before, grads = b.before(), b.gradients()
    b.opt.step(grads, 0.5)
    b.check(before, grads, 0.5, betas=(0.0, 0.0), epsilon=0.0)


def test_zero_gradients(ngsgd):
    """Nothing moves but by the decay; with epsilon 0 a zero moment over a zero root is NaN by the formula."""
    import torch
    for bits in (32, 8):
        p = torch.full((300,), 2.0, device="cuda")
        opt = ngsgd.AdamW([p], state_bits=bits, weight_decay=0.5)
        opt.step([torch.zeros(300, device="cuda")], 0.25)
        assert bool((p == 1.75).all()) and all(bool((a == 0).all()) for a in opt.state())
        opt = ngsgd.AdamW([p], state_bits=bits, epsilon=0.0)
        opt.step([torch.zeros(300, device="cuda")], 0.25)
        assert bool(p.isnan().all())


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_bad_gradients_stay_with_their_element(ngsgd, bits, bad):
    import torch
    a, b = (Bench(torch, ngsgd, [1000], bits=bits, t=4) for _ in range(2))
    grads = a.gradients()
    a.opt.step(grads, 1e-3)
    grads[0][300] = bad
    b.opt.step(grads, 1e-3)
    for _ in range(2):
        others = [i for i in range(1000) if i != 300]
        assert torch.equal(a.params[0][others], b.params[0][others]) and bool(b.params[0][300].isnan())
        for x, y in zip(a.opt.state(), b.opt.state()):
            assert torch.equal(x[others], y[others]) and not bool(y[300].isfinite())
        grads[0][300] = 0.5
        a.opt.step(grads, 1e-3)
        b.opt.step(grads, 1e-3)


def test_codes_of_every_size_of_number(ngsgd):
    """Blocks far from 1, blocks with one number, numbers below the least code: what set_state holds is the nearest code, and setting
    what was read changes nothing."""
    import torch
    rng = np.random.default_rng(8)
    blocks = []
    for scale in (0, -20, -60, -100, -115, -125, 20, 60):
        blocks.append(rng.standard_normal(256) * np.exp2(rng.uniform(-25, 0, 256) + scale))
    blocks.append(np.zeros(256))
    one = np.zeros(256)
    one[17] = -3.0
    blocks.append(one)
    top = rng.standard_normal(256)
    top[3] = 1.875
    blocks.append(top)
    m = np.concatenate(blocks).astype(np.float32)
    with np.errstate(under="ignore", over="ignore"):
        v = np.minimum(m.astype(np.float64) ** 2, 3e38).astype(np.float32)
    opt = ngsgd.AdamW([torch.zeros(len(m), device="cuda")], state_bits=8)
    opt.set_state(torch.from_numpy(m).cuda(), torch.from_numpy(v).cuda(), 7)
    held_m, held_v = opt.state()
    assert np.array_equal(f64(held_m), oracle.coded(oracle.coded_m, m))
    want_v = oracle.coded(oracle.coded_v, v)      # (its square may be too small for fp32)
    assert np.array_equal(f64(held_v), want_v.astype(np.float32).astype(np.float64))
    # (a square below 2^-126, the least normal number, is one that bf16 rounds)
    as_bf16 = opt.state(torch.bfloat16)
    normal = held_v >= 2.0 ** -126
    assert torch.equal(as_bf16[0].float(), held_m) and torch.equal(as_bf16[1].float()[normal], held_v[normal])
    opt.set_state(held_m, held_v, 7)
    assert torch.equal(opt.state()[0], held_m) and opt.steps() == 7
    normal = held_v > 1e-30                         # (a root of a number that fp32 holds with few bits is another one)
    assert torch.equal(opt.state()[1][normal], held_v[normal])


def test_small_changes_of_v_add_up(ngsgd):
    """8 bits: v follows a changed gradient as in 32 bits, though a step changes it by a thousandth."""
    import torch
    n = 2048
    p = [torch.zeros(n, device="cuda") for _ in range(2)]
    opts = [ngsgd.AdamW([q], state_bits=bits) for q, bits in zip(p, (8, 32))]
    start = torch.full((n,), 1.0, device="cuda")
    g = [torch.full((n,), 2.0, device="cuda")]
    for opt in opts:
        opt.set_state(start, start, 1000)
    for _ in range(1000):
        for opt in opts:
            opt.step(g, 1e-4)
    v8, v32 = (float(opt.state()[1].mean()) for opt in opts)
    assert v32 == pytest.approx(4.0 - 3.0 * 0.999 ** 1000, rel=1e-4)
    # an element's root is held to an eighth of its binade, and rounded evenly: the mean over the elements is within a twentieth
    assert abs(v8 - v32) < v32 / 20
    assert abs(float(p[0].mean()) / float(p[1].mean()) - 1.0) < 0.05


def test_captured_steps_count_on(ngsgd):
    """A captured step replayed between eager ones: bit for bit what eager steps give."""
    import torch
    for bits in (32, 8):
        a, b = (Bench(torch, ngsgd, [300, 5000], bits=bits, t=2) for _ in range(2))
        grads = a.gradients()
        lr = torch.tensor([1e-3], device="cuda")
        a.opt.step(grads, lr)
        b.opt.step(grads, lr)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            b.opt.step(grads, lr)
        for k in range(5):
            for g in grads:
                g.copy_(torch.randn(g.shape, device="cuda") * 1e-2)
            lr.fill_(1e-3 / (k + 1))
            a.opt.step(grads, lr)
            if k == 2:
                b.opt.step(grads, lr)
            else:
                graph.replay()
            torch.cuda.synchronize()
            assert a.opt.steps() == b.opt.steps() == 4 + k
            assert all(torch.equal(x, y) for x, y in zip(a.params + list(a.opt.state()), b.params + list(b.opt.state())))


def test_on_another_stream(ngsgd):
    import torch
    a, b = (Bench(torch, ngsgd, [300, 50000], bits=8, t=2) for _ in range(2))
    grads = a.gradients()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        a.opt.step(grads, 1e-3)
        b.opt.step(grads, 1e-3, stream=s)
    want, got = a.opt.state(), b.opt.state(stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(x, y) for x, y in zip(a.params + list(want), b.params + list(got)))


@pytest.mark.parametrize("bits", [8, 32])
def test_more_than_2_31_elements(ngsgd, bits):
    """The last elements of a tensor whose places need more than 32 bits, and the first ones."""
    import torch
    n, ends = 2 ** 31 + 300, 600
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(5)
    # from places that begin a block: 2^31 - 512 and 0
    for at in (0, 2 ** 31 - 512):
        p[at:at + ends] = torch.from_numpy(rng.standard_normal(ends)).bfloat16().cuda()
        g[at:at + ends] = torch.from_numpy(rng.standard_normal(ends)).bfloat16().cuda()
    before = {at: (f64(p[at:at + ends]), f64(g[at:at + ends])) for at in (0, 2 ** 31 - 512)}
    opt = ngsgd.AdamW([p], state_bits=bits)
    opt.step([g], 0.01)
    m, v = opt.state()
    for at, (p0, g0) in before.items():
        want, m1, v1 = oracle.step(p0, g0, np.zeros(ends), np.zeros(ends), 1, float(np.float32(0.01)))
        assert np.all(np.abs(f64(p[at:at + ends]) - want) <= 2.0 ** -8 * np.abs(want) + 16 * U * 0.01 + 3 * U * np.abs(p0))
        k = slice(at, at + 512)          # whole blocks
        if bits == 8:
            for got, which, a in ((m, oracle.coded_m, m1), (v, oracle.coded_v, v1)):
                want = np.concatenate([which(a[i:i + 256], oracle.share(256, 1, at + i)) for i in (0, 256)])
                assert np.array_equal(f64(got[k]), want)
        else:
            assert np.all(np.abs(f64(m[k]) - m1[:512]) <= 4 * U * np.abs(m1[:512])) and np.all(np.abs(f64(v[k]) - v1[:512]) <= 6 * U * v1[:512])
    middle = slice(2 ** 30, 2 ** 30 + 10 ** 6)
    assert not bool(p[middle].any()) and not bool(m[middle].any()) and not bool(v[middle].any())
    del p, g, m, v, opt
    torch.cuda.empty_cache()


def test_state_goes_out_and_in(ngsgd):
    """A second optimizer with the first one's state goes on as the first does."""
    import torch
    for kw in (dict(bits=32), dict(bits=8), dict(bits=8, ptype="bfloat16", gtype="bfloat16", master=True)):
        a = Bench(torch, ngsgd, SIZES, t=30, **kw)
        a.steps(2)
        b = Bench(torch, ngsgd, SIZES, seed=1, **kw)
        m, v = (x.clone() for x in a.opt.state())
        for p, q in zip(a.params, b.params):
            q.copy_(p)
        b.opt.set_state(m, v, a.opt.steps(), master=None if a.opt.master is None else a.opt.master.clone())
        grads = a.gradients()
        a.opt.step(grads, 1e-3)
        b.opt.step(grads, 1e-3)
        assert all(torch.equal(x, y) for x, y in zip(a.params + list(a.opt.state()), b.params + list(b.opt.state())))
        b.opt.set_state(None, None, 0)
        assert b.opt.steps() == 0 and all(bool((x == 0).all()) for x in b.opt.state())


def test_refusals(ngsgd):
    import torch
    p = [torch.zeros(10, device="cuda"), torch.zeros(4, 5, device="cuda")]
    for bad in (lambda: ngsgd.AdamW([p[0], p[1].half()]), lambda: ngsgd.AdamW([p[1].t()]), lambda: ngsgd.AdamW([p[0].double()]),
                lambda: ngsgd.AdamW(p, weight_decay=[0.1]), lambda: ngsgd.AdamW(p, grad_dtype=torch.float64)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: ngsgd.AdamW([p[0], p[0]]), lambda: ngsgd.AdamW([p[0], p[0][9:]]), lambda: ngsgd.AdamW(p, master=True),
                lambda: ngsgd.AdamW(p, state_bits=16), lambda: ngsgd.AdamW(p, betas=(0.9, 1.0))):
        with pytest.raises(ngsgd.NgsgdError):
            bad()
    opt = ngsgd.AdamW(p)
    g = [torch.zeros(10, device="cuda"), torch.zeros(4, 5, device="cuda")]
    for bad in (lambda: opt.step(g[:1], 0.1), lambda: opt.step([g[0], g[0]], 0.1), lambda: opt.step([g[0].half(), g[1]], 0.1),
                lambda: opt.step([g[0].cpu(), g[1]], 0.1), lambda: opt.step([g[0], torch.zeros(5, 4, device="cuda").t()], 0.1),
                lambda: opt.step(g, torch.tensor([0.1])), lambda: opt.step(g, torch.zeros(2, device="cuda")),
                lambda: opt.step(g, 0.1, grad_scale=torch.ones(1, device="cuda").double()),
                lambda: opt.set_state(g[0], g[0], 1)):
        with pytest.raises(ValueError):
            bad()
    flat = torch.zeros(opt.elements, device="cuda")
    with pytest.raises(ngsgd.NgsgdError):
        opt.set_state(flat, flat, -1)
    with pytest.raises(ngsgd.NgsgdError):
        opt.set_state(flat, flat, 1, master=flat)
    assert opt.steps() == 0


@pytest.mark.parametrize("lr,decay", [(2e-5, 0.01), (1e-5, 0.01), (1e-6, 0.1), (1e-6, 0.01)])
@pytest.mark.parametrize("bits,master", [(32, False), (8, False), (32, True), (8, True)])
def test_small_decays_are_applied(ngsgd, bits, master, lr, decay):
    """A decay of less than a step of fp32 shows in the mean over many elements.

    Tolerance for the mean of (p - want) / before: an element is rounded once, by at most u of itself, evenly over the elements (their
    steps differ by many times their last bit), so the mean has a standard deviation of u / sqrt(3 n), taken six times; the step, known to 16 u, has
    a sign of its own in each element.  A factor 1 - lr decay rounded to fp32 would be off by up to u / 2 in all elements alike, 150 times that."""
    import torch
    n = 1 << 20
    b = Bench(torch, ngsgd, [n], *(("bfloat16", "bfloat16") if master else ()), bits=bits, master=master, t=500, weight_decay=decay)
    start = b.rng.choice([-1.0, 1.0], n) * b.rng.uniform(1 / 16, 1 / 8, n)
    fp32 = torch.from_numpy(start).float().cuda()
    m, v = (a.clone() for a in b.opt.state())
    if not master:
        b.params[0].copy_(fp32)
    b.opt.set_state(m, v, 500, master=fp32 if master else None)
    (p0,), (m0,), (v0,) = b.before()
    grads = b.gradients()
    b.opt.step(grads, lr)
    rate, fade = float(np.float32(lr)), float(np.float32(decay))
    want, _, _ = oracle.step(p0, f64(grads[0]), m0, v0, 501, rate, decay=fade)
    got = f64(b.opt.master if master else b.params[0])
    moved = want - p0 * (1 - rate * fade)
    assert abs(np.mean((got - want) / p0)) <= 6 * U / np.sqrt(3 * n) + 16 * U * abs(np.mean(moved / p0))


@pytest.mark.parametrize("decay", [0.0, 0.25])
@pytest.mark.parametrize("bits", [32, 8])
def test_infinite_parameters_stay(ngsgd, bits, decay):
    """p (1 - lr decay) of an infinite p (a bias that masks) is p; its neighbours move as without it."""
    import torch
    a, b = (Bench(torch, ngsgd, [300], bits=bits, t=3, weight_decay=decay) for _ in range(2))
    for at, value in ((5, float("inf")), (299, float("-inf"))):
        b.params[0][at] = value
    grads = a.gradients()
    for opt in (a.opt, b.opt):
        opt.step(grads, 0.5)
    assert float(b.params[0][5]) == float("inf") and float(b.params[0][299]) == float("-inf")
    others = [i for i in range(300) if i not in (5, 299)]
    assert torch.equal(a.params[0][others], b.params[0][others])


@pytest.mark.parametrize("betas", [(0.99999, 0.999995), (0.999995, 0.99999), (0.9999, 0.9999)])
def test_betas_near_one(ngsgd, betas):
    """Moments in fp32 fade by 1 - beta in the mean, though beta itself has no more than 24 bits there.

    Tolerance, with c = (1 - beta) 2^23 the steps of the last bit by which a number of 1 fades: roundings are even over many elements (6 standard deviations
    of u / sqrt(3 n)), but for the ends of the range of what fades, c to 2 c steps, which shift the mean by at most 1 / 8 of a step's c-th
    part at either."""
    import torch
    n = 1 << 20
    b = Bench(torch, ngsgd, [n], betas=betas, t=500)
    _, (m0,), (v0,) = b.before()
    b.opt.step([torch.zeros(n, device="cuda")], 1e-3)
    _, (m1,), (v1,) = b.before()
    for before, after, beta in ((m0, m1, betas[0]), (v0, v1, betas[1])):
        part, c = 1 - beta, (1 - beta) * 2 ** 23
        assert abs(np.mean((before - after) / before) - part) <= 6 * U / np.sqrt(3 * n) + part * 0.25 / c ** 2


@pytest.mark.parametrize("betas", [(0.9, 0.999), (0.5, 0.5)])
def test_infinite_moments_stay_infinite(ngsgd, betas):
    """A v above what fp32 holds stays so, and its element (whose step is 0) where it is."""
    import torch
    p = torch.ones(4, device="cuda")
    opt = ngsgd.AdamW([p], betas=betas)
    opt.step([torch.tensor([1e30, 1.0, -1e30, 0.0], device="cuda")], 0.125)
    for _ in range(2):
        v = opt.state()[1]
        assert v[[0, 2]].tolist() == [float("inf")] * 2 and bool(v[[1, 3]].isfinite().all())
        assert p[[0, 2, 3]].tolist() == [1.0] * 3
        opt.step([torch.zeros(4, device="cuda")], 0.125)


@pytest.mark.parametrize("master", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", ["epsilon", "lr", "scale"])
def test_what_is_behind_a_tensor_stays_zero(ngsgd, bad, bits, master):
    """The flat arrays' padding, whatever becomes of the elements."""
    import torch
    sizes = [1, 300, 256, 4097, 6]
    dtype = "bfloat16" if master else "float32"
    b = Bench(torch, ngsgd, sizes, dtype, dtype, bits=bits, master=master, weight_decay=0.1, **({"epsilon": 0.0} if bad == "epsilon" else {}))
    infinite = torch.tensor([float("inf")], device="cuda")
    for grads in (b.gradients(), [torch.zeros_like(p) for p in b.params]):
        b.opt.step(grads, infinite if bad == "lr" else 1e-3, grad_scale=infinite if bad == "scale" else None)
    flat = list(b.opt.state()) + list(b.opt.state(torch.bfloat16)) + ([b.opt.master] if master else [])
    for a in flat:
        for o, n in zip(b.opt.offsets, sizes):
            assert bool((a[o + n:o + -(-n // 256) * 256] == 0).all())


def test_codes_of_the_largest_numbers(ngsgd):
    """What fp32 holds is held as a number, not as infinity, when it is installed and by the steps."""
    import torch
    top = float(torch.finfo(torch.float32).max)
    m = np.zeros(512)
    m[:5] = top, -top, 3.3e38, -3.19e38, 1e38
    m[256:260] = 2.0 ** 127, 1.9 * 2.0 ** 126, 1.0, -2.0 ** 112
    v = np.abs(m)
    for betas in ((0.9, 0.999), (1 - 1e-9, 1 - 1e-9)):
        opt = ngsgd.AdamW([torch.zeros(512, device="cuda")], state_bits=8, betas=betas)
        opt.set_state(*(torch.from_numpy(a).float().cuda() for a in (m, v)), 100)
        held = [f64(a) for a in opt.state()]
        for got, which, a in zip(held, (oracle.coded_m, oracle.coded_v), (m, v)):
            assert np.all(np.isfinite(got)) and np.array_equal(got, oracle.coded(which, a.astype(np.float32)))
        for t in range(101, 109):
            opt.step([torch.zeros(512, device="cuda")], 0.0)
            for k, (which, beta) in enumerate(zip((oracle.coded_m, oracle.coded_v), betas)):
                held[k] = oracle.coded(which, beta * held[k], t)
                assert np.all(np.isfinite(held[k])) and np.array_equal(f64(opt.state()[k]), held[k])


def test_steps_on_the_stream_that_steps(ngsgd):
    import torch
    big = torch.randn(4096, 4096, device="cuda")
    opt = ngsgd.AdamW([torch.zeros(300, device="cuda")])
    g = torch.ones(300, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(30):          # some milliseconds before the steps' turn
            big = big @ big * 1e-3
    for _ in range(3):
        opt.step([g], 1e-3, stream=s)
    assert opt.steps(stream=s) == 3
    with torch.cuda.stream(s):
        opt.step([g], 1e-3)
        assert opt.steps() == 4
    torch.cuda.current_stream().wait_stream(s)


@pytest.mark.parametrize("types", [("float32", "bfloat16"), ("bfloat16", "float32")], ids="-".join)
def test_codes_are_those_of_the_definition(ngsgd, types):
    """Every code of a million, and the same from run to run.  What is coded is known to 2^-44 of itself, and a border between codes is as near
    to one element in 10^11."""
    import torch
    n, t = 1 << 20, 40
    runs = [Bench(torch, ngsgd, [n], *types, bits=8, t=t) for _ in range(3)]
    _, (m0,), (v0,) = runs[0].before()
    grads = runs[0].gradients()
    for b in runs:
        b.opt.step(grads, 1e-3, grad_scale=0.375)
    for b in runs[1:]:
        assert torch.equal(b.params[0], runs[0].params[0]) and all(torch.equal(x, y) for x, y in zip(b.opt.state(), runs[0].opt.state()))
    _, m, v = oracle.step(np.zeros(n), f64(grads[0]), m0, v0, t + 1, 1e-3, scale=0.375)
    for got, which, a in zip(runs[0].opt.state(), (oracle.coded_m, oracle.coded_v), (m, v)):
        assert np.array_equal(f64(got), oracle.coded(which, a, t + 1).astype(np.float32))
