"""The operators for parameters and layers beside the natural gradient: layer norm with its gradients, and AdamW over many tensors.

Three kinds of case:

  forward    ngsgd_layernorm_forward: y, and the mean and 1 / standard deviation of each row that the backward pass takes
  backward   ngsgd_layernorm_backward: the gradients of the input, the weight and the bias
  adamw      ngsgd_adamw_step over many tensors: the parameters, their fp32 copies where they are kept, and both moments

The tensors of an `adamw` case lie in one flat buffer, each on a multiple of 256 elements, as programs with flat parameter
buffers lay them out; the elements between them are zero and stay so.  Moments in 8 bits are returned as the values that they
stand for, which bfloat16 holds exactly.
"""
import math

import torch

own = False                          # set by the program that measures: the plain forms, or the framework's calls

EPSILON = 1e-5                       # layer norm
BETAS, ADAM_EPSILON = (0.9, 0.999), 1e-8
LR = 2e-5                            # late in a schedule
STEPS_BEFORE = 200                   # the moments are those of a training under way
BLOCK = 256                          # elements that share an exponent where moments are held in 8 bits
DITHER_INDEX, DITHER_STEP = 0x9E3779B1, 0x6A09E667
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def listed():
    return [
        # the smallest call: the hidden layer of a tiny tanh network, 64 rows of 128
        dict(name="forward_smallest", kind="forward", rows=64, dim=128, pad=0, type="fp32", weights="fp32"),
        # odd sizes, rows inside a wider buffer
        dict(name="forward_ragged", kind="forward", rows=3333, dim=1001, pad=6, type="fp16", weights="fp16"),
        # the largest: many rows of a wide layer
        dict(name="forward_large", kind="forward", rows=32768, dim=8192, pad=0, type="bf16", weights="fp32"),
        # the backward pass of the smallest layer
        dict(name="backward_smallest", kind="backward", rows=64, dim=128, pad=0, type="fp32", weights="fp32"),
        # a minibatch of the wide tanh network: 1024 rows of 2048, in 32 bits
        dict(name="backward_wide_tanh", kind="backward", rows=1024, dim=2048, pad=0, type="fp32", weights="fp32"),
        # odd sizes, rows without a common alignment
        dict(name="backward_ragged", kind="backward", rows=4001, dim=773, pad=0, type="bf16", weights="bf16"),
        # the largest: activations in 16 bits, the weight's gradient in 32
        dict(name="backward_large", kind="backward", rows=16384, dim=8192, pad=0, type="bf16", weights="fp32"),
        # the tensors of a tiny tanh network, where the launch is everything
        dict(name="adamw_smallest", kind="adamw", tensors="network", input=40, hidden=128, layers=3, classes=50, type="fp32", grads="fp32",
             bits=32, master=False, clip=False, decay=0.0),
        # the tensors of the speech-shaped network with tanh layers (360 -> 4 x 3000 -> 5000)
        dict(name="adamw_speech", kind="adamw", tensors="network", input=360, hidden=3000, layers=5, classes=5000, type="fp32", grads="fp32",
             bits=32, master=False, clip=False, decay=0.01),
        # odd sizes and moments in 8 bits: blocks that end inside the last exponent's range, tensors of one element
        dict(name="adamw8_ragged", kind="adamw", tensors="mixed", count=61, largest=40009, type="fp16", grads="fp16", bits=8, master=True,
             clip=True, decay=0.1),
        # parameters and gradients in 16 bits, an fp32 copy, clipped gradients
        dict(name="adamw_large_master", kind="adamw", tensors="blocks", width=2048, count=4, type="bf16", grads="bf16", bits=32, master=True,
             clip=True, decay=0.1),
        # the largest: fp32 parameters, gradients in 16 bits, moments in 8
        dict(name="adamw8_large", kind="adamw", tensors="blocks", width=2048, count=5, type="fp32", grads="bf16", bits=8, master=False,
             clip=False, decay=0.1),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["forward", "backward", "adamw"])
    if kind != "adamw":
        dim = _log(rng, 24, 16384)
        most = (1 << 27) // dim
        kind_of = rng.choice(["fp32", "bf16", "bf16", "fp16"])
        return dict(kind=kind, rows=_log(rng, 1, min(65536, most // 2)), dim=dim, pad=rng.choice([0, 0, 8, rng.randint(1, 40)]), type=kind_of,
                    weights=rng.choice(["fp32", kind_of]))
    kind_of = rng.choice(["fp32", "fp32", "bf16", "fp16"])
    case = dict(kind=kind, type=kind_of, grads=rng.choice(["fp32", kind_of] if kind_of != "fp32" else ["fp32", "bf16", "fp16"]),
                bits=rng.choice([8, 32]), master=kind_of != "fp32" and rng.random() < 0.6, clip=rng.random() < 0.5, decay=rng.choice([0.0, 0.01, 0.1]))
    which = rng.choice(["network", "mixed", "blocks"])
    if which == "network":
        case.update(tensors=which, input=4 * _log(rng, 10, 110), hidden=_log(rng, 100, 3000), layers=rng.randint(2, 6), classes=_log(rng, 50, 6000))
    elif which == "mixed":
        case.update(tensors=which, count=rng.randint(1, 120), largest=_log(rng, 2, 200000))
    else:
        case.update(tensors=which, width=8 * _log(rng, 16, 128), count=rng.randint(1, 8))
    return case


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _tensor_sizes(case):
    """Elements of each tensor."""
    if case["tensors"] == "network":      # weights with the bias in the last column; a gain and a bias behind each hidden layer
        dims = [case["input"]] + [case["hidden"]] * (case["layers"] - 1) + [case["classes"]]
        return [dims[l + 1] * (dims[l] + 1) for l in range(case["layers"])] + [case["hidden"]] * (2 * (case["layers"] - 1))
    if case["tensors"] == "mixed":        # from one element up, spread over the logarithm
        n, big = case["count"], case["largest"]
        return [int(round(big ** ((k + 1) / n))) for k in range(n)]
    w = case["width"]                     # blocks of a wide network: matrices, biases, the gain and bias of two layer norms
    return [3 * w * w, 3 * w, w * w, w, 4 * w * w, 4 * w, 4 * w * w, w, w, w, w, w] * case["count"]


def _offsets(sizes):
    at, offsets = 0, []
    for n in sizes:
        offsets.append(at)
        at += -(-n // BLOCK) * BLOCK
    return offsets, at


def _real(sizes, total):
    """One where a tensor has an element, zero in the gaps."""
    offsets, _ = _offsets(sizes)
    steps = torch.zeros(total + 1, dtype=torch.int32)
    steps.index_add_(0, torch.tensor(offsets), torch.ones(len(sizes), dtype=torch.int32))
    steps.index_add_(0, torch.tensor([o + n for o, n in zip(offsets, sizes)]), torch.full((len(sizes),), -1, dtype=torch.int32))
    return steps.cuda().cumsum(0)[:total].to(torch.float32)


def _layer_norm_inputs(case, seed):
    g, n, d = _gen(seed), case["rows"], case["dim"]
    kind, wkind = TYPES[case["type"]], TYPES[case["weights"]]

    def rows(t):                          # inside a wider buffer where the case says so
        wide = torch.zeros(n, d + case["pad"], dtype=kind, device="cuda")
        wide[:, :d] = t.to(kind)
        return wide[:, :d]

    x = torch.randn(n, d, generator=g, device="cuda")
    x *= torch.rand(n, 1, generator=g, device="cuda") * 2.0 + 0.25
    x += torch.randn(n, 1, generator=g, device="cuda") + 0.3 * torch.randn(d, generator=g, device="cuda")
    s = dict(x=rows(x), weight=(1.0 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(wkind),
             bias=(0.2 * torch.randn(d, generator=g, device="cuda")).to(wkind))
    del x
    if case["kind"] == "backward":
        s["dy"] = rows(torch.randn(n, d, generator=g, device="cuda") * 0.1)
        x64 = s["x"].double()             # what the forward pass has kept
        mean = x64.mean(1)
        x64 -= mean[:, None]
        s["mean"], s["rstd"] = mean.float(), (x64.square().mean(1) + EPSILON).rsqrt().float()
    return s


def _adamw_inputs(case, seed):
    g, sizes = _gen(seed), _tensor_sizes(case)
    offsets, total = _offsets(sizes)
    real = _real(sizes, total)
    exact_p = 0.03 * torch.randn(total, generator=g, device="cuda") * real
    p = exact_p.to(TYPES[case["type"]])
    grads = (1e-3 * torch.randn(total, generator=g, device="cuda") * torch.rand(total, generator=g, device="cuda") * real).to(TYPES[case["grads"]])
    m = 2e-4 * torch.randn(total, generator=g, device="cuda") * real
    v = (5e-4 * (0.2 + torch.rand(total, generator=g, device="cuda")) * real).square()
    if case["bits"] == 8:
        half = torch.full((1, 1), 1 << 19, dtype=torch.int32, device="cuda")
        m, v = _held_m(m, half), _held_v(v, half)
    s = dict(p=p, grads=grads, m=m, v=v, sizes=sizes, offsets=offsets, t=STEPS_BEFORE)
    if case["master"]:
        s["master"] = exact_p
    s["clip"] = 0.25 + 0.75 * torch.rand(1, generator=g, device="cuda") if case["clip"] else None
    return s


def prepare(case, seed):
    if case["kind"] != "adamw":
        s = _layer_norm_inputs(case, seed)
        if own:
            import paper_1410_7455_amd as ng
            s["op"] = ng.LayerNorm(case["rows"], case["dim"], EPSILON)
    else:
        s = _adamw_inputs(case, seed)
        if own:
            import paper_1410_7455_amd as ng
            views = [s["p"][o:o + n] for o, n in zip(s["offsets"], s["sizes"])]
            s["op"] = ng.AdamW(views, betas=BETAS, epsilon=ADAM_EPSILON, weight_decay=case["decay"], grad_dtype=TYPES[case["grads"]],
                               state_bits=case["bits"], master=case["master"])
            s["op"].set_state(s["m"].float(), s["v"].float(), s["t"], master=s.get("master"))
            s["grad_list"] = [s["grads"][o:o + n] for o, n in zip(s["offsets"], s["sizes"])]
    s["case"] = case
    return s


def run(state):
    kind = state["case"]["kind"]
    if kind == "forward":
        return _own_forward(state) if own else _forward(state)
    if kind == "backward":
        return _own_backward(state) if own else _backward(state)
    return _own_adamw(state) if own else _adamw(state)


# ---- the framework's calls ----------------------------------------------------------------------------

def _own_forward(s):
    return s["op"].forward(s["x"], s["weight"], s["bias"])


def _own_backward(s):
    return s["op"].backward(s["dy"], s["x"], s["mean"], s["rstd"], s["weight"])


def _own_adamw(s):
    op = s["op"]
    op.step(s["grad_list"], LR, grad_scale=s["clip"])
    m, v = op.state(torch.bfloat16 if s["case"]["bits"] == 8 else torch.float32)
    return [s["p"], m, v] + ([op.master] if s["case"]["master"] else [])


# ---- the plain forms ------------------------------------------------------------------------------------

def _forward(s):
    x = s["x"].float()
    d = x.shape[1]
    mean = x.sum(1) / d
    x = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((x * x).sum(1) / d + EPSILON)
    y = x * rstd[:, None] * s["weight"].float() + s["bias"].float()
    return y.to(s["x"].dtype), mean, rstd


def _backward(s):
    dy, d = s["dy"].float(), s["x"].shape[1]
    xhat = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    dbias = dy.sum(0)
    dweight = (dy * xhat).sum(0)
    g = dy * s["weight"].float()
    c1 = g.sum(1, keepdim=True) / d
    c2 = (g * xhat).sum(1, keepdim=True) / d
    dx = (g - c1 - xhat * c2) * s["rstd"][:, None]
    return dx.to(s["x"].dtype), dweight.to(s["weight"].dtype), dbias.to(s["weight"].dtype)


def _as_bits(a):
    return a.view(torch.int32)


def _held_m(m, dither):
    """The values that the codes of m stand for: a sign, 15 binades below the block's largest, three bits behind the point."""
    shape = m.shape
    a = m.abs().view(-1, BLOCK)
    e = ((_as_bits(a.amax(1)) + 0xFFFFF) >> 23).clamp_min(16)
    base = ((e + 1) * 8 - 128)[:, None]
    least = ((base + 1) << 20).view(torch.float32)
    code = (((_as_bits(a) + dither) >> 20) - base).clamp(1, 127)
    code = torch.where(a < least, (a > least * (dither.float() * 2.0 ** -20)).to(torch.int32), code)
    held = torch.where(code > 0, ((code + base) << 20).view(torch.float32), 0.0)
    return torch.where(m.view(-1, BLOCK) < 0, -held, held).to(torch.bfloat16).view(shape)


def _held_v(v, dither):
    """The values that the codes of v stand for: its root in 31 binades below the block's largest, three bits behind the point."""
    shape = v.shape
    r = torch.sqrt(v).view(-1, BLOCK)
    e = ((_as_bits(r.amax(1)) + 0xFFFFF) >> 23).clamp_min(32)
    base = ((e + 1) * 8 - 255)[:, None]
    code = (((_as_bits(r) + dither) >> 20) - base).clamp(1, 254)
    held = torch.where(r > 0, ((code + base) << 20).view(torch.float32), 0.0)
    return (held * held).to(torch.bfloat16).view(shape)


def _dither(n, t):
    """20 bits for each element: a sequence that visits [0, 1) evenly over the steps, at another phase for each element."""
    u = torch.arange(n, dtype=torch.int32, device="cuda") * (DITHER_INDEX - (1 << 32)) + ((t * DITHER_STEP + (1 << 31)) % (1 << 32) - (1 << 31))
    return ((u >> 12) & 0xFFFFF).view(-1, BLOCK)


def _adamw(s):
    case, t = s["case"], s["t"] + 1
    s["t"] = t
    g = s["grads"].float()
    if s["clip"] is not None:
        g = g * s["clip"]
    b1, b2 = BETAS
    m = b1 * s["m"].float() + (1.0 - b1) * g
    v = b2 * s["v"].float() + (1.0 - b2) * (g * g)
    p = s["master"] if case["master"] else s["p"].float()
    p = p * (1.0 - LR * case["decay"]) - LR * (m / (1.0 - b1 ** t)) / (torch.sqrt(v / (1.0 - b2 ** t)) + ADAM_EPSILON)
    if case["master"]:
        s["master"] = p
    s["p"] = p.to(s["p"].dtype)
    if case["bits"] == 8:
        d = _dither(p.numel(), t)
        m, v = _held_m(m, d), _held_v(v, d)
    s["m"], s["v"] = m, v
    return [s["p"], m, v] + ([p] if case["master"] else [])


# ---- what a pass cannot do without, and the definitions in 64 bits --------------------------------------

def work(case):
    if case["kind"] != "adamw":
        n, d = case["rows"], case["dim"]
        s, w = TYPES[case["type"]].itemsize, TYPES[case["weights"]].itemsize
        if case["kind"] == "forward":
            return {"bytes": 2 * n * d * s + 2 * d * w + 8 * n, "flops": 8 * n * d}
        return {"bytes": 3 * n * d * s + 3 * d * w + 8 * n, "flops": 15 * n * d}
    n = sum(_tensor_sizes(case))
    p, g = TYPES[case["type"]].itemsize, TYPES[case["grads"]].itemsize
    kept = p + 8 if case["master"] else 2 * p                  # the fp32 copy is read in place of the parameter
    moments = 16 if case["bits"] == 32 else 4 + 4 / BLOCK + 4     # in 8 bits: and the values that are returned
    return {"bytes": int(n * (kept + g + moments)), "flops": 16 * n}


def exact(case, seed):
    if case["kind"] == "adamw":
        return _exact_adamw(case, seed)
    s = _layer_norm_inputs(case, seed)
    x, w = s["x"].double(), s["weight"].double()
    if case["kind"] == "forward":
        var, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = (var + EPSILON) ** -0.5
        x -= mean.unsqueeze(1)
        x *= rstd.unsqueeze(1)
        x *= w
        x += s["bias"].double()
        return x, mean, rstd
    # the projections of the derivative off the constant row and off xhat
    x -= s["mean"].double().unsqueeze(1)
    x *= s["rstd"].double().unsqueeze(1)
    dy = s["dy"].double()
    dweight, dbias = torch.linalg.vecdot(x, dy, dim=0), dy.sum(dim=0)
    dy *= w
    along = torch.linalg.vecdot(x, dy, dim=1) / x.shape[1]
    dy -= dy.mean(dim=1, keepdim=True)
    dy.addcmul_(x, along.unsqueeze(1), value=-1.0)
    dy *= s["rstd"].double().unsqueeze(1)
    return dy, dweight, dbias


def _exact_code(a, share, binades, lowest):
    """Magnitudes on the grid of eighths of their binade, rounded down behind `share` of a step; E of each block by its largest."""
    f, e = torch.frexp(a.amax(dim=1, keepdim=True))
    top = torch.where(f > 0.9375, e, e - 1).double().clamp_min(-127.0 + lowest)
    least = torch.exp2(top - binades) * (1.125 if binades == 15 else 1.25)
    _, e = torch.frexp(a)
    step = torch.exp2(e.double() - 4.0)
    on_grid = torch.floor(a / step + share) * step
    on_grid = torch.minimum(torch.maximum(on_grid, least), 1.875 * torch.exp2(top))
    return on_grid, least


def _exact_adamw(case, seed):
    s = _adamw_inputs(case, seed)
    t, (b1, b2) = s["t"] + 1, BETAS
    g = s["grads"].double()
    if s["clip"] is not None:
        g *= s["clip"].double()
    m, v = torch.lerp(g, s["m"].double(), b1), torch.lerp(g.square(), s["v"].double(), b2)
    p = (s["master"] if case["master"] else s["p"]).double()
    p = p - LR * (case["decay"] * p + m / (1 - b1 ** t) / (v.div(1 - b2 ** t).sqrt() + ADAM_EPSILON))
    if case["bits"] == 8:
        n = p.numel()
        place = torch.arange(n, dtype=torch.int64, device="cuda")
        share = (((place * DITHER_INDEX + t * DITHER_STEP) % (1 << 32)) // (1 << 12)).double().div(1 << 20).view(-1, BLOCK)
        a = m.abs().view(-1, BLOCK)
        coded, least = _exact_code(a, share, 15, 16)
        coded = torch.where(a >= least, coded, torch.where(a > share * least, least, 0.0))
        m = coded.view(-1) * m.sign()
        r = v.sqrt().view(-1, BLOCK)
        coded, _ = _exact_code(r, share, 31, 32)
        v = torch.where(r > 0, coded, 0.0).square().view(-1)
    return [p, m, v] + ([p] if case["master"] else [])
