"""The operators at the two ends of a network that reads and predicts tokens, and in front of its optimizer.

Five kinds of case:

  lookup     ngsgd_embedding_forward: the rows of a table that tokens name, scaled
  gradient   ngsgd_embedding_backward: the table's gradient, from the derivative of those rows
  norm       ngsgd_grad_norm: the norm of all gradients as one vector, and the factor that brings it to a bound
  clip       ngsgd_grad_clip: the same, and the gradients times that factor, into other tensors
  loss       ngsgd_cross_entropy: the cross-entropy of each row of logits and the gradient of their sum

Tokens and labels follow a Zipf law, as words and speech states do; some are -1, the padding of a batch.  The tensors of a `norm` or
`clip` case lie in one flat buffer, each on a multiple of 256 elements; the elements between them are zero.
"""
import math

import torch

own = False                          # set by the program that measures: the plain forms, or the framework's calls

ZIPF = 1.1                           # exponent of the law of tokens and labels
SPACING = 256                        # elements: where tensors in a flat buffer start
SIZE = 1e-3                          # of the gradients
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16, "int32": torch.int32, "int64": torch.int64}


def listed():
    return [
        # the smallest call: the tokens of one step of a search with sixteen hypotheses
        dict(name="lookup_smallest", kind="lookup", tokens=16, vocabulary=5000, dim=512, pad=0, table="bf16", type="bf16", index="int64",
             padded=0.0, scale=1.0),
        # the largest: a batch of long sequences, an odd vocabulary, a table kept in 32 bits inside a wider buffer
        dict(name="lookup_large", kind="lookup", tokens=196613, vocabulary=50021, dim=4096, pad=8, table="fp32", type="bf16", index="int64",
             padded=0.06, scale=64.0),
        # a tiny network over characters
        dict(name="gradient_smallest", kind="gradient", tokens=64, vocabulary=50, dim=128, pad=0, table="fp32", type="fp32", index="int32",
             padded=0.0, scale=1.0),
        # odd sizes, rows without a common alignment
        dict(name="gradient_ragged", kind="gradient", tokens=20011, vocabulary=30011, dim=773, pad=0, table="bf16", type="bf16", index="int64",
             padded=0.1, scale=27.8),
        # the largest: a large batch over a large vocabulary, the gradient in 32 bits
        dict(name="gradient_large", kind="gradient", tokens=262144, vocabulary=131072, dim=2048, pad=0, table="fp32", type="bf16", index="int64",
             padded=0.03, scale=1.0),
        # the gradients of a tiny tanh network with layer norms
        dict(name="norm_smallest", kind="norm", tensors="network", input=40, hidden=128, layers=3, classes=50, type="fp32", ratio=0.5),
        # odd sizes, tensors of one element; the clipped gradients go to a buffer of their own
        dict(name="clip_ragged", kind="clip", tensors="mixed", count=61, largest=400009, type="fp16", ratio=0.7),
        # the largest: blocks of a wide network, in 16 bits
        dict(name="clip_large", kind="clip", tensors="blocks", width=4096, count=5, type="bf16", ratio=0.5),
        # the last layer of a tiny network
        dict(name="loss_smallest", kind="loss", rows=64, classes=50, pad=0, masked=0, type="fp32", index="int32", ignored=0.0, scale=1.0),
        # a minibatch of the speech-shaped network: 512 rows of 5000 in 32 bits
        dict(name="loss_speech", kind="loss", rows=512, classes=5000, pad=0, masked=0, type="fp32", index="int32", ignored=0.0, scale=1.0),
        # few rows of a large vocabulary, its last columns there for the product's sake only and masked
        dict(name="loss_few_rows", kind="loss", rows=24, classes=128256, pad=0, masked=219, type="bf16", index="int64", ignored=0.1, scale=0.05),
        # the largest: a batch of sequences over an odd vocabulary
        dict(name="loss_large", kind="loss", rows=12288, classes=100277, pad=3, masked=0, type="bf16", index="int64", ignored=0.05, scale=1e-4),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["lookup", "gradient", "gradient", "norm", "clip", "clip", "loss", "loss"])
    if kind in ("lookup", "gradient"):
        dim = _log(rng, 24, 8192)
        most = (1 << 29) // dim
        type_ = rng.choice(["fp32", "bf16", "bf16", "fp16"])
        return dict(kind=kind, tokens=_log(rng, 1, min(1 << 18, most)), vocabulary=_log(rng, 20, min(1 << 18, (1 << 28) // dim)), dim=dim,
                    pad=rng.choice([0, 0, 8, rng.randint(1, 40)]), table=rng.choice(["fp32", type_]), type=type_,
                    index=rng.choice(["int32", "int64"]), padded=rng.choice([0.0, rng.random() * 0.3]), scale=rng.choice([1.0, math.sqrt(dim)]))
    if kind == "loss":
        classes = _log(rng, 20, 262144)
        return dict(kind=kind, rows=_log(rng, 1, min(32768, (1 << 29) // classes)), classes=classes, pad=rng.choice([0, 0, 8, rng.randint(1, 40)]),
                    masked=rng.choice([0, rng.randint(0, classes // 10)]), type=rng.choice(["fp32", "bf16", "bf16", "fp16"]),
                    index=rng.choice(["int32", "int64"]), ignored=rng.choice([0.0, rng.random() * 0.5]), scale=rng.choice([1.0, 0.01]))
    case = dict(kind=kind, type=rng.choice(["fp32", "bf16", "fp16"]), ratio=rng.choice([0.2, 0.6, 3.0]))
    which = rng.choice(["network", "mixed", "blocks"])
    if which == "network":
        case.update(tensors=which, input=4 * _log(rng, 10, 110), hidden=_log(rng, 100, 2900), layers=rng.randint(2, 6), classes=_log(rng, 50, 6000))
    elif which == "mixed":
        case.update(tensors=which, count=rng.randint(1, 120), largest=_log(rng, 2, 400000))
    else:
        case.update(tensors=which, width=8 * _log(rng, 16, 256), count=rng.randint(1, 8))
    return case


# ---- inputs ------------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _law(n):
    """Share of each of n tokens or classes."""
    p = torch.arange(1, n + 1, dtype=torch.float64).pow(-ZIPF)
    return p / p.sum()


def _indices(g, count, n, left_out, kind):
    """`count` numbers below n by that law, a share of them -1."""
    border = _law(n).cumsum(0).cuda()
    u = torch.rand(count, generator=g, device="cuda", dtype=torch.float64)
    out = torch.searchsorted(border, u).clamp_max(n - 1)
    out[torch.randperm(count, generator=g, device="cuda")[:int(count * left_out)]] = -1
    return out.to(TYPES[kind])


def _rows(t, kind, pad):
    """In the given type, inside a wider buffer where the case says so."""
    wide = torch.zeros(t.shape[0], t.shape[1] + pad, dtype=kind, device="cuda")
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def _tensor_sizes(case):
    """Elements of each tensor."""
    if case["tensors"] == "network":      # weights with the bias in the last column; a gain and a bias behind each hidden layer
        dims = [case["input"]] + [case["hidden"]] * (case["layers"] - 1) + [case["classes"]]
        return [dims[l + 1] * (dims[l] + 1) for l in range(case["layers"])] + [case["hidden"]] * (2 * (case["layers"] - 1))
    if case["tensors"] == "mixed":        # from one element up, spread over the logarithm
        n, big = case["count"], case["largest"]
        return [int(round(big ** ((k + 1) / n))) for k in range(n)]
    w = case["width"]                     # blocks of a wide network: matrices, biases, the gain and bias of two layer norms
    return [w * w, w, w * w, w, w * w, w, w * w, w, 4 * w * w, 4 * w, 4 * w * w, w, w, w, w, w] * case["count"]


def _offsets(sizes):
    at, offsets = 0, []
    for n in sizes:
        offsets.append(at)
        at += -(-n // SPACING) * SPACING
    return offsets, at


def _inputs(case, seed):
    g = _gen(seed)
    if case["kind"] in ("lookup", "gradient"):
        n, v, d = case["tokens"], case["vocabulary"], case["dim"]
        s = dict(tokens=_indices(g, n, v, case["padded"], case["index"]))
        if case["kind"] == "lookup":
            s["table"] = _rows(0.05 * torch.randn(v, d, generator=g, device="cuda"), TYPES[case["table"]], case["pad"])
        else:
            s["dy"] = _rows(0.1 * torch.randn(n, d, generator=g, device="cuda"), TYPES[case["type"]], case["pad"])
        return s
    if case["kind"] == "loss":
        n, v = case["rows"], case["classes"]
        s = dict(labels=_indices(g, n, v - case["masked"], case["ignored"], case["index"]))
        x = torch.randn(n, v, generator=g, device="cuda").mul_(2.0)
        surer = 4.0 + 12.0 * torch.rand(n, generator=g, device="cuda")       # some rows are as good as decided
        x[torch.arange(n, device="cuda"), s["labels"].long().clamp_min(0)] += surer
        x[:, v - case["masked"]:] = -math.inf
        s["logits"] = _rows(x, TYPES[case["type"]], case["pad"])
        return s
    sizes = _tensor_sizes(case)
    offsets, total = _offsets(sizes)
    flat = torch.zeros(total, dtype=TYPES[case["type"]], device="cuda")
    grads = [flat[o:o + n] for o, n in zip(offsets, sizes)]
    for t in grads:
        t.copy_(SIZE * torch.randn(t.numel(), generator=g, device="cuda") * torch.rand(t.numel(), generator=g, device="cuda"))
    return dict(flat=flat, grads=grads, max_norm=case["ratio"] * SIZE * math.sqrt(sum(sizes) / 3.0))


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "clip":            # where the clipped gradients go
        s["clipped"] = torch.zeros_like(s["flat"])
        offsets, _ = _offsets(_tensor_sizes(case))
        s["clipped_list"] = [s["clipped"][o:o + t.numel()] for o, t in zip(offsets, s["grads"])]
    if own:                               # the object that a program makes once, with its workspace
        import paper_1410_7455_amd as ng
        if case["kind"] in ("lookup", "gradient"):
            s["op"] = ng.Embedding(case["tokens"], case["vocabulary"], case["dim"], scale=case["scale"])
        elif case["kind"] == "loss":
            s["op"] = ng.CrossEntropy(case["rows"], case["classes"])
        else:
            s["op"] = ng.GradientNorm(s["grads"])
    return s


def run(state):
    kind = state["case"]["kind"]
    if kind == "lookup":
        return _own_lookup(state) if own else _lookup(state)
    if kind == "gradient":
        return _own_gradient(state) if own else _gradient(state)
    if kind == "norm":
        return _own_norm(state) if own else _norm(state)
    if kind == "clip":
        return _own_clip(state) if own else _clip(state)
    return _own_loss(state) if own else _loss(state)


# ---- the framework's calls ----------------------------------------------------------------------------

def _own_lookup(s):
    return s["op"].forward(s["tokens"], s["table"], dtype=TYPES[s["case"]["type"]])


def _own_gradient(s):
    return s["op"].backward(s["dy"], s["tokens"], dtype=TYPES[s["case"]["table"]])


def _own_norm(s):
    return s["op"].norm(s["grads"], s["max_norm"])


def _own_clip(s):
    norm, factor = s["op"].clip(s["grads"], s["max_norm"], out=s["clipped_list"])
    return s["clipped"], norm, factor


def _own_loss(s):
    return s["op"].gradient(s["logits"], s["labels"], scale=s["case"]["scale"])


# ---- the plain forms ------------------------------------------------------------------------------------

def _lookup(s):
    t, v = s["tokens"], s["table"].shape[0]
    there = (t >= 0) & (t < v)
    y = s["table"][t.clamp(0, v - 1)].float() * s["case"]["scale"]
    return torch.where(there[:, None], y, 0.0).to(TYPES[s["case"]["type"]])


def _gradient(s):
    t, v = s["tokens"], s["case"]["vocabulary"]
    by_token, order = torch.sort(torch.where((t >= 0) & (t < v), t, v).long(), stable=True)      # padding goes last
    ends = torch.searchsorted(by_token, torch.arange(-1, v, device="cuda"), right=True)
    sums = torch.zeros(t.numel() + 1, s["case"]["dim"], dtype=torch.float64, device="cuda")      # in 64 bits: differences of long sums
    torch.cumsum(s["dy"][order].double(), 0, out=sums[1:])
    return ((sums[ends[1:]] - sums[ends[:-1]]) * s["case"]["scale"]).to(TYPES[s["case"]["table"]])


def _norm(s):
    g = s["flat"].float()
    norm = torch.sqrt((g * g).sum(dtype=torch.float64))
    factor = torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0)
    return norm.float().view(1), factor.float().view(1)


def _clip(s):
    norm, factor = _norm(s)
    return (s["flat"].float() * factor).to(s["flat"].dtype), norm, factor


def _loss(s):
    y = s["labels"].long()
    there = (y >= 0) & (y < s["case"]["classes"])
    at = torch.where(there, y, 0)[:, None]
    x = s["logits"].float()
    x = x - x.amax(1, keepdim=True)
    e = torch.exp(x)
    total = e.sum(1, keepdim=True)
    loss = torch.log(total) - torch.gather(x, 1, at)
    d = e / total
    d.scatter_add_(1, at, torch.full_like(total, -1.0))
    d = torch.where(there[:, None], d * s["case"]["scale"], 0.0)
    return torch.where(there, loss[:, 0], 0.0), d.to(s["logits"].dtype)


# ---- what a pass cannot do without, and the definitions in 64 bits --------------------------------------

def _distinct(case):
    """How many rows of the table the tokens are expected to name."""
    n = case["tokens"] - int(case["tokens"] * case["padded"])
    return float((1.0 - (1.0 - _law(case["vocabulary"])).pow(n)).sum())


def work(case):
    if case["kind"] in ("lookup", "gradient"):
        n, d = case["tokens"], case["dim"]
        there = n - int(n * case["padded"])
        t, w = TYPES[case["type"]].itemsize, TYPES[case["table"]].itemsize
        names = n * TYPES[case["index"]].itemsize
        if case["kind"] == "lookup":
            return {"bytes": int(names + _distinct(case) * d * w + n * d * t), "flops": there * d}
        return {"bytes": names + there * d * t + case["vocabulary"] * d * w, "flops": there * d}
    if case["kind"] == "loss":
        n, v = case["rows"], case["classes"]
        there = n - int(n * case["ignored"])
        t = TYPES[case["type"]].itemsize
        return {"bytes": n * TYPES[case["index"]].itemsize + there * v * t + n * v * t + 4 * n, "flops": 8 * there * v}
    n, t = sum(_tensor_sizes(case)), TYPES[case["type"]].itemsize
    return {"bytes": n * t * (2 if case["kind"] == "clip" else 1) + 8, "flops": n * (3 if case["kind"] == "clip" else 2)}


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "lookup":
        table = torch.cat([s["table"].double() * case["scale"], torch.zeros(1, case["dim"], dtype=torch.float64, device="cuda")])
        return torch.nn.functional.embedding(torch.where(s["tokens"] < 0, case["vocabulary"], s["tokens"].long()), table)
    if case["kind"] == "gradient":
        order = torch.argsort(s["tokens"], stable=True)
        order = order[int((s["tokens"] < 0).sum()):]
        out = torch.zeros(case["vocabulary"], case["dim"], dtype=torch.float64, device="cuda")
        which, counts = torch.unique_consecutive(s["tokens"][order].long(), return_counts=True)
        out[which] = torch.segment_reduce(s["dy"][order].double(), "sum", lengths=counts, axis=0) * case["scale"]
        return out
    if case["kind"] == "loss":
        y = torch.where(s["labels"] < 0, -100, s["labels"].long())
        logp = torch.log_softmax(s["logits"].double(), dim=1)
        loss = torch.nn.functional.nll_loss(logp, y, reduction="none", ignore_index=-100)
        d = logp.exp_()
        rows = torch.nonzero(y >= 0)[:, 0]
        d[rows, y[rows]] -= 1.0
        d[y < 0] = 0.0
        return loss, d.mul_(case["scale"])
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(t.double()) for t in s["grads"]]))
    factor = (s["max_norm"] / norm).clamp_max(1.0)
    if case["kind"] == "norm":
        return norm.view(1), factor.view(1)
    return s["flat"].double() * factor, norm.view(1), factor.view(1)
