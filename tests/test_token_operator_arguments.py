"""CPU-side checks of the embedding's, the cross-entropy's and the gradient norm's entry points: sizes, refusals.  Every call here is refused,
or has nothing to do, before any device work."""
import sys
from ctypes import byref, c_int64, c_size_t, c_void_p

import pytest

import paper_1410_7455_amd as ng

F32, BF16, F16, I32, I64 = ng.NGSGD_FLOAT32, ng.NGSGD_BFLOAT16, ng.NGSGD_FLOAT16, ng.NGSGD_INT32, ng.NGSGD_INT64
A = 1 << 20          # an address that is never used: aligned, not NULL
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def lib():
    return ng.load_library()


def lookup(lib, tokens=A, index=I32, N=4, table=A, ldt=8, ttype=F32, V=10, D=8, scale=1.0, y=A, ldy=8, type=F32):
    return lib.ngsgd_embedding_forward(tokens, index, N, table, ldt, ttype, V, D, scale, y, ldy, type, None)


@pytest.mark.parametrize("bad", [
    dict(index=F32), dict(index=5), dict(index=-1), dict(type=I32), dict(type=-1), dict(ttype=3), dict(type=BF16, ttype=F16), dict(type=F32, ttype=BF16),
    dict(N=-1), dict(N=(1 << 30) + 1), dict(V=0), dict(V=-3), dict(V=(1 << 30) + 1), dict(D=0), dict(D=-1), dict(D=(1 << 25) + 1, ldt=1 << 26, ldy=1 << 26),
    dict(scale=INF), dict(scale=NAN), dict(tokens=None), dict(table=None), dict(y=None), dict(tokens=A + 2), dict(index=I64, tokens=A + 4),
    dict(table=A + 2), dict(y=A + 1), dict(type=BF16, ttype=BF16, table=A + 1), dict(ldt=7), dict(ldy=7), dict(ldt=-8), dict(ldy=1 << 62)])
def test_embedding_forward_refuses(lib, bad):
    assert lookup(lib, **bad) == ng.NGSGD_EINVAL


def test_embedding_forward_of_no_tokens(lib):
    assert lookup(lib, tokens=None, table=None, y=None, N=0) == ng.NGSGD_OK


def gather(lib, dy=A, lddy=8, type=F32, tokens=A, index=I32, N=4, V=10, D=8, scale=1.0, dt=A, lddt=8, ttype=F32, acc=0, ws=A, nbytes=1 << 40):
    return lib.ngsgd_embedding_backward(dy, lddy, type, tokens, index, N, V, D, scale, dt, lddt, ttype, acc, ws, nbytes, None)


@pytest.mark.parametrize("bad", [
    dict(index=F32), dict(type=I64), dict(ttype=-1), dict(type=F16, ttype=BF16), dict(type=F32, ttype=F16), dict(N=-1), dict(N=(1 << 30) + 1), dict(V=0),
    dict(V=(1 << 30) + 1), dict(D=0), dict(D=(1 << 25) + 1, lddy=1 << 26, lddt=1 << 26), dict(scale=INF), dict(scale=NAN), dict(acc=2), dict(acc=-1),
    dict(dy=None), dict(tokens=None), dict(dt=None), dict(dy=A + 2), dict(tokens=A + 1), dict(index=I64, tokens=A + 4), dict(dt=A + 2), dict(lddy=7),
    dict(lddt=7), dict(lddt=-1), dict(lddy=1 << 62), dict(ws=None), dict(ws=A + 128)])
def test_embedding_backward_refuses(lib, bad):
    assert gather(lib, **bad) == ng.NGSGD_EINVAL


def test_embedding_workspace(lib):
    n, sizes = c_size_t(0), []
    for tokens in [0, 1, 2, 63, 64, 65, 100, 1000, 4095, 4096, 4097, 8192, 8193, 10 ** 5, 10 ** 6, 10 ** 7, 1 << 30]:
        assert lib.ngsgd_embedding_workspace_bytes(tokens, 50000, 1000, byref(n)) == 0 and n.value % 256 == 0
        sizes.append(n.value)
        if n.value > 0:
            assert gather(lib, N=tokens, V=50000, D=1000, lddy=1000, lddt=1000, nbytes=n.value - 1) == ng.NGSGD_ENOMEM
    assert sizes == sorted(sizes)                     # fewer tokens never need more
    for tokens, vocabulary, dim in ((-1, 8, 8), ((1 << 30) + 1, 8, 8), (4, 0, 8), (4, (1 << 30) + 1, 8), (4, 8, 0), (4, 8, (1 << 25) + 1)):
        assert lib.ngsgd_embedding_workspace_bytes(tokens, vocabulary, dim, byref(n)) == ng.NGSGD_EINVAL
    assert lib.ngsgd_embedding_workspace_bytes(4, 8, 8, None) == ng.NGSGD_EINVAL


def loss(lib, x=A, ld=8, type=F32, labels=A, index=I32, N=4, V=8, out=A, scale=1.0, dev_scale=None, d=A, ldd=8, ws=A, nbytes=1 << 40):
    return lib.ngsgd_cross_entropy(x, ld, type, labels, index, N, V, out, scale, dev_scale, d, ldd, ws, nbytes, None)


@pytest.mark.parametrize("bad", [
    dict(type=I32), dict(type=-1), dict(index=F32), dict(index=5), dict(N=-1), dict(N=(1 << 30) + 1), dict(V=0), dict(V=(1 << 29) + 1, ld=1 << 31, ldd=1 << 31),
    dict(x=None), dict(labels=None), dict(out=None, d=None), dict(x=A + 2), dict(type=BF16, x=A + 1), dict(labels=A + 2), dict(index=I64, labels=A + 4),
    dict(out=A + 2), dict(dev_scale=A + 1), dict(d=2 * A + 2), dict(ld=7), dict(ldd=7, d=2 * A), dict(ld=-1), dict(ldd=1 << 62), dict(ldd=9), dict(ws=None),
    dict(ws=A + 64)])
def test_cross_entropy_refuses(lib, bad):
    assert loss(lib, **bad) == ng.NGSGD_EINVAL


def test_cross_entropy_of_no_rows(lib):
    assert loss(lib, x=None, labels=None, out=None, d=None, ws=None, N=0) == ng.NGSGD_OK


def test_cross_entropy_workspace(lib):
    n = c_size_t(0)
    for classes in (1, 2, 100, 5000, 32768, 65537, 131072, 262144, 10 ** 6, 1 << 29):
        sizes = []
        for rows in (0, 1, 2, 15, 16, 17, 63, 64, 255, 256, 257, 1000, 10 ** 5, 10 ** 7, 1 << 30):
            assert lib.ngsgd_cross_entropy_workspace_bytes(rows, classes, byref(n)) == 0 and n.value % 256 == 0
            sizes.append(n.value)
            if rows > 0 and n.value > 0 and rows * classes < 1 << 56:
                assert loss(lib, N=rows, V=classes, ld=classes, ldd=classes, nbytes=n.value - 1) == ng.NGSGD_ENOMEM
        assert sizes == sorted(sizes)                 # fewer rows never need more
    for rows, classes in ((-1, 8), ((1 << 30) + 1, 8), (4, 0), (4, -1), (4, (1 << 29) + 1)):
        assert lib.ngsgd_cross_entropy_workspace_bytes(rows, classes, byref(n)) == ng.NGSGD_EINVAL
    assert lib.ngsgd_cross_entropy_workspace_bytes(4, 8, None) == ng.NGSGD_EINVAL


def norm(lib, sizes=(5, 7), grads=(A, 2 * A), type=F32, bound=1.0, out=None, clip=False, norm_out=A, factor=A, ws=A, nbytes=1 << 40, n=None):
    k = max(1, len(sizes))
    s, g = (c_int64 * k)(*sizes), (c_void_p * k)(*grads)
    n = len(sizes) if n is None else n
    if clip:
        return lib.ngsgd_grad_clip(n, s, g, type, bound, None if out is None else (c_void_p * k)(*out), norm_out, factor, ws, nbytes, None)
    return lib.ngsgd_grad_norm(n, s, g, type, bound, norm_out, factor, ws, nbytes, None)


BAD = [dict(sizes=(), grads=()), dict(n=0), dict(n=-1), dict(n=(1 << 20) + 1), dict(sizes=(5, -1)), dict(sizes=(5, (1 << 40) + 1)), dict(type=I32), dict(type=-1), dict(grads=(A, A + 2)),
       dict(type=BF16, grads=(A + 1, A)), dict(bound=-1.0), dict(bound=NAN), dict(norm_out=A + 2), dict(factor=A + 1), dict(ws=None), dict(ws=A + 8)]


@pytest.mark.parametrize("clip", [False, True])
@pytest.mark.parametrize("bad", BAD)
def test_grad_norm_refuses(lib, bad, clip):
    assert norm(lib, clip=clip, **bad) == ng.NGSGD_EINVAL


@pytest.mark.parametrize("bad", [dict(out=(A, None)), dict(out=(A, A + 2)), dict(out=(None, 2 * A)), dict(type=F16, out=(A + 1, 2 * A))])
def test_grad_clip_refuses(lib, bad):
    assert norm(lib, clip=True, **bad) == ng.NGSGD_EINVAL


@pytest.mark.parametrize("bad", [
    dict(grads=(A, A)), dict(grads=(A, A + 16)), dict(grads=(A + 24, A)), dict(out=(3 * A, 3 * A)), dict(out=(3 * A, 3 * A + 16)), dict(out=(2 * A, A)),
    dict(out=(A, A)), dict(out=(A + 4, 2 * A)), dict(out=(2 * A + 24, 2 * A)), dict(out=(3 * A, 2 * A - 4)), dict(sizes=(5, 0, 9), grads=(A, A, A + 12)),
    dict(sizes=(100, 100, 100), grads=(A, A, A), out=(2 * A, 3 * A, A))])
def test_grad_clip_refuses_shared_memory(lib, bad):
    """Refused, while everything else about the call is right: with a workspace that is too small the same call is refused for that."""
    assert norm(lib, clip=True, **bad) == ng.NGSGD_EINVAL
    assert norm(lib, clip=True, nbytes=16, **bad) == ng.NGSGD_ENOMEM


def test_grad_norm_without_arrays(lib):
    s, g = (c_int64 * 2)(5, 7), (c_void_p * 2)(A, A)
    assert lib.ngsgd_grad_norm(2, None, g, F32, 1.0, None, None, A, 1 << 30, None) == ng.NGSGD_EINVAL
    assert lib.ngsgd_grad_norm(2, s, None, F32, 1.0, None, None, A, 1 << 30, None) == ng.NGSGD_EINVAL
    assert lib.ngsgd_grad_clip(2, s, None, F32, 1.0, None, None, None, A, 1 << 30, None) == ng.NGSGD_EINVAL


def test_grad_norm_workspace(lib):
    n, last = c_size_t(0), 0
    for tensors in (1, 2, 127, 128, 129, 448, 449, 1000, 1 << 20):
        assert lib.ngsgd_grad_norm_workspace_bytes(tensors, byref(n)) == 0 and n.value % 256 == 0 and n.value >= max(256, last)
        last = n.value
        assert norm(lib, sizes=(5,) * min(tensors, 1000), grads=(A,) * min(tensors, 1000), nbytes=255) == ng.NGSGD_ENOMEM
    for tensors in (0, -1, (1 << 20) + 1):
        assert lib.ngsgd_grad_norm_workspace_bytes(tensors, byref(n)) == ng.NGSGD_EINVAL
    assert lib.ngsgd_grad_norm_workspace_bytes(1, None) == ng.NGSGD_EINVAL


def made(torch, kind, **fields):
    """An object of the binding without device memory."""
    op = kind.__new__(kind)
    op.device = torch.device("cuda", 0)
    for name, value in fields.items():
        setattr(op, name, value)
    return op


def test_binding_refuses_tensors_off_the_device(monkeypatch):
    torch = pytest.importorskip("torch")
    ng.load_library()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError):
        ng.GradientNorm([torch.zeros(4)])
    with pytest.raises(ValueError):
        ng.GradientNorm([])
    e = made(torch, ng.Embedding, max_tokens=4, vocabulary=8, dim=8, scale=1.0)
    c = made(torch, ng.CrossEntropy, max_rows=4, classes=8)
    g = made(torch, ng.GradientNorm, sizes=[4], grad_dtype=torch.float32, _sizes=(4).to_bytes(8, "little"), _like=torch.empty(0))
    tokens, x = torch.zeros(4, dtype=torch.int32), torch.zeros(4, 8)
    for call in (lambda: e.forward(tokens, x), lambda: e.backward(x, tokens), lambda: c.forward(x, tokens), lambda: c.gradient(x, tokens),
                 lambda: g.norm([torch.zeros(4)]), lambda: g.clip([torch.zeros(4)], 1.0), lambda: g.norm([])):
        with pytest.raises(ValueError):
            call()


def test_binding_refuses_another_current_device(monkeypatch):
    torch = pytest.importorskip("torch")
    ng.load_library()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    e, c, g = (made(torch, kind) for kind in (ng.Embedding, ng.CrossEntropy, ng.GradientNorm))
    for call in (lambda: e.forward(None, None), lambda: e.backward(None, None), lambda: c.forward(None, None), lambda: c.gradient(None, None),
                 lambda: g.norm([None]), lambda: g.clip([None], 1.0)):
        with pytest.raises(ValueError):
            call()


def test_missing_helper_fails_loudly(monkeypatch):
    pytest.importorskip("torch")
    ng.load_library()
    monkeypatch.setattr(ng, "_lib", None)
    monkeypatch.delattr(ng, "_tensors")
    monkeypatch.setitem(sys.modules, ng.__name__ + "._tensors", None)
    with pytest.raises(ImportError, match="_tensors.so"):
        ng.load_library()


def test_addresses_of_many_tensors():
    """What the helper takes, and what it does not (the binding then says why); it looks at the device, so on a CPU only what has no address is taken."""
    torch = pytest.importorskip("torch")
    ng.load_library()
    like, size = torch.empty(0), lambda *n: b"".join(k.to_bytes(8, "little") for k in n)
    assert ng._tensors.addresses([], b"", like, 0) == b""
    assert ng._tensors.addresses([None, torch.zeros(0)], size(5, 0), like, 0) == bytes(16)
    assert ng._tensors.addresses((None,), size(5), like, 0) == bytes(8)
    for tensors, sizes in (([torch.zeros(5)], size(5)), ([None], size(5, 5)), ([None, None], size(5)), ([3], size(5)), (["x"], size(1))):
        assert ng._tensors.addresses(tensors, sizes, like, 0) is None
    for bad in ((5, size(5), like, 0), ([None], [5], like, 0), ([None], size(5), torch.float32, 0), ([None], size(5), like, "0"), ([None], size(5), like)):
        with pytest.raises(TypeError):
            ng._tensors.addresses(*bad)


@pytest.mark.parametrize("there", [False, True], ids=["missing", "of another torch"])
def test_the_helper_is_needed_where_it_is_used(monkeypatch, there):
    """Without it (built where there was no torch), or with one that does not load, everything but the norm of many gradients works."""
    torch = pytest.importorskip("torch")
    ng.load_library()
    monkeypatch.setattr(ng, "_lib", None)
    monkeypatch.delattr(ng, "_tensors")
    monkeypatch.setitem(sys.modules, ng.__name__ + "._tensors", None)
    if not there:
        monkeypatch.setattr(ng, "HELPER_PATH", ng.HELPER_PATH + ".none")
        assert ng.load_library().ngsgd_version() >= 100
        monkeypatch.setattr(ng, "_lib", None)
    monkeypatch.setattr(torch, "empty", lambda *_, **__: made(torch, Buffer))
    monkeypatch.setattr(ng, "_raw_stream", lambda *_: 0)
    for make in (lambda: ng.Embedding(4, 10, 8), lambda: ng.CrossEntropy(4, 10), lambda: ng.LayerNorm(4, 8)):
        assert make().lib.ngsgd_version() >= 100
    with pytest.raises(ImportError, match="_tensors.so"):
        ng.GradientNorm([torch.zeros(4)])


class Buffer:
    """Stands for device memory."""


def test_clip_needs_no_output_for_what_does_not_count(monkeypatch):
    """out has to have a tensor only where a gradient with elements is."""
    torch = pytest.importorskip("torch")
    ng.load_library()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(ng, "_raw_stream", lambda *_: None)
    calls = []
    taken = type("Library", (), {"ngsgd_grad_clip": lambda self, *a: calls.append(a) or ng.NGSGD_OK})()
    some = torch.zeros(1)
    g = made(torch, ng.GradientNorm, lib=taken, sizes=[0, 5], grad_dtype=torch.float32, _sizes=bytes(8) + (5).to_bytes(8, "little"), _like=torch.empty(0),
             type=F32, workspace=some, workspace_bytes=4, _home=None, _results=lambda *_: (some, some))
    for grads, out in (([torch.zeros(0), None], [None, None]), ([torch.zeros(0), None], [torch.zeros(0), None]), ([None, None], [None, None])):
        g.clip(grads, 1.0, out=out)
    assert len(calls) == 3 and all(a[2] == a[5] == bytes(16) for a in calls)
    for grads, out in (([None, torch.zeros(5)], [None, None]), ([None, None], [None]), ([None, None], [None] * 3)):
        with pytest.raises(ValueError, match="out has no tensor"):
            g.clip(grads, 1.0, out=out)
