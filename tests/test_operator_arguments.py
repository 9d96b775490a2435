"""CPU-side checks of layer norm's and AdamW's entry points: sizes, refusals.  Every call here is refused before any device work."""
import ctypes
from ctypes import byref, c_double, c_float, c_int32, c_int64, c_size_t, c_void_p

import pytest

import paper_1410_7455_amd as ng

F32, BF16, F16 = ng.NGSGD_FLOAT32, ng.NGSGD_BFLOAT16, ng.NGSGD_FLOAT16
A = 1 << 20          # an address that is never used: aligned, not NULL


@pytest.fixture(scope="module")
def lib():
    return ng.load_library()


def forward(lib, x=A, ldx=8, type=F32, w=A, b=A, wtype=F32, N=4, D=8, eps=1e-5, y=A, ldy=8, mean=A, rstd=A):
    return lib.ngsgd_layernorm_forward(x, ldx, type, w, b, wtype, N, D, eps, y, ldy, mean, rstd, None)


@pytest.mark.parametrize("bad", [
    dict(type=3), dict(type=-1), dict(wtype=3), dict(type=BF16, wtype=F16), dict(type=F32, wtype=BF16), dict(N=-1), dict(D=0), dict(D=-4), dict(D=(1 << 25) + 1, ldx=1 << 26, ldy=1 << 26),
    dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf")), dict(x=None), dict(y=None), dict(ldx=7), dict(ldy=7), dict(ldx=-8),
    dict(ldx=1 << 62), dict(x=A + 2), dict(y=A + 1), dict(w=A + 2), dict(b=A + 1), dict(mean=A + 2), dict(rstd=A + 1),
    dict(type=BF16, x=A + 1), dict(type=F16, wtype=F16, w=A + 1)])
def test_layernorm_forward_refuses(lib, bad):
    assert forward(lib, **bad) == ng.NGSGD_EINVAL


def test_layernorm_forward_of_no_rows(lib):
    assert forward(lib, x=None, y=None, N=0) == ng.NGSGD_OK


def backward(lib, dy=A, lddy=8, x=A, ldx=8, type=F32, w=A, wtype=F32, mean=A, rstd=A, N=4, D=8, dx=A, lddx=8, dw=A, db=A, ws=A, nbytes=1 << 30):
    return lib.ngsgd_layernorm_backward(dy, lddy, x, ldx, type, w, wtype, mean, rstd, N, D, dx, lddx, dw, db, ws, nbytes, None)


@pytest.mark.parametrize("bad", [
    dict(type=3), dict(wtype=-1), dict(type=F16, wtype=BF16), dict(N=-1), dict(D=0), dict(dy=None), dict(x=None), dict(mean=None),
    dict(rstd=None), dict(lddy=7), dict(ldx=7), dict(lddx=7), dict(dx=None, dw=None, db=None), dict(ws=None), dict(ws=A + 128), dict(dx=A + 2),
    dict(dw=A + 2), dict(db=A + 1), dict(w=A + 1), dict(mean=A + 2), dict(dy=A + 1)])
def test_layernorm_backward_refuses(lib, bad):
    assert backward(lib, **bad) == ng.NGSGD_EINVAL


def test_layernorm_workspace(lib):
    n, last = c_size_t(0), 0
    for rows in list(range(0, 70)) + [100, 1000, 4001, 10 ** 5, 10 ** 9]:
        assert lib.ngsgd_layernorm_workspace_bytes(rows, 1000, byref(n)) == 0
        assert n.value % 256 == 0 and n.value >= max(last, 2 * 1000 * 4)     # fewer rows never need more
        last = n.value
        assert backward(lib, N=max(rows, 1), D=1000, ldx=1000, lddy=1000, lddx=1000, nbytes=2 * 1000 * 4 - 1) == ng.NGSGD_ENOMEM
    assert last < 64 << 20
    for dim in (16384, 16385, 40000, 10 ** 6, 1 << 25):      # rows of any width: no more than 64 MiB, or eight sums of them
        last = 0
        for rows in (0, 1, 100, 10 ** 4, 10 ** 9):
            assert lib.ngsgd_layernorm_workspace_bytes(rows, dim, byref(n)) == 0 and last <= n.value <= max(64 << 20, 64 * dim) + 512
            last = n.value
    for rows, dim in ((-1, 8), (4, 0), (4, (1 << 25) + 1)):
        assert lib.ngsgd_layernorm_workspace_bytes(rows, dim, byref(n)) == ng.NGSGD_EINVAL
    assert lib.ngsgd_layernorm_workspace_bytes(4, 8, None) == ng.NGSGD_EINVAL


def config(addresses=(A, 2 * A), sizes=(5, 7), decay=None, rate=None, ptype=F32, gtype=F32, bits=32, master=0, betas=(0.9, 0.999), eps=1e-8, n=None):
    n = len(sizes) if n is None else n
    k = max(1, len(sizes))
    keep = ((c_void_p * k)(*addresses), (c_int64 * k)(*sizes), None if decay is None else (c_float * k)(*decay),
            None if rate is None else (c_float * k)(*rate))
    cfg = ng.ngsgd_adamw_config(n, keep[0], keep[1], keep[2], keep[3], ptype, gtype, bits, master, betas[0], betas[1], eps)
    cfg._keep = keep
    return cfg


BAD = [
    dict(sizes=(), addresses=()), dict(n=0), dict(n=-1), dict(sizes=(5, -1)), dict(sizes=(5, 1 << 60)), dict(sizes=(5, 1 << 36)), dict(addresses=(A, None)), dict(addresses=(A, A)),
    dict(addresses=(A, A + 16)), dict(addresses=(A + 4 * 5 - 4, A)), dict(addresses=(A + 2, 2 * A)), dict(ptype=3), dict(gtype=-1),
    dict(ptype=BF16, gtype=F16), dict(ptype=F16, gtype=BF16), dict(bits=16), dict(bits=0), dict(master=1), dict(master=2, ptype=BF16, gtype=BF16),
    dict(betas=(1.0, 0.999)), dict(betas=(-0.1, 0.999)), dict(betas=(0.9, 1.0)), dict(betas=(float("nan"), 0.999)), dict(eps=-1.0),
    dict(eps=float("inf")), dict(eps=float("nan")), dict(eps=1e-39), dict(decay=(0.1, float("nan"))), dict(rate=(float("inf"), 1.0))]


@pytest.mark.parametrize("bad", BAD)
def test_adamw_refuses(lib, bad):
    n, h = c_size_t(0), c_void_p(0)
    cfg = config(**bad)
    assert lib.ngsgd_adamw_workspace_bytes(byref(cfg), byref(n)) == ng.NGSGD_EINVAL
    assert lib.ngsgd_adamw_create(byref(cfg), A, 1 << 40, byref(h)) == ng.NGSGD_EINVAL and not h.value


def test_adamw_workspace(lib):
    def need(**kw):
        n = c_size_t(0)
        assert lib.ngsgd_adamw_workspace_bytes(byref(config(**kw)), byref(n)) == 0
        return n.value
    big = dict(sizes=(100000, 1), addresses=(A, 4 * A))
    elements = 100096 + 256
    assert 8 * elements <= need(**big) <= 8 * elements + 4096
    assert 2 * elements <= need(bits=8, **big) <= 2 * elements + 4 * elements // 256 + 4096
    assert 12 * elements <= need(ptype=BF16, gtype=BF16, master=1, **big) <= 12 * elements + 4096
    assert need(sizes=(0, 0), addresses=(None, None)) > 0
    # neighbours in memory are no overlap
    assert need(addresses=(A, A + 20)) > 0
    h = c_void_p(0)
    cfg = config()
    assert lib.ngsgd_adamw_workspace_bytes(byref(cfg), None) == ng.NGSGD_EINVAL
    assert lib.ngsgd_adamw_workspace_bytes(None, byref(c_size_t(0))) == ng.NGSGD_EINVAL
    assert lib.ngsgd_adamw_create(byref(cfg), None, 1 << 40, byref(h)) == ng.NGSGD_EINVAL
    assert lib.ngsgd_adamw_create(byref(cfg), A + 64, 1 << 40, byref(h)) == ng.NGSGD_EINVAL
    assert lib.ngsgd_adamw_create(byref(cfg), A, 16, byref(h)) == ng.NGSGD_ENOMEM
    assert lib.ngsgd_adamw_create(byref(cfg), A, 1 << 40, None) == ng.NGSGD_EINVAL


def test_adamw_calls_without_a_handle(lib):
    assert lib.ngsgd_adamw_destroy(None) == ng.NGSGD_EINVAL
    assert lib.ngsgd_adamw_step(None, (c_void_p * 1)(), 0.1, None, 1.0, None, None) == ng.NGSGD_EINVAL
    assert lib.ngsgd_adamw_arrays(None, None, None, None, None) == ng.NGSGD_EINVAL
    assert lib.ngsgd_adamw_get_state(None, None, None, F32, None, None) == ng.NGSGD_EINVAL
    assert lib.ngsgd_adamw_set_state(None, None, None, None, 0, None) == ng.NGSGD_EINVAL


def test_config_structure_matches_the_header():
    """The offsets that a C compiler gives the structure on this machine (natural alignment)."""
    cfg = ng.ngsgd_adamw_config
    assert [getattr(cfg, f).offset for f, _ in cfg._fields_] == [0, 8, 16, 24, 32, 40, 44, 48, 52, 56, 64, 72]
    assert ctypes.sizeof(cfg) == 80 and ctypes.sizeof(c_double) == 8 and ctypes.sizeof(c_int32) == 4


def test_binding_refuses_tensors_off_the_device():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError):
        ng.AdamW([torch.zeros(4)])
    with pytest.raises(ValueError):
        ng.AdamW([])
    ln = ng.LayerNorm.__new__(ng.LayerNorm)
    ln.max_rows, ln.dim, ln.epsilon, ln.device = 4, 8, 1e-5, torch.device("cuda", 0)
    with pytest.raises(ValueError):
        ln._rows(torch.zeros(2, 8), "x")
    with pytest.raises(ValueError):
        ng._check_dense(torch.zeros(8), "weight", ln.device)
    with pytest.raises(ValueError):
        ng._type_of(torch.float64)


def test_binding_refuses_another_current_device(monkeypatch):
    torch = pytest.importorskip("torch")
    ng.load_library()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    ng._current_device(torch.device("cuda", 1))
    ln = ng.LayerNorm.__new__(ng.LayerNorm)
    ln.device = torch.device("cuda", 0)
    opt = ng.AdamW.__new__(ng.AdamW)
    opt.device, opt.handle, opt.grad_dtype, opt.sizes, opt._m = ln.device, None, torch.float32, [1], None
    for call in (lambda: ln.forward(None), lambda: ln.backward(None, None, None, None), lambda: opt.step([None], 0.1), lambda: opt.state(),
                 lambda: opt.set_state(None, None, 0), lambda: opt.steps()):
        with pytest.raises(ValueError):
            call()


def test_networks_with_layer_norm_or_adamw(lib):
    from test_library_abi import make_cfg
    n = c_size_t(0)

    def need(nonlin, **kw):
        rc = lib.ngsgd_workspace_bytes(byref(make_cfg([40, 128, 50], [nonlin], rank_in=4, rank_out=8, max_batch=64, **kw)), byref(n))
        return n.value if rc == 0 else rc

    plain = need(ng.NGSGD_TANH)
    normed = need(ng.NGSGD_TANH | ng.NGSGD_LAYERNORM)
    # the nonlinearity's output, parameters, gradients and two moments
    assert normed >= plain + 64 * 128 * 4 + 5 * 2 * 128 * 4
    params = 128 * 64 + 50 * 160                       # padded rows
    by32, by8 = (need(ng.NGSGD_TANH, method=m) for m in (ng.NGSGD_METHOD_ADAMW, ng.NGSGD_METHOD_ADAMW8))
    assert by32 - by8 == pytest.approx(6 * params, abs=2048)
    assert need(ng.NGSGD_PNORM | ng.NGSGD_LAYERNORM, pnorm_group=4) > 0
    for nonlin, kw in ((ng.NGSGD_LAYERNORM + 2, {}), (2 * ng.NGSGD_LAYERNORM, {}), (-1, {}), (ng.NGSGD_TANH, dict(method=4)),
                       (ng.NGSGD_TANH, dict(method=ng.NGSGD_METHOD_ADAMW, max_change_per_sample=0.1)),
                       (ng.NGSGD_PNORM | ng.NGSGD_LAYERNORM, dict(pnorm_group=5))):
        assert need(nonlin, **kw) == ng.NGSGD_EINVAL
    huge = make_cfg([4, 2 ** 31 - 65, 2 ** 10], [ng.NGSGD_TANH], max_batch=1, method=ng.NGSGD_METHOD_ADAMW)
    assert lib.ngsgd_workspace_bytes(byref(huge), byref(n)) == ng.NGSGD_EINVAL
    for call in (lambda: lib.ngsgd_get_norm(None, 0, None, None, None), lambda: lib.ngsgd_set_norm(None, 0, None, None, None),
                 lambda: lib.ngsgd_last_norm_gradient(None, 0, None, None, None), lambda: lib.ngsgd_set_adamw(None, 1.0, 0.9, 0.999, 1e-8, 0.0)):
        assert call() == ng.NGSGD_EINVAL


def test_layernorm_workspace_of_any_count(lib):
    """Up to the largest count that its type holds: never less than for fewer rows."""
    n = c_size_t(0)
    for dim in (5, 200, 1000, 5000, 16384, 20000):
        last = 0
        for rows in (10 ** 9, 2 ** 62, 2 ** 63 - 16, 2 ** 63 - 2, 2 ** 63 - 1):
            assert lib.ngsgd_layernorm_workspace_bytes(rows, dim, byref(n)) == 0 and n.value >= last
            last = n.value
