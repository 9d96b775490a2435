"""MI355X-native NG-SGD minibatch step (online natural-gradient SGD, arXiv 1410.7455).

Thin ctypes binding over the C ABI of ``libngsgd.so`` (declared in ``include/ngsgd.h``).
Every step of the method runs in the library's HIP kernels; this module only marshals
arguments.  PyTorch supplies device memory and streams.

The shared library is built in-tree by ``paper_1410_7455_amd.build.build()``; importing the
binding without it raises, there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from contextlib import nullcontext
from ctypes import POINTER, byref, c_char_p, c_double, c_float, c_int, c_int32, c_int64, c_size_t, c_void_p

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libngsgd.so")

NGSGD_OK = 0
NGSGD_EINVAL = -1
NGSGD_ENOMEM = -2
NGSGD_EHIP = -3
NGSGD_TANH = 0
NGSGD_PNORM = 1
NGSGD_LAYERNORM = 16
NGSGD_FLOAT32 = 0
NGSGD_BFLOAT16 = 1
NGSGD_FLOAT16 = 2
NGSGD_SIDE_INPUT = 0
NGSGD_SIDE_OUTPUT = 1
NGSGD_MAX_RANK = 96
NGSGD_MAX_LAYERS = 16
NGSGD_METHOD_ONLINE = 0
NGSGD_METHOD_SIMPLE = 1
NGSGD_METHOD_ADAMW = 2
NGSGD_METHOD_ADAMW8 = 3


class NgsgdError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = _lib.ngsgd_strerror(code).decode() if _lib is not None else str(code)
        extra = f" (hipError {_lib.ngsgd_last_hip_error()})" if _lib is not None and code == NGSGD_EHIP else ""
        super().__init__(f"{where}: {msg}{extra}")


class ngsgd_config(ctypes.Structure):
    _fields_ = [
        ("n_layers", c_int32), ("dims", POINTER(c_int32)), ("nonlin", POINTER(c_int32)),
        ("pnorm_group", c_int32), ("max_batch", c_int32), ("rank_in", c_int32), ("rank_out", c_int32),
        ("alpha", c_float), ("num_samples_history", c_float), ("epsilon", c_float),
        ("update_period", c_int32), ("always_update_first", c_int32), ("renorm", c_int32),
        ("max_change_per_sample", c_float), ("method", c_int32), ("simple_epsilon", c_float),
        ("side_streams", c_int32),
    ]


class ngsgd_adamw_config(ctypes.Structure):
    _fields_ = [
        ("n_tensors", c_int32), ("dev_params", POINTER(c_void_p)), ("sizes", POINTER(c_int64)),
        ("weight_decay", POINTER(c_float)), ("rate", POINTER(c_float)), ("param_type", c_int32), ("grad_type", c_int32),
        ("state_bits", c_int32), ("master", c_int32), ("beta1", c_double), ("beta2", c_double), ("epsilon", c_float),
    ]


# name -> (restype, argtypes); one entry per symbol declared in include/ngsgd.h
_SIGNATURES = {
    "ngsgd_precond_workspace_bytes": (c_int, [c_int32, c_int32, c_int32, POINTER(c_size_t)]),
    "ngsgd_precond_create": (c_int, [c_int32, c_int32, c_int32, c_float, c_float, c_float, c_int32, c_int32,
                                     c_void_p, c_size_t, POINTER(c_void_p)]),
    "ngsgd_precond_destroy": (c_int, [c_void_p]),
    "ngsgd_precond_reset": (c_int, [c_void_p]),
    "ngsgd_precondition": (c_int, [c_void_p, c_void_p, c_int32, c_int32, c_void_p, c_void_p, c_void_p]),
    "ngsgd_precond_get_state": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, POINTER(c_int64), c_void_p]),
    "ngsgd_precond_diagnostics": (c_int, [c_void_p, POINTER(c_int32), POINTER(c_int32), c_void_p]),
    "ngsgd_precond_set_state": (c_int, [c_void_p, c_void_p, c_void_p, c_double, c_int64, c_void_p]),
    "ngsgd_simple_workspace_bytes": (c_int, [c_int32, c_int32, POINTER(c_size_t)]),
    "ngsgd_precondition_simple": (c_int, [c_void_p, c_int32, c_int32, c_int32, c_float, c_float, c_void_p, c_size_t,
                                          c_void_p, c_void_p, c_void_p]),
    "ngsgd_precondition_simple_static": (c_int, [c_void_p, c_int32, c_int32, c_int32, c_float, c_float, c_void_p,
                                                 c_void_p, c_void_p]),
    "ngsgd_layernorm_forward": (c_int, [c_void_p, c_int64, c_int32, c_void_p, c_void_p, c_int32, c_int64, c_int32, c_float,
                                        c_void_p, c_int64, c_void_p, c_void_p, c_void_p]),
    "ngsgd_layernorm_workspace_bytes": (c_int, [c_int64, c_int32, POINTER(c_size_t)]),
    "ngsgd_layernorm_backward": (c_int, [c_void_p, c_int64, c_void_p, c_int64, c_int32, c_void_p, c_int32, c_void_p, c_void_p,
                                         c_int64, c_int32, c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_size_t,
                                         c_void_p]),
    "ngsgd_adamw_workspace_bytes": (c_int, [POINTER(ngsgd_adamw_config), POINTER(c_size_t)]),
    "ngsgd_adamw_create": (c_int, [POINTER(ngsgd_adamw_config), c_void_p, c_size_t, POINTER(c_void_p)]),
    "ngsgd_adamw_destroy": (c_int, [c_void_p]),
    "ngsgd_adamw_step": (c_int, [c_void_p, POINTER(c_void_p), c_float, c_void_p, c_float, c_void_p, c_void_p]),
    "ngsgd_adamw_arrays": (c_int, [c_void_p, POINTER(c_int64), POINTER(c_void_p), POINTER(c_void_p), POINTER(c_void_p)]),
    "ngsgd_adamw_get_state": (c_int, [c_void_p, c_void_p, c_void_p, c_int32, c_void_p, c_void_p]),
    "ngsgd_adamw_set_state": (c_int, [c_void_p, c_void_p, c_void_p, c_void_p, c_int64, c_void_p]),
    "ngsgd_workspace_bytes": (c_int, [POINTER(ngsgd_config), POINTER(c_size_t)]),
    "ngsgd_create": (c_int, [POINTER(ngsgd_config), c_void_p, c_size_t, POINTER(c_void_p)]),
    "ngsgd_destroy": (c_int, [c_void_p]),
    "ngsgd_step": (c_int, [c_void_p, c_void_p, c_void_p, c_int32, c_float, c_void_p, c_void_p]),
    "ngsgd_join": (c_int, [c_void_p, c_void_p]),
    "ngsgd_average": (c_int, [POINTER(c_void_p), c_int32, c_int32, c_void_p]),
    "ngsgd_get_params": (c_int, [c_void_p, c_int32, c_void_p, c_void_p]),
    "ngsgd_set_params": (c_int, [c_void_p, c_int32, c_void_p, c_void_p]),
    "ngsgd_get_norm": (c_int, [c_void_p, c_int32, c_void_p, c_void_p, c_void_p]),
    "ngsgd_set_norm": (c_int, [c_void_p, c_int32, c_void_p, c_void_p, c_void_p]),
    "ngsgd_set_adamw": (c_int, [c_void_p, c_float, c_double, c_double, c_float, c_float]),
    "ngsgd_last_norm_gradient": (c_int, [c_void_p, c_int32, c_void_p, c_void_p, c_void_p]),
    "ngsgd_net_precond": (c_int, [c_void_p, c_int32, c_int32, POINTER(c_void_p)]),
    "ngsgd_last_preconditioned": (c_int, [c_void_p, c_int32, c_int32, c_void_p, c_void_p]),
    "ngsgd_last_gradient": (c_int, [c_void_p, c_int32, c_void_p, c_void_p]),
    "ngsgd_last_max_change_scale": (c_int, [c_void_p, c_int32, c_void_p, c_void_p]),
    "ngsgd_profile_enable": (c_int, [c_int32]),
    "ngsgd_profile_read": (c_int, [POINTER(c_double), POINTER(c_int64), c_int32]),
    "ngsgd_strerror": (c_char_p, [c_int]),
    "ngsgd_set_wait_limit_us": (c_int, [c_int64]),
    "ngsgd_last_hip_error": (c_int, []),
    "ngsgd_version": (c_int, []),
}

_lib = None
_torch = None   # for calls that are short enough for an import statement to count


def load_library():
    """Loads libngsgd.so and binds every declared entry point; raises if the library is missing."""
    global _lib, _torch
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -m paper_1410_7455_amd.build` "
            "(hipcc, gfx950); there is no CPU fallback")
    try:
        # PyTorch ships its own HIP runtime: load it first, so that the library binds to the same copy as the
        # tensors whose pointers it is given (two runtimes in one process do not know each other's memory)
        import torch
        _torch = torch
    except ImportError:
        pass
    lib = ctypes.CDLL(LIB_PATH)
    for name, (restype, argtypes) in _SIGNATURES.items():
        fn = getattr(lib, name)          # AttributeError if the symbol is not exported
        fn.restype = restype
        fn.argtypes = argtypes
    _lib = lib
    return lib


def _check(code: int, where: str) -> None:
    if code != NGSGD_OK:
        raise NgsgdError(code, where)


def _stream_ptr(stream=None):
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return c_void_p(s.cuda_stream)


def _ptr(t):
    return c_void_p(0) if t is None else c_void_p(t.data_ptr())


class Preconditioner:
    """One online natural-gradient instance (ngsgd_precond_*) on the current CUDA/HIP device."""

    def __init__(self, dim, rank, max_batch, alpha=4.0, num_samples_history=2000.0, epsilon=1e-10,
                 update_period=4, always_update_first=10, _borrowed=None):
        import torch
        self.lib = load_library()
        self.dim, self.rank, self.max_batch = dim, rank, max_batch
        self._owner = None
        if _borrowed is not None:
            self.handle, self._owner = _borrowed
            self.workspace = None
            return
        nbytes = c_size_t(0)
        _check(self.lib.ngsgd_precond_workspace_bytes(dim, rank, max_batch, byref(nbytes)),
               "ngsgd_precond_workspace_bytes")
        self.workspace = torch.empty(nbytes.value, dtype=torch.uint8, device="cuda")
        h = c_void_p(0)
        _check(self.lib.ngsgd_precond_create(dim, rank, max_batch, alpha, num_samples_history, epsilon,
                                             update_period, always_update_first, _ptr(self.workspace),
                                             nbytes.value, byref(h)), "ngsgd_precond_create")
        self.handle = h

    def close(self):
        if self._owner is None and self.handle is not None:
            self.lib.ngsgd_precond_destroy(self.handle)
        self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def reset(self):
        _check(self.lib.ngsgd_precond_reset(self.handle), "ngsgd_precond_reset")

    def precondition(self, M, gamma=None, rownorm2=None, stream=None):
        """In place on the float32 CUDA tensor M (N x dim, row stride M.stride(0))."""
        assert M.is_cuda and M.dtype.is_floating_point and M.element_size() == 4 and M.stride(1) == 1
        _check(self.lib.ngsgd_precondition(self.handle, _ptr(M), M.shape[0], M.stride(0), _ptr(gamma),
                                           _ptr(rownorm2), _stream_ptr(stream)), "ngsgd_precondition")

    def get_state(self):
        import torch
        W = torch.empty((self.rank, self.dim), dtype=torch.float32, device="cuda")
        d = torch.empty(self.rank, dtype=torch.float64, device="cuda")
        rho = torch.empty(1, dtype=torch.float64, device="cuda")
        t = c_int64(0)
        _check(self.lib.ngsgd_precond_get_state(self.handle, _ptr(W), _ptr(d), _ptr(rho), byref(t),
                                                _stream_ptr()), "ngsgd_precond_get_state")
        torch.cuda.synchronize()
        return W, d, float(rho.item()), t.value

    def diagnostics(self):
        """(flags, Jacobi sweeps) of the latest factor update (flag 16: of the latest first factor); waits for the stream."""
        flags, sweeps = c_int32(0), c_int32(0)
        _check(self.lib.ngsgd_precond_diagnostics(self.handle, byref(flags), byref(sweeps), _stream_ptr()),
               "ngsgd_precond_diagnostics")
        return flags.value, sweeps.value

    def set_state(self, R, d, rho, t):
        """R: rank x dim float64 CUDA tensor with orthonormal rows, d: rank float64, rho > 0, t >= 1."""
        assert R.is_cuda and R.dtype.itemsize == 8 and R.is_contiguous() and tuple(R.shape) == (self.rank, self.dim)
        assert d.is_cuda and d.dtype.itemsize == 8 and d.numel() == self.rank
        _check(self.lib.ngsgd_precond_set_state(self.handle, _ptr(R), _ptr(d), float(rho), int(t),
                                                _stream_ptr()), "ngsgd_precond_set_state")


class SimplePreconditioner:
    """The simple method of App. A (ngsgd_precondition_simple): stateless, the workspace is kept for reuse."""

    def __init__(self, max_rows, dim, alpha=4.0, epsilon=1e-20):
        import torch
        self.lib = load_library()
        self.max_rows, self.dim, self.alpha, self.epsilon = max_rows, dim, alpha, epsilon
        nbytes = c_size_t(0)
        _check(self.lib.ngsgd_simple_workspace_bytes(max_rows, dim, byref(nbytes)), "ngsgd_simple_workspace_bytes")
        self.workspace_bytes = nbytes.value
        self.workspace = torch.empty(nbytes.value, dtype=torch.uint8, device="cuda")

    def precondition(self, M, gamma=None, rownorm2=None, stream=None):
        """In place on the float32 CUDA tensor M (N x dim, row stride M.stride(0)), N <= max_rows."""
        assert M.is_cuda and M.element_size() == 4 and M.stride(1) == 1 and M.shape[1] == self.dim
        _check(self.lib.ngsgd_precondition_simple(_ptr(M), M.shape[0], M.shape[1], M.stride(0), self.alpha,
                                                  self.epsilon, _ptr(self.workspace), self.workspace_bytes,
                                                  _ptr(gamma), _ptr(rownorm2), _stream_ptr(stream)),
               "ngsgd_precondition_simple")


def precondition_simple_static(M, alpha=4.0, epsilon=1e-20, gamma=None, rownorm2=None, stream=None):
    """ngsgd_precondition_simple_static: the simple method in place on M with the library's fixed scratch."""
    assert M.is_cuda and M.element_size() == 4 and M.stride(1) == 1
    _check(load_library().ngsgd_precondition_simple_static(_ptr(M), M.shape[0], M.shape[1], M.stride(0), alpha,
                                                           epsilon, _ptr(gamma), _ptr(rownorm2),
                                                           _stream_ptr(stream)),
           "ngsgd_precondition_simple_static")


_TYPES = {}


def _type_of(dtype):
    """NGSGD_FLOAT32 / _BFLOAT16 / _FLOAT16 of a torch dtype."""
    if not _TYPES:
        import torch
        _TYPES.update({torch.float32: NGSGD_FLOAT32, torch.bfloat16: NGSGD_BFLOAT16, torch.float16: NGSGD_FLOAT16})
    code = _TYPES.get(dtype)
    if code is None:
        raise ValueError(f"{dtype}: the types are float32, bfloat16 and float16")
    return code


# The argument checks below keep a kernel inside its buffers: they raise where assertions are switched off too.  Messages are only
# formed when they are needed (the calls are short: a small layer norm takes 2 us on the GPU).

def _current_device(device):
    if device.index != _torch.cuda.current_device():
        raise ValueError(f"made for {device}, which is not the current device")


def _check_dense(t, name, device, dtype=None, numel=None):
    """A dense tensor on the device."""
    if t.get_device() != device.index:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} is not dense")
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{name} is {t.dtype}, not {dtype}")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{name} has {t.numel()} elements, not {numel}")


def _raw_stream(stream, device, workspace=None, home=None):
    """The stream's hipStream_t.  A workspace that is used on another stream than the one it was allocated on (`home`) is not given to
    anybody else before that stream is done with it, though its owner may be gone."""
    stream = _torch.cuda.current_stream(device.index) if stream is None else stream
    raw = stream.cuda_stream
    if workspace is not None and raw != home:
        workspace.record_stream(stream)
    return raw


def _address(t):
    return None if t is None else t.data_ptr()


def _allocate_on(stream):
    """Outputs are allocated on the stream that writes them."""
    return nullcontext() if stream is None else _torch.cuda.stream(stream)


class LayerNorm:
    """ngsgd_layernorm_forward / ngsgd_layernorm_backward: stateless, the workspace of the gradients is kept for reuse.

    Inputs are float32, bfloat16 or float16, (..., dim) with up to max_rows rows; rows are dense (the last stride is 1) and,
    as a matrix, may lie any distance apart.  Weight and bias (optional) have the input's type or float32, the same for both.  Calls on
    one object are issued in order on one stream: the workspace is shared.  As with torch's own operators, tensors that are given to a
    call on another stream than their own are the caller's to keep until it has run (torch.Tensor.record_stream)."""

    def __init__(self, max_rows, dim, epsilon=1e-5):
        import torch
        self.lib = load_library()
        self.max_rows, self.dim, self.epsilon = max_rows, dim, epsilon
        nbytes = c_size_t(0)
        _check(self.lib.ngsgd_layernorm_workspace_bytes(max_rows, dim, byref(nbytes)), "ngsgd_layernorm_workspace_bytes")
        self.workspace_bytes = nbytes.value
        self.workspace = torch.empty(nbytes.value, dtype=torch.uint8, device="cuda")
        self.device = self.workspace.device
        self._home = _raw_stream(None, self.device)

    def _rows(self, t, name, like=None):
        """(number of rows, leading dimension)"""
        if t.get_device() != self.device.index:
            raise ValueError(f"{name} is on {t.device}, not on {self.device}")
        shape = t.shape
        if len(shape) < 1 or shape[-1] != self.dim:
            raise ValueError(f"{name} does not end in {self.dim} columns")
        if like is not None and (t.dtype != like.dtype or shape != like.shape):
            raise ValueError(f"{name} has another type or shape than x")
        if len(shape) != 2:
            t = t.view(-1, self.dim) if t.numel() else t.new_empty(0, self.dim)
        rows = t.shape[0]
        ld, inner = t.stride()
        if inner != 1 and self.dim != 1:
            raise ValueError(f"{name}: rows are not dense")
        if rows > self.max_rows:
            raise ValueError(f"{name} has more than {self.max_rows} rows")
        return rows, ld if rows > 1 else self.dim

    def _vector_dtype(self, x, *named):
        """The type of the given weights (of the first one present; float32 if there is none)."""
        dtype = None
        for name, v in named:
            if v is None:
                continue
            if dtype is None:
                dtype = v.dtype
                if dtype != x.dtype and dtype != _torch.float32:
                    raise ValueError(f"{name} is {dtype} for {x.dtype} rows")
            _check_dense(v, name, self.device, dtype, self.dim)
        return _torch.float32 if dtype is None else dtype

    def forward(self, x, weight=None, bias=None, out=None, mean=None, rstd=None, stream=None):
        """(y, mean, rstd); y into `out` if given (which may be x), the rows' float32 mean and rstd into `mean` and `rstd`."""
        _current_device(self.device)
        rows, ldx = self._rows(x, "x")
        weight_type = _type_of(self._vector_dtype(x, ("weight", weight), ("bias", bias)))
        ldy = self.dim if out is None else self._rows(out, "out", x)[1]
        if mean is not None:
            _check_dense(mean, "mean", self.device, _torch.float32, rows)
        if rstd is not None:
            _check_dense(rstd, "rstd", self.device, _torch.float32, rows)
        if out is None or mean is None or rstd is None:
            with _allocate_on(stream):
                if out is None:
                    out = _torch.empty_like(x, memory_format=_torch.contiguous_format)
                if mean is None:
                    mean = _torch.empty(rows, dtype=_torch.float32, device=self.device)
                if rstd is None:
                    rstd = _torch.empty(rows, dtype=_torch.float32, device=self.device)
        _check(self.lib.ngsgd_layernorm_forward(x.data_ptr(), ldx, _type_of(x.dtype), _address(weight), _address(bias), weight_type,
                                                rows, self.dim, self.epsilon, out.data_ptr(), ldy, mean.data_ptr(),
                                                rstd.data_ptr(), _raw_stream(stream, self.device)), "ngsgd_layernorm_forward")
        return out, mean, rstd

    def backward(self, dy, x, mean, rstd, weight=None, needs=(True, True, True), dx=None, dweight=None, dbias=None,
                 stream=None):
        """(dx, dweight, dbias) for the derivative dy of y and the mean and rstd of the forward pass; None where `needs`
        says so and none is given.  dx may be dy.  dweight and dbias are of the weight's type (float32 without a weight)."""
        _current_device(self.device)
        rows, ldx = self._rows(x, "x")
        _, lddy = self._rows(dy, "dy", x)
        _check_dense(mean, "mean", self.device, _torch.float32, rows)
        _check_dense(rstd, "rstd", self.device, _torch.float32, rows)
        vector = self._vector_dtype(x, ("weight", weight), ("dweight", dweight), ("dbias", dbias))
        lddx = self.dim if dx is None else self._rows(dx, "dx", x)[1]
        with _allocate_on(stream):
            if dx is None and needs[0]:
                dx = _torch.empty_like(x, memory_format=_torch.contiguous_format)
            if dweight is None and needs[1]:
                dweight = _torch.empty(self.dim, dtype=vector, device=self.device)
            if dbias is None and needs[2]:
                dbias = _torch.empty(self.dim, dtype=vector, device=self.device)
        _check(self.lib.ngsgd_layernorm_backward(dy.data_ptr(), lddy, x.data_ptr(), ldx, _type_of(x.dtype), _address(weight),
                                                 _type_of(vector), mean.data_ptr(), rstd.data_ptr(), rows, self.dim,
                                                 _address(dx), lddx, _address(dweight), _address(dbias),
                                                 self.workspace.data_ptr(), self.workspace_bytes,
                                                 _raw_stream(stream, self.device, self.workspace, self._home)),
               "ngsgd_layernorm_backward")
        return dx, dweight, dbias


class AdamW:
    """ngsgd_adamw_*: one AdamW step over many tensors of one type per call, on the current device.

    The parameters are dense tensors, updated in place where they lie.  weight_decay and rate (a factor on the learning rate) are
    numbers or one number per tensor.  state_bits is 32 or 8; master keeps fp32 copies of parameters in 16 bits.  Calls on
    one object are issued in order on one stream.  As with torch's own operators, tensors that are given to a call on another
    stream than their own are the caller's to keep until it has run (torch.Tensor.record_stream)."""

    def __init__(self, params, betas=(0.9, 0.999), epsilon=1e-8, weight_decay=0.0, rate=1.0, grad_dtype=None, state_bits=32,
                 master=False):
        import torch
        self.handle = None
        self.lib = load_library()
        self.params = list(params)
        n = len(self.params)
        if n == 0:
            raise ValueError("no parameters")
        if not self.params[0].is_cuda:
            raise ValueError("the parameters are not on the GPU")
        self.device, dtype = self.params[0].device, self.params[0].dtype
        _current_device(self.device)
        for i, p in enumerate(self.params):
            _check_dense(p, f"parameter {i}", self.device, dtype)
        self.grad_dtype = dtype if grad_dtype is None else grad_dtype
        self.sizes = [p.numel() for p in self.params]
        self.offsets, at = [], 0
        for size in self.sizes:
            self.offsets.append(at)
            at += -(-size // 256) * 256

        def per_tensor(value, name):
            values = list(value) if isinstance(value, (list, tuple)) else [float(value)] * n
            if len(values) != n:
                raise ValueError(f"{len(values)} numbers in {name} for {n} tensors")
            return (c_float * n)(*values)

        cfg = ngsgd_adamw_config(n, (c_void_p * n)(*[p.data_ptr() for p in self.params]), (c_int64 * n)(*self.sizes),
                                 per_tensor(weight_decay, "weight_decay"), per_tensor(rate, "rate"), _type_of(dtype),
                                 _type_of(self.grad_dtype), state_bits, 1 if master else 0, betas[0], betas[1], epsilon)
        nbytes = c_size_t(0)
        _check(self.lib.ngsgd_adamw_workspace_bytes(byref(cfg), byref(nbytes)), "ngsgd_adamw_workspace_bytes")
        self.workspace_bytes = nbytes.value
        self.workspace = torch.empty(nbytes.value, dtype=torch.uint8, device=self.device)
        self._home = _raw_stream(None, self.device)
        h = c_void_p(0)
        _check(self.lib.ngsgd_adamw_create(byref(cfg), _ptr(self.workspace), nbytes.value, byref(h)), "ngsgd_adamw_create")
        self.handle = h
        elements, m, v, fp32 = c_int64(0), c_void_p(0), c_void_p(0), c_void_p(0)
        _check(self.lib.ngsgd_adamw_arrays(h, byref(elements), byref(m), byref(v), byref(fp32)), "ngsgd_adamw_arrays")
        self.elements = elements.value

        def view(address):
            if not address.value:
                return None
            start = address.value - self.workspace.data_ptr()
            return self.workspace[start:start + 4 * self.elements].view(torch.float32)

        self._m, self._v = view(m), view(v)
        self.master = view(fp32)          # flat, None without fp32 copies
        self._grads = (c_void_p * n)()

    def close(self):
        if self.handle is not None:
            self.lib.ngsgd_adamw_destroy(self.handle)
        self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def step(self, grads, lr, grad_scale=None, stream=None):
        """One step.  grads: a dense tensor of grad_dtype for each parameter, or None to leave that one as it is.  lr and grad_scale are
        numbers or float32 tensors of one element on the device."""
        device, dtype, sizes, addresses = self.device, self.grad_dtype, self.sizes, []
        index = device.index
        _current_device(device)
        if len(grads) != len(sizes):
            raise ValueError(f"{len(grads)} gradients for {len(sizes)} tensors")
        for g, size in zip(grads, sizes):
            if g is None or size == 0:
                addresses.append(None)
                continue
            if g.dtype != dtype or g.numel() != size or g.get_device() != index or not g.is_contiguous():
                raise ValueError(f"gradient {len(addresses)}: {g.dtype}, {g.numel()} elements on {g.device}, for {dtype}, {size} on "
                                 f"{device}, dense")
            addresses.append(g.data_ptr())
        self._grads[:] = addresses
        factors = []
        for name, value in (("lr", lr), ("grad_scale", grad_scale)):
            if isinstance(value, _torch.Tensor):
                _check_dense(value, name, device, _torch.float32, 1)
                factors += [1.0, value.data_ptr()]
            else:
                factors += [1.0 if value is None else value, None]
        _check(self.lib.ngsgd_adamw_step(self.handle, self._grads, *factors, _raw_stream(stream, self.device, self.workspace, self._home)), "ngsgd_adamw_step")

    def state(self, dtype=None, stream=None):
        """(m, v), flat; tensor k's are [offsets[k] : offsets[k] + sizes[k]].  With 32 bits the arrays themselves (or copies in
        bfloat16, if asked for); with 8 bits the values of the codes, in float32 or in bfloat16, which holds them exactly (but for a
        v below 2^-126)."""
        dtype = _torch.float32 if dtype is None else dtype
        if self._m is not None and dtype == _torch.float32:
            return self._m, self._v
        _current_device(self.device)
        with _allocate_on(stream):
            m = _torch.empty(self.elements, dtype=dtype, device=self.device)
            v = _torch.empty(self.elements, dtype=dtype, device=self.device)
        _check(self.lib.ngsgd_adamw_get_state(self.handle, m.data_ptr(), v.data_ptr(), _type_of(dtype), None, _raw_stream(stream, self.device, self.workspace, self._home)),
               "ngsgd_adamw_get_state")
        return m, v

    def set_state(self, m, v, t, master=None, stream=None):
        """Installs flat float32 moments (zeros between the tensors; None: zeros) and the step count; the fp32 copies from `master` (flat), which is rounded to the
        parameters too, or from the parameters."""
        import torch
        _current_device(self.device)
        for name, a in (("m", m), ("v", v), ("master", master)):
            if a is not None:
                _check_dense(a, name, self.device, torch.float32, self.elements)
        _check(self.lib.ngsgd_adamw_set_state(self.handle, _address(m), _address(v), _address(master), int(t), _raw_stream(stream, self.device, self.workspace, self._home)),
               "ngsgd_adamw_set_state")

    def steps(self, stream=None):
        """The step count behind the calls on `stream` so far (None: the current one); waits for them."""
        import torch
        _current_device(self.device)
        with _allocate_on(stream):
            t = torch.empty(1, dtype=torch.int64, device=self.device)
            _check(self.lib.ngsgd_adamw_get_state(self.handle, None, None, NGSGD_FLOAT32, t.data_ptr(),
                                                  _raw_stream(stream, self.device, self.workspace, self._home)), "ngsgd_adamw_get_state")
            return int(t.item())


class Network:
    """One replica (ngsgd_create / ngsgd_step / ...)."""

    def __init__(self, dims, nonlin, max_batch, pnorm_group=10, rank_in=20, rank_out=80, alpha=4.0,
                 num_samples_history=2000.0, epsilon=1e-10, update_period=4, always_update_first=10,
                 renorm=False, max_change_per_sample=0.0, method="online", simple_epsilon=1e-20, side_streams=0):
        import torch
        self.lib = load_library()
        self.handle = None
        self.method = {"online": NGSGD_METHOD_ONLINE, "simple": NGSGD_METHOD_SIMPLE, "adamw": NGSGD_METHOD_ADAMW,
                       "adamw8": NGSGD_METHOD_ADAMW8}[method]
        self.dims = list(dims)
        self.nonlin = list(nonlin)
        self.n_layers = len(dims) - 1
        self.pnorm_group = pnorm_group
        self.max_batch = max_batch
        self.rank_in, self.rank_out = rank_in, rank_out
        self.in_dims = []
        d_in = dims[0]
        for l in range(self.n_layers):
            self.in_dims.append(d_in)
            if l < self.n_layers - 1:
                d_in = dims[l + 1] // pnorm_group if nonlin[l] & ~NGSGD_LAYERNORM == NGSGD_PNORM else dims[l + 1]
        self._dims_arr = (c_int32 * len(dims))(*dims)
        self._nonlin_arr = (c_int32 * max(1, len(nonlin)))(*nonlin)
        cfg = ngsgd_config(self.n_layers, self._dims_arr, self._nonlin_arr, pnorm_group, max_batch, rank_in,
                           rank_out, alpha, num_samples_history, epsilon, update_period, always_update_first,
                           1 if renorm else 0, max_change_per_sample, self.method, simple_epsilon, side_streams)
        nbytes = c_size_t(0)
        _check(self.lib.ngsgd_workspace_bytes(byref(cfg), byref(nbytes)), "ngsgd_workspace_bytes")
        self.workspace_bytes = nbytes.value
        self.workspace = torch.empty(nbytes.value, dtype=torch.uint8, device="cuda")
        h = c_void_p(0)
        _check(self.lib.ngsgd_create(byref(cfg), _ptr(self.workspace), nbytes.value, byref(h)), "ngsgd_create")
        self.handle = h
        self._logprob = torch.zeros(1, dtype=torch.float64, device="cuda")

    def close(self):
        if self.handle is not None:
            self.lib.ngsgd_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_params(self, layer, w):
        assert w.is_cuda and w.is_contiguous() and w.element_size() == 4
        assert tuple(w.shape) == (self.dims[layer + 1], self.in_dims[layer] + 1)
        _check(self.lib.ngsgd_set_params(self.handle, layer, _ptr(w), _stream_ptr()), "ngsgd_set_params")

    def get_params(self, layer):
        import torch
        w = torch.empty((self.dims[layer + 1], self.in_dims[layer] + 1), dtype=torch.float32, device="cuda")
        _check(self.lib.ngsgd_get_params(self.handle, layer, _ptr(w), _stream_ptr()), "ngsgd_get_params")
        return w

    def _norm_vectors(self, layer, *vectors):
        import torch
        dim = self.in_dims[layer + 1] if 0 <= layer < self.n_layers - 1 else 0
        for v in vectors:
            if v is not None:
                _check_dense(v, "layer-norm vector", self.workspace.device, torch.float32, dim)
        return dim

    def set_norm(self, layer, weight=None, bias=None, stream=None):
        """Weight and bias of the layer norm behind hidden layer `layer` (None: left as it is)."""
        self._norm_vectors(layer, weight, bias)
        _check(self.lib.ngsgd_set_norm(self.handle, layer, _ptr(weight), _ptr(bias), _stream_ptr(stream)), "ngsgd_set_norm")

    def get_norm(self, layer, stream=None):
        """(weight, bias) of the layer norm behind hidden layer `layer`."""
        import torch
        dim = self._norm_vectors(layer)
        with _allocate_on(stream):
            w, b = (torch.empty(dim, dtype=torch.float32, device=self.workspace.device) for _ in range(2))
        _check(self.lib.ngsgd_get_norm(self.handle, layer, _ptr(w), _ptr(b), _stream_ptr(stream)), "ngsgd_get_norm")
        return w, b

    def set_adamw(self, rate=1.0, betas=(0.9, 0.999), epsilon=1e-8, weight_decay=0.0):
        """Numbers of the AdamW step (layer norms; with the AdamW methods the weight matrices too); forgets its moments."""
        _check(self.lib.ngsgd_set_adamw(self.handle, rate, betas[0], betas[1], epsilon, weight_decay), "ngsgd_set_adamw")

    def last_norm_gradient(self, layer, stream=None):
        """Gradients of the latest step by the weight and the bias of the layer norm behind hidden layer `layer`."""
        import torch
        dim = self._norm_vectors(layer)
        with _allocate_on(stream):
            w, b = (torch.empty(dim, dtype=torch.float32, device=self.workspace.device) for _ in range(2))
        _check(self.lib.ngsgd_last_norm_gradient(self.handle, layer, _ptr(w), _ptr(b), _stream_ptr(stream)),
               "ngsgd_last_norm_gradient")
        return w, b

    def step(self, x, labels, lr, logprob_out=None, stream=None):
        """Enqueues one minibatch step; the sum of log-probabilities lands in `logprob_out` (1 float64)."""
        assert x.is_cuda and x.is_contiguous() and x.element_size() == 4 and x.shape[1] == self.dims[0]
        assert labels.is_cuda and labels.is_contiguous() and labels.element_size() == 4
        out = self._logprob if logprob_out is None else logprob_out
        _check(self.lib.ngsgd_step(self.handle, _ptr(x), _ptr(labels), x.shape[0], float(lr), _ptr(out),
                                   _stream_ptr(stream)), "ngsgd_step")
        return out

    def join(self, stream=None):
        """Makes the stream wait for the factor updates the network has in flight on its internal streams."""
        _check(self.lib.ngsgd_join(self.handle, _stream_ptr(stream)), "ngsgd_join")

    def precond(self, layer, side):
        h = c_void_p(0)
        _check(self.lib.ngsgd_net_precond(self.handle, layer, side, byref(h)), "ngsgd_net_precond")
        if not h.value:
            return None
        dim = self.in_dims[layer] + 1 if side == NGSGD_SIDE_INPUT else self.dims[layer + 1]
        rank = self.rank_in if side == NGSGD_SIDE_INPUT else self.rank_out
        return Preconditioner(dim, rank, self.max_batch, _borrowed=(h, self))

    def last_preconditioned(self, layer, side, n_rows):
        import torch
        dim = self.in_dims[layer] + 1 if side == NGSGD_SIDE_INPUT else self.dims[layer + 1]
        out = torch.empty((n_rows, dim), dtype=torch.float32, device="cuda")
        _check(self.lib.ngsgd_last_preconditioned(self.handle, layer, side, _ptr(out), _stream_ptr()),
               "ngsgd_last_preconditioned")
        return out

    def last_gradient(self, layer):
        import torch
        out = torch.empty((self.dims[layer + 1], self.in_dims[layer] + 1), dtype=torch.float32, device="cuda")
        _check(self.lib.ngsgd_last_gradient(self.handle, layer, _ptr(out), _stream_ptr()), "ngsgd_last_gradient")
        return out

    def last_max_change_scale(self, layer):
        import torch
        out = torch.empty(1, dtype=torch.float64, device="cuda")
        _check(self.lib.ngsgd_last_max_change_scale(self.handle, layer, _ptr(out), _stream_ptr()),
               "ngsgd_last_max_change_scale")
        return out


PROFILE_CATEGORIES = ["gemm_fwd", "gemm_bwd", "gemm_upd", "precond_h", "precond_j", "precond_xhat", "precond_kl",
                      "precond_small", "precond_wnew", "elementwise", "precond_misc", "init", "simple_gram",
                      "simple_inverse", "simple_apply", "precond_fused"]


def profile_enable(on: bool) -> None:
    _check(load_library().ngsgd_profile_enable(1 if on else 0), "ngsgd_profile_enable")


def profile_read():
    """{category: (milliseconds, bracketed launch groups)} since the last read."""
    n = len(PROFILE_CATEGORIES)
    ms = (c_double * n)()
    cnt = (c_int64 * n)()
    _check(load_library().ngsgd_profile_read(ms, cnt, n), "ngsgd_profile_read")
    return {name: (ms[i], cnt[i]) for i, name in enumerate(PROFILE_CATEGORIES)}


def set_wait_limit_us(microseconds: int) -> None:
    """ngsgd_set_wait_limit_us: bound of the waits between workgroups (fused apply kernel, first factors)."""
    _check(load_library().ngsgd_set_wait_limit_us(int(microseconds)), "ngsgd_set_wait_limit_us")


def average(networks, reset_preconditioners=True, stream=None):
    """ngsgd_average over replicas living on the same device."""
    lib = load_library()
    arr = (c_void_p * len(networks))(*[n.handle for n in networks])
    _check(lib.ngsgd_average(arr, len(networks), 1 if reset_preconditioners else 0, _stream_ptr(stream)),
           "ngsgd_average")
