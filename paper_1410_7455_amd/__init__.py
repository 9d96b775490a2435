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
from array import array
from contextlib import nullcontext
from ctypes import POINTER, byref, c_char_p, c_double, c_float, c_int, c_int32, c_int64, c_size_t, c_void_p

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libngsgd.so")
HELPER_PATH = os.path.join(_HERE, "_tensors.so")

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
NGSGD_INT32 = 3
NGSGD_INT64 = 4
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
    "ngsgd_embedding_forward": (c_int, [c_void_p, c_int32, c_int64, c_void_p, c_int64, c_int32, c_int64, c_int32, c_float,
                                        c_void_p, c_int64, c_int32, c_void_p]),
    "ngsgd_embedding_workspace_bytes": (c_int, [c_int64, c_int64, c_int32, POINTER(c_size_t)]),
    "ngsgd_embedding_backward": (c_int, [c_void_p, c_int64, c_int32, c_void_p, c_int32, c_int64, c_int64, c_int32, c_float,
                                         c_void_p, c_int64, c_int32, c_int32, c_void_p, c_size_t, c_void_p]),
    "ngsgd_cross_entropy_workspace_bytes": (c_int, [c_int64, c_int32, POINTER(c_size_t)]),
    "ngsgd_cross_entropy": (c_int, [c_void_p, c_int64, c_int32, c_void_p, c_int32, c_int64, c_int32, c_void_p, c_float, c_void_p,
                                    c_void_p, c_int64, c_void_p, c_size_t, c_void_p]),
    "ngsgd_grad_norm_workspace_bytes": (c_int, [c_int32, POINTER(c_size_t)]),
    "ngsgd_grad_norm": (c_int, [c_int32, c_void_p, c_void_p, c_int32, c_double, c_void_p, c_void_p, c_void_p,
                                c_size_t, c_void_p]),
    "ngsgd_grad_clip": (c_int, [c_int32, c_void_p, c_void_p, c_int32, c_double, c_void_p, c_void_p,
                                c_void_p, c_void_p, c_size_t, c_void_p]),
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


def _library():
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


def _load_helper():
    """Loads _tensors.so (addresses of many tensors at once), which GradientNorm needs; from then on it is a name of this package."""
    try:
        from . import _tensors   # noqa: F401
    except ImportError as e:
        raise ImportError(f"{HELPER_PATH} is missing or of another torch: build it with `python -m paper_1410_7455_amd.build`") from e


def load_library():
    """Loads libngsgd.so, binds every declared entry point and loads the helper of GradientNorm, if it was built; raises if the library is missing,
    or if the helper is of another torch."""
    lib = _library()
    if _torch is not None and "_tensors" not in globals() and os.path.exists(HELPER_PATH):
        _load_helper()
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
        self.lib = _library()
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
        self.lib = _library()
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
    _check(_library().ngsgd_precondition_simple_static(_ptr(M), M.shape[0], M.shape[1], M.stride(0), alpha,
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


def _current_raw_stream(index):
    """hipStream_t of the device's current stream, without an object for it where torch has a call for that."""
    get = getattr(_torch._C, "_cuda_getCurrentRawStream", None)
    return _torch.cuda.current_stream(index).cuda_stream if get is None else get(index)


def _raw_stream(stream, device, workspace=None, home=None):
    """The stream's hipStream_t.  A workspace that is used on another stream than the one it was allocated on (`home`) is not given to
    anybody else before that stream is done with it, though its owner may be gone."""
    raw = _current_raw_stream(device.index) if stream is None else stream.cuda_stream
    if workspace is not None and raw != home:
        workspace.record_stream(_torch.cuda.current_stream(device.index) if stream is None else stream)
    return raw


def _address(t):
    return None if t is None else t.data_ptr()


_HERE_AND_NOW = nullcontext()


def _allocate_on(stream):
    """Outputs are allocated on the stream that writes them."""
    return _HERE_AND_NOW if stream is None else _torch.cuda.stream(stream)


class LayerNorm:
    """ngsgd_layernorm_forward / ngsgd_layernorm_backward: stateless, the workspace of the gradients is kept for reuse.

    Inputs are float32, bfloat16 or float16, (..., dim) with up to max_rows rows; rows are dense (the last stride is 1) and,
    as a matrix, may lie any distance apart.  Weight and bias (optional) have the input's type or float32, the same for both.  Calls on
    one object are issued in order on one stream: the workspace is shared.  As with torch's own operators, tensors that are given to a
    call on another stream than their own are the caller's to keep until it has run (torch.Tensor.record_stream)."""

    def __init__(self, max_rows, dim, epsilon=1e-5):
        import torch
        self.lib = _library()
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


def _index_type(t, name, device):
    """NGSGD_INT32 / _INT64 of a dense tensor of tokens or labels on the device."""
    if t.get_device() != device.index:
        raise ValueError(f"{name} are on {t.device}, not on {device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} are not dense")
    if t.dtype == _torch.int64:
        return NGSGD_INT64
    if t.dtype == _torch.int32:
        return NGSGD_INT32
    raise ValueError(f"{name} are {t.dtype}: the types are int32 and int64")


def _matrix(t, name, device, rows, columns):
    """Leading dimension of a matrix on the device whose rows are dense; any distance apart."""
    if t.get_device() != device.index:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    if t.dim() != 2 or t.shape[0] != rows or t.shape[1] != columns:
        raise ValueError(f"{name} has the shape {tuple(t.shape)}, not {(rows, columns)}")
    ld, inner = t.stride()
    if inner != 1 and columns != 1:
        raise ValueError(f"{name}: rows are not dense")
    return ld if rows > 1 else columns


class Embedding:
    """ngsgd_embedding_forward / ngsgd_embedding_backward: rows of a table by tokens, times `scale`; the workspace of the gradient is
    kept for reuse.

    Tokens are int32 or int64, dense, of any shape, up to max_tokens; those outside [0, vocabulary) are padding.  The table is (vocabulary, dim),
    its rows dense and any distance apart, float32 or of the type of the rows that are looked up (float32, bfloat16 or float16).  Calls on one object
    are issued in order on one stream: the workspace is shared.  As with torch's own operators, tensors that are given to a
    call on another stream than their own are the caller's to keep until it has run (torch.Tensor.record_stream)."""

    def __init__(self, max_tokens, vocabulary, dim, scale=1.0):
        import torch
        self.lib = _library()
        self.max_tokens, self.vocabulary, self.dim, self.scale = max_tokens, vocabulary, dim, scale
        nbytes = c_size_t(0)
        _check(self.lib.ngsgd_embedding_workspace_bytes(max_tokens, vocabulary, dim, byref(nbytes)), "ngsgd_embedding_workspace_bytes")
        self.workspace_bytes = nbytes.value
        self.workspace = torch.empty(nbytes.value, dtype=torch.uint8, device="cuda")
        self.device = self.workspace.device
        self._home = _raw_stream(None, self.device)

    def _tokens(self, tokens):
        """(count, index type)"""
        index = _index_type(tokens, "tokens", self.device)
        n = tokens.numel()
        if n > self.max_tokens:
            raise ValueError(f"more than {self.max_tokens} tokens")
        return n, index

    def _rows(self, t, name, tokens, n):
        """Leading dimension of tokens.shape + (dim,)."""
        shape = t.shape
        if len(shape) != 2 or tokens.dim() != 1:
            if shape != tokens.shape + (self.dim,):
                raise ValueError(f"{name} has the shape {tuple(shape)}, not {tuple(tokens.shape) + (self.dim,)}")
            t = t.view(-1, self.dim) if n else t.new_empty(0, self.dim)
        return _matrix(t, name, self.device, n, self.dim)

    def _table_type(self, table_dtype, dtype):
        if table_dtype != dtype and table_dtype != _torch.float32:
            raise ValueError(f"a table of {table_dtype} for rows of {dtype}")
        return _type_of(table_dtype)

    def forward(self, tokens, table, dtype=None, out=None, stream=None):
        """tokens.shape + (dim,) rows of `dtype` (the table's, if none is given), into `out` if given."""
        _current_device(self.device)
        n, index = self._tokens(tokens)
        ldt = _matrix(table, "table", self.device, self.vocabulary, self.dim)
        if out is not None:
            if dtype is not None and dtype != out.dtype:
                raise ValueError(f"out is {out.dtype}, not {dtype}")
            dtype, ldy = out.dtype, self._rows(out, "out", tokens, n)
        else:
            dtype, ldy = table.dtype if dtype is None else dtype, self.dim
        table_type = self._table_type(table.dtype, dtype)
        type_ = _type_of(dtype)
        if out is None:
            with _allocate_on(stream):
                out = _torch.empty((*tokens.shape, self.dim), dtype=dtype, device=self.device)
        _check(self.lib.ngsgd_embedding_forward(tokens.data_ptr(), index, n, table.data_ptr(), ldt, table_type, self.vocabulary, self.dim,
                                                self.scale, out.data_ptr(), ldy, type_, _raw_stream(stream, self.device)),
               "ngsgd_embedding_forward")
        return out

    def backward(self, dy, tokens, dtype=None, dtable=None, accumulate=False, stream=None):
        """The table's gradient (vocabulary, dim) of `dtype` (dy's, if none is given) for the derivative dy of the rows, into `dtable` if
        given: in its place, or with `accumulate` added to it."""
        _current_device(self.device)
        n, index = self._tokens(tokens)
        lddy = self._rows(dy, "dy", tokens, n)
        if dtable is not None:
            if dtype is not None and dtype != dtable.dtype:
                raise ValueError(f"dtable is {dtable.dtype}, not {dtype}")
            dtype, lddt = dtable.dtype, _matrix(dtable, "dtable", self.device, self.vocabulary, self.dim)
        elif accumulate:
            raise ValueError("nothing to add to: no dtable")
        else:
            dtype, lddt = dy.dtype if dtype is None else dtype, self.dim
        table_type = self._table_type(dtype, dy.dtype)
        type_ = _type_of(dy.dtype)
        if dtable is None:
            with _allocate_on(stream):
                dtable = _torch.empty((self.vocabulary, self.dim), dtype=dtype, device=self.device)
        _check(self.lib.ngsgd_embedding_backward(dy.data_ptr(), lddy, type_, tokens.data_ptr(), index, n, self.vocabulary, self.dim, self.scale,
                                                 dtable.data_ptr(), lddt, table_type, 1 if accumulate else 0, self.workspace.data_ptr(),
                                                 self.workspace_bytes, _raw_stream(stream, self.device, self.workspace, self._home)),
               "ngsgd_embedding_backward")
        return dtable


class CrossEntropy:
    """ngsgd_cross_entropy: the loss of each row of logits, and the gradient of their sum.

    Logits are float32, bfloat16 or float16, (..., classes) with up to max_rows rows, which are dense and, as a matrix, may lie any
    distance apart.  Labels are int32 or int64, dense, one for each row; a row whose label is outside [0, classes) does not count.  Calls
    on one object are issued in order on one stream: the workspace is shared.  As with torch's own operators, tensors that are given to a call on
    another stream than their own are the caller's to keep until it has run (torch.Tensor.record_stream)."""

    def __init__(self, max_rows, classes):
        import torch
        self.lib = _library()
        self.max_rows, self.classes = max_rows, classes
        nbytes = c_size_t(0)
        _check(self.lib.ngsgd_cross_entropy_workspace_bytes(max_rows, classes, byref(nbytes)), "ngsgd_cross_entropy_workspace_bytes")
        self.workspace_bytes = nbytes.value
        self.workspace = torch.empty(nbytes.value, dtype=torch.uint8, device="cuda")
        self.device = self.workspace.device
        self._home = _raw_stream(None, self.device)

    def _rows(self, t, name, labels, n):
        shape = t.shape
        if len(shape) != 2 or labels.dim() != 1:
            if shape != labels.shape + (self.classes,):
                raise ValueError(f"{name} has the shape {tuple(shape)}, not {tuple(labels.shape) + (self.classes,)}")
            t = t.view(-1, self.classes) if n else t.new_empty(0, self.classes)
        return _matrix(t, name, self.device, n, self.classes)

    def _call(self, logits, labels, scale, loss, dlogits, wants_gradient, stream):
        _current_device(self.device)
        index = _index_type(labels, "labels", self.device)
        n = labels.numel()
        if n > self.max_rows:
            raise ValueError(f"more than {self.max_rows} rows")
        type_, ld, ldd = _type_of(logits.dtype), self._rows(logits, "logits", labels, n), self.classes
        if loss is not None:
            _check_dense(loss, "loss", self.device, _torch.float32, n)
        if dlogits is not None:
            if dlogits.dtype != logits.dtype:
                raise ValueError(f"dlogits is {dlogits.dtype}, not {logits.dtype}")
            ldd = self._rows(dlogits, "dlogits", labels, n)
        dev_scale = None
        if isinstance(scale, _torch.Tensor):
            _check_dense(scale, "scale", self.device, _torch.float32, 1)
            scale, dev_scale = 1.0, scale.data_ptr()
        if loss is None or (wants_gradient and dlogits is None):
            with _allocate_on(stream):
                if loss is None:
                    loss = _torch.empty(labels.shape, dtype=_torch.float32, device=self.device)
                if wants_gradient and dlogits is None:
                    dlogits = _torch.empty_like(logits, memory_format=_torch.contiguous_format)
        _check(self.lib.ngsgd_cross_entropy(logits.data_ptr(), ld, type_, labels.data_ptr(), index, n, self.classes, loss.data_ptr(), scale,
                                            dev_scale, _address(dlogits), ldd, self.workspace.data_ptr(), self.workspace_bytes,
                                            _raw_stream(stream, self.device, self.workspace, self._home)), "ngsgd_cross_entropy")
        return loss, dlogits

    def forward(self, logits, labels, loss=None, stream=None):
        """The loss of each row, float32 of the labels' shape, into `loss` if given."""
        return self._call(logits, labels, 1.0, loss, None, False, stream)[0]

    def gradient(self, logits, labels, scale=1.0, loss=None, dlogits=None, stream=None):
        """(loss, dlogits): the loss of each row, and the gradient of `scale` times their sum, into `dlogits` if given (which may be the
        logits).  scale is a number or a float32 tensor of one element on the device."""
        return self._call(logits, labels, scale, loss, dlogits, True, stream)


class GradientNorm:
    """ngsgd_grad_norm / ngsgd_grad_clip: the norm of many gradients as one vector, and clipping, on the current device.

    `like` are tensors of the gradients' sizes (the parameters, or the gradients themselves): only their sizes, device and type are taken.
    grad_dtype is the gradients' type, `like`'s if none is given.  Calls on one object are issued in order on one stream: the
    workspace is shared.  As with torch's own operators, tensors that are given to a call on another stream than their own are the
    caller's to keep until it has run (torch.Tensor.record_stream)."""

    def __init__(self, like, grad_dtype=None):
        import torch
        self.lib = _library()
        _load_helper()
        like = list(like)
        n = len(like)
        if n == 0:
            raise ValueError("no tensors")
        if not like[0].is_cuda:
            raise ValueError("the tensors are not on the GPU")
        self.device = like[0].device
        _current_device(self.device)
        for i, p in enumerate(like):
            if p.device != self.device:
                raise ValueError(f"tensor {i} is on {p.device}, not on {self.device}")
        self.grad_dtype = like[0].dtype if grad_dtype is None else grad_dtype
        self.type = _type_of(self.grad_dtype)
        self.sizes = [p.numel() for p in like]
        self._sizes = array("q", self.sizes).tobytes()
        self._like = torch.empty(0, dtype=self.grad_dtype)
        nbytes = c_size_t(0)
        _check(self.lib.ngsgd_grad_norm_workspace_bytes(n, byref(nbytes)), "ngsgd_grad_norm_workspace_bytes")
        self.workspace_bytes = nbytes.value
        self.workspace = torch.empty(nbytes.value, dtype=torch.uint8, device=self.device)
        self._home = _raw_stream(None, self.device)

    def _addresses(self, tensors, name):
        """The tensors' addresses as bytes (0: does not count)."""
        if len(tensors) != len(self.sizes):
            raise ValueError(f"{len(tensors)} {name}s for {len(self.sizes)} tensors")
        found = _tensors.addresses(tensors, self._sizes, self._like, self.device.index)
        if found is None:
            for i, (t, size) in enumerate(zip(tensors, self.sizes)):
                if t is None or size == 0:
                    continue
                if t.dtype != self.grad_dtype or t.numel() != size or t.get_device() != self.device.index or not t.is_contiguous():
                    raise ValueError(f"{name} {i}: {t.dtype}, {t.numel()} elements on {t.device}, for {self.grad_dtype}, {size} on "
                                     f"{self.device}, dense")
            raise ValueError(f"a {name} has no memory of its own")
        return found

    def _results(self, norm, factor, stream):
        for name, t in (("norm", norm), ("factor", factor)):
            if t is not None:
                _check_dense(t, name, self.device, _torch.float32, 1)
        if norm is None or factor is None:
            with _allocate_on(stream):
                if norm is None:
                    norm = _torch.empty(1, dtype=_torch.float32, device=self.device)
                if factor is None:
                    factor = _torch.empty(1, dtype=_torch.float32, device=self.device)
        return norm, factor

    def norm(self, grads, max_norm=float("inf"), norm=None, factor=None, stream=None):
        """(norm, factor), float32 tensors of one element: the norm of all gradients, and max_norm / norm where the norm is above max_norm, else 1, which
        AdamW.step takes as grad_scale.  grads: a dense tensor of grad_dtype for each size, or None for one that does not count."""
        _current_device(self.device)
        grads = self._addresses(grads, "gradient")
        norm, factor = self._results(norm, factor, stream)
        _check(self.lib.ngsgd_grad_norm(len(self.sizes), self._sizes, grads, self.type, max_norm, norm.data_ptr(), factor.data_ptr(),
                                        self.workspace.data_ptr(), self.workspace_bytes,
                                        _raw_stream(stream, self.device, self.workspace, self._home)), "ngsgd_grad_norm")
        return norm, factor

    def clip(self, grads, max_norm, out=None, norm=None, factor=None, stream=None):
        """(norm, factor); every gradient is multiplied by the factor, in place or into `out` (a tensor for each gradient, which may be it)."""
        _current_device(self.device)
        if out is not None:
            if len(out) != len(grads) or any(o is None and g is not None and n != 0 for o, g, n in zip(out, grads, self.sizes)):
                raise ValueError("out has no tensor for a gradient")
            out = self._addresses(out, "output")
        grads = self._addresses(grads, "gradient")
        norm, factor = self._results(norm, factor, stream)
        _check(self.lib.ngsgd_grad_clip(len(self.sizes), self._sizes, grads, self.type, max_norm,
                                        out, norm.data_ptr(), factor.data_ptr(),
                                        self.workspace.data_ptr(), self.workspace_bytes,
                                        _raw_stream(stream, self.device, self.workspace, self._home)), "ngsgd_grad_clip")
        return norm, factor


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
        self.lib = _library()
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
        self.lib = _library()
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
    _check(_library().ngsgd_profile_enable(1 if on else 0), "ngsgd_profile_enable")


def profile_read():
    """{category: (milliseconds, bracketed launch groups)} since the last read."""
    n = len(PROFILE_CATEGORIES)
    ms = (c_double * n)()
    cnt = (c_int64 * n)()
    _check(_library().ngsgd_profile_read(ms, cnt, n), "ngsgd_profile_read")
    return {name: (ms[i], cnt[i]) for i, name in enumerate(PROFILE_CATEGORIES)}


def set_wait_limit_us(microseconds: int) -> None:
    """ngsgd_set_wait_limit_us: bound of the waits between workgroups (fused apply kernel, first factors)."""
    _check(_library().ngsgd_set_wait_limit_us(int(microseconds)), "ngsgd_set_wait_limit_us")


def average(networks, reset_preconditioners=True, stream=None):
    """ngsgd_average over replicas living on the same device."""
    lib = _library()
    arr = (c_void_p * len(networks))(*[n.handle for n in networks])
    _check(lib.ngsgd_average(arr, len(networks), 1 if reset_preconditioners else 0, _stream_ptr(stream)),
           "ngsgd_average")
