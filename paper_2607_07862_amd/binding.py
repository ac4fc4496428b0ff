"""ctypes binding of ``libmlp2.so`` (the C ABI in ``include/mlp2.h``).

Argument marshalling only: every step of the computation runs in the HIP
kernels of the library.  PyTorch supplies device memory and the stream.  When
the compiled library is missing, ``load()`` raises: there is no fallback.
"""
from __future__ import annotations

import ctypes
import os

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libmlp2.so")
TRACE_LIB_PATH = os.path.join(PKG, "libmlp2_trace.so")

ACT_IDENTITY, ACT_GELU_TANH, ACT_SWIGLU = 0, 1, 2
DTYPE_BF16, DTYPE_F32 = 0, 1
MODE_SEQUENTIAL, MODE_TILE_PIPELINED, MODE_WORKQUEUE, MODE_STAGE1, MODE_STAGE2, MODE_SENTINEL = 0, 1, 2, 3, 4, 5
MODES = {"sequential": MODE_SEQUENTIAL, "tile_pipelined": MODE_TILE_PIPELINED, "workqueue": MODE_WORKQUEUE,
         "stage1": MODE_STAGE1, "stage2": MODE_STAGE2, "sentinel": MODE_SENTINEL}
ORDER_AUTO, ORDER_COLUMN_FIRST, ORDER_ROW_FIRST, ORDER_REVERSED, ORDER_SHUFFLED, ORDER_BANDED = 0, 1, 2, 3, 4, 5
OPT_SPIN_LIMIT, OPT_DROP_SIGNAL, OPT_ORDER, OPT_GRID = 1, 2, 3, 4

OK = 0
ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_ALIGNMENT, ERR_HIP, ERR_TIMEOUT, ERR_DEVICE = -1, -2, -3, -4, -5, -6

# Every symbol include/mlp2.h declares.
EXPORTS = (
    "mlp2_plan",
    "mlp2_plan_ex",
    "mlp2_run",
    "mlp2_destroy",
    "mlp2_last_error",
    "mlp2_strerror",
    "mlp2_check",
    "mlp2_plan_info",
    "mlp2_intermediate",
    "mlp2_set_option",
    "mlp2_trace_attach",
    "mlp2_chain_plan",
    "mlp2_chain_run",
    "mlp2_chain_check",
    "mlp2_chain_set_spin_limit",
    "mlp2_chain_destroy",
    "mlp2_chain_grid",
    "mlp2_chain_trace_attach",
    "mlp2_run_noalloc",
    "mlp2_train_plan",
    "mlp2_train_forward",
    "mlp2_train_backward",
    "mlp2_train_destroy",
    "mlp2_norm_plan",
    "mlp2_norm_forward",
    "mlp2_norm_backward",
    "mlp2_norm_destroy",
    "mlp2_ortho_plan",
    "mlp2_ortho_run",
    "mlp2_ortho_destroy",
)


class Tuning(ctypes.Structure):
    _fields_ = [
        ("bm", ctypes.c_int),
        ("bn1", ctypes.c_int),
        ("splitk1", ctypes.c_int),
        ("bn2", ctypes.c_int),
        ("splitk2", ctypes.c_int),
        ("grid", ctypes.c_int),
        ("order", ctypes.c_int),
        ("stages", ctypes.c_int),
        ("row_group", ctypes.c_int),
        ("waves", ctypes.c_int),
        ("lag", ctypes.c_int),
        ("p1", ctypes.c_int),
        ("bk", ctypes.c_int),
        ("weights_nt", ctypes.c_int),
    ]


class Info(ctypes.Structure):
    _fields_ = [
        ("M", ctypes.c_int64),
        ("H", ctypes.c_int64),
        ("F", ctypes.c_int64),
        ("act", ctypes.c_int),
        ("bm", ctypes.c_int),
        ("bn1", ctypes.c_int),
        ("splitk1", ctypes.c_int),
        ("bn2", ctypes.c_int),
        ("splitk2", ctypes.c_int),
        ("bk", ctypes.c_int),
        ("row_blocks", ctypes.c_int),
        ("col_blocks1", ctypes.c_int),
        ("col_blocks2", ctypes.c_int),
        ("items1", ctypes.c_int),
        ("items2", ctypes.c_int),
        ("grid_pipelined", ctypes.c_int),
        ("occupancy", ctypes.c_int),
        ("num_cus", ctypes.c_int),
        ("order", ctypes.c_int),
        ("workspace_bytes", ctypes.c_int64),
        ("spin_limit", ctypes.c_uint32),
        ("stages", ctypes.c_int),
        ("grid_gemm1", ctypes.c_int),
        ("grid_gemm2", ctypes.c_int),
        ("row_group", ctypes.c_int),
        ("waves", ctypes.c_int),
        ("lag", ctypes.c_int),
        ("p1", ctypes.c_int),
        ("weights_nt", ctypes.c_int),
    ]


class Mlp2Error(RuntimeError):
    def __init__(self, code: int, what: str):
        self.code = code
        super().__init__(f"{what}: {strerror(code)} ({code})")


_lib = None


def load(path: str | None = None) -> ctypes.CDLL:
    """Load the compiled library (raises if it was not built).

    The first call loads the product library ``libmlp2.so`` unless ``path``
    names another build (the timing-trace tool passes ``TRACE_LIB_PATH``);
    later calls without a path return the loaded one.  A process holds one
    library: asking for a different path after the first load raises.
    """
    global _lib
    if _lib is not None:
        if path is not None and os.path.abspath(_lib._name) != os.path.abspath(path):
            raise RuntimeError(f"{_lib._name} is already loaded; cannot also load {path}")
        return _lib
    if path is None:
        path = LIB_PATH
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -m paper_2607_07862_amd.build`")
    lib = ctypes.CDLL(path)
    P = ctypes.c_void_p
    lib.mlp2_plan.restype = P
    lib.mlp2_plan.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int, ctypes.c_int]
    lib.mlp2_plan_ex.restype = P
    lib.mlp2_plan_ex.argtypes = lib.mlp2_plan.argtypes + [ctypes.POINTER(Tuning)]
    lib.mlp2_run.restype = ctypes.c_int
    lib.mlp2_run.argtypes = [P, P, P, P, P, P, ctypes.c_int]
    lib.mlp2_destroy.restype = None
    lib.mlp2_destroy.argtypes = [P]
    lib.mlp2_last_error.restype = ctypes.c_int
    lib.mlp2_last_error.argtypes = []
    lib.mlp2_strerror.restype = ctypes.c_char_p
    lib.mlp2_strerror.argtypes = [ctypes.c_int]
    lib.mlp2_check.restype = ctypes.c_int
    lib.mlp2_check.argtypes = [P]
    lib.mlp2_plan_info.restype = ctypes.c_int
    lib.mlp2_plan_info.argtypes = [P, ctypes.POINTER(Info)]
    lib.mlp2_intermediate.restype = P
    lib.mlp2_intermediate.argtypes = [P]
    lib.mlp2_set_option.restype = ctypes.c_int
    lib.mlp2_set_option.argtypes = [P, ctypes.c_int, ctypes.c_int64]
    lib.mlp2_trace_attach.restype = ctypes.c_int
    lib.mlp2_trace_attach.argtypes = [P, P, ctypes.c_int]
    lib.mlp2_chain_plan.restype = P
    lib.mlp2_chain_plan.argtypes = [ctypes.c_int64, ctypes.c_int, ctypes.POINTER(ctypes.c_int64), ctypes.c_int, ctypes.c_int]
    lib.mlp2_chain_run.restype = ctypes.c_int
    lib.mlp2_chain_run.argtypes = [P, P, ctypes.POINTER(P), P, P, ctypes.c_int]
    lib.mlp2_chain_check.restype = ctypes.c_int
    lib.mlp2_chain_check.argtypes = [P]
    lib.mlp2_chain_set_spin_limit.restype = ctypes.c_int
    lib.mlp2_chain_set_spin_limit.argtypes = [P, ctypes.c_int64]
    lib.mlp2_chain_grid.restype = ctypes.c_int
    lib.mlp2_chain_grid.argtypes = [P]
    lib.mlp2_chain_trace_attach.restype = ctypes.c_int
    lib.mlp2_chain_trace_attach.argtypes = [P, P, ctypes.c_int]
    lib.mlp2_chain_destroy.restype = None
    lib.mlp2_chain_destroy.argtypes = [P]
    lib.mlp2_run_noalloc.restype = ctypes.c_int
    lib.mlp2_run_noalloc.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int, ctypes.c_int,
                                     P, P, P, P, P, ctypes.c_int]
    I64, F32 = ctypes.c_int64, ctypes.c_float
    for name in ("train", "norm", "ortho"):
        getattr(lib, f"mlp2_{name}_plan").restype = P
        getattr(lib, f"mlp2_{name}_destroy").restype = None
        getattr(lib, f"mlp2_{name}_destroy").argtypes = [P]
    lib.mlp2_train_plan.argtypes = [I64, I64, I64, ctypes.c_int, ctypes.c_int]
    lib.mlp2_train_forward.restype = ctypes.c_int
    lib.mlp2_train_forward.argtypes = [P, I64] + [P] * 6
    lib.mlp2_train_backward.restype = ctypes.c_int
    lib.mlp2_train_backward.argtypes = [P, I64] + [P] * 9
    lib.mlp2_norm_plan.argtypes = [I64, I64, ctypes.c_int, ctypes.c_int]
    lib.mlp2_norm_forward.restype = ctypes.c_int
    lib.mlp2_norm_forward.argtypes = [P, I64, P, I64, P, P, F32, P, I64, P, P, P]
    lib.mlp2_norm_backward.restype = ctypes.c_int
    lib.mlp2_norm_backward.argtypes = [P, I64, P, I64, P, I64, P, P, P, P, I64, P, P, P]
    lib.mlp2_ortho_plan.argtypes = [I64, I64, I64, ctypes.c_int]
    lib.mlp2_ortho_run.restype = ctypes.c_int
    lib.mlp2_ortho_run.argtypes = [P, P, P, ctypes.c_int, ctypes.POINTER(F32), F32, P]
    _lib = lib
    return lib


def loaded_path() -> str | None:
    """Path of the library this process has loaded, or None."""
    return None if _lib is None else _lib._name


def strerror(code: int) -> str:
    return load().mlp2_strerror(int(code)).decode()


def _ptr(t) -> int:
    return 0 if t is None else int(t.data_ptr())


def _check_tensor(t, name, numel, device):
    import torch

    if t.dtype != torch.bfloat16:
        raise TypeError(f"{name} must be bfloat16")
    if not t.is_cuda or t.device != device:
        raise ValueError(f"{name} must live on {device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if t.numel() != numel:
        raise ValueError(f"{name} must hold {numel} elements, has {t.numel()}")


class Plan:
    """A plan for ``Y[M,H] = act(X[M,H] @ W1) @ W2`` on the current device."""

    def __init__(self, M: int, H: int, F: int, act: int, tuning: dict | None = None):
        import torch

        self.lib = load()
        self.M, self.H, self.F, self.act = int(M), int(H), int(F), int(act)
        self.device = torch.device("cuda", torch.cuda.current_device())
        if tuning:
            t = Tuning()
            for k, v in tuning.items():
                setattr(t, k, int(v))
            h = self.lib.mlp2_plan_ex(self.M, self.H, self.F, self.act, DTYPE_BF16, ctypes.byref(t))
        else:
            h = self.lib.mlp2_plan(self.M, self.H, self.F, self.act, DTYPE_BF16)
        if not h:
            raise Mlp2Error(self.lib.mlp2_last_error(), "mlp2_plan")
        self.handle = ctypes.c_void_p(h)

    def close(self):
        if getattr(self, "handle", None):
            self.lib.mlp2_destroy(self.handle)
            self.handle = None

    def __del__(self):  # pragma: no cover - best effort
        try:
            self.close()
        except Exception:
            pass

    def run(self, X, W1, W2, Y, mode, stream=None) -> None:
        """Enqueue one evaluation on ``stream`` (default: torch's current stream)."""
        import torch

        n1 = 2 if self.act == ACT_SWIGLU else 1
        _check_tensor(X, "X", self.M * self.H, self.device)
        _check_tensor(W1, "W1", n1 * self.H * self.F, self.device)
        _check_tensor(W2, "W2", self.F * self.H, self.device)
        _check_tensor(Y, "Y", self.M * self.H, self.device)
        mode = MODES.get(mode, mode)
        if stream is None:
            stream = torch.cuda.current_stream(self.device)
        sp = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
        rc = self.lib.mlp2_run(self.handle, _ptr(X), _ptr(W1), _ptr(W2), _ptr(Y), sp, int(mode))
        if rc != OK:
            raise Mlp2Error(rc, "mlp2_run")

    def run_raw(self, X: int, W1: int, W2: int, Y: int, stream: int, mode: int) -> int:
        """The C call with raw integers (no checks here), returning its status."""
        return self.lib.mlp2_run(self.handle, X, W1, W2, Y, stream, mode)

    def check(self) -> int:
        return self.lib.mlp2_check(self.handle)

    def info(self) -> dict:
        i = Info()
        rc = self.lib.mlp2_plan_info(self.handle, ctypes.byref(i))
        if rc != OK:
            raise Mlp2Error(rc, "mlp2_plan_info")
        return {f: getattr(i, f) for f, _ in Info._fields_}

    def set_option(self, key: int, value: int) -> None:
        rc = self.lib.mlp2_set_option(self.handle, int(key), int(value))
        if rc != OK:
            raise Mlp2Error(rc, "mlp2_set_option")

    def attach_trace(self, buffer, records_per_group: int) -> None:
        """Attach a device uint64/int64 tensor as the timing-trace buffer (trace builds only)."""
        rc = self.lib.mlp2_trace_attach(self.handle, _ptr(buffer), int(records_per_group))
        if rc != OK:
            raise Mlp2Error(rc, "mlp2_trace_attach")

    def intermediate_ptr(self) -> int:
        return int(self.lib.mlp2_intermediate(self.handle) or 0)

    def intermediate(self):
        """A copy of the plan's bf16 Z as a torch tensor [row_blocks*bm, F] (synchronises)."""
        import torch

        info = self.info()
        rows = info["row_blocks"] * info["bm"]
        out = torch.empty(rows, self.F, dtype=torch.bfloat16, device=self.device)
        torch.cuda.synchronize(self.device)
        _hip_memcpy_d2d(out.data_ptr(), self.intermediate_ptr(), rows * self.F * 2)
        return out


_hip = None


def _hip_memcpy_d2d(dst: int, src: int, nbytes: int) -> None:
    global _hip
    if _hip is None:
        _hip = ctypes.CDLL("libamdhip64.so")
        _hip.hipMemcpy.restype = ctypes.c_int
        _hip.hipMemcpy.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int]
    rc = _hip.hipMemcpy(dst, src, nbytes, 3)  # hipMemcpyDeviceToDevice
    if rc != 0:
        raise RuntimeError(f"hipMemcpy failed ({rc})")


def run_noalloc(X, W1, W2, Y, act: int, mode, stream=None) -> None:
    """``mlp2_run_noalloc``: one evaluation with the library's static device
    workspace (no allocation; shapes from X [M,H] and W1 [H,F] / [2,H,F])."""
    import torch

    lib = load()
    M, H = int(X.shape[0]), int(X.shape[1])
    F = int(W1.shape[-1])
    n1 = 2 if act == ACT_SWIGLU else 1
    dev = X.device
    _check_tensor(X, "X", M * H, dev)
    _check_tensor(W1, "W1", n1 * H * F, dev)
    _check_tensor(W2, "W2", F * H, dev)
    _check_tensor(Y, "Y", M * H, dev)
    mode = MODES.get(mode, mode)
    if stream is None:
        stream = torch.cuda.current_stream(dev)
    sp = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    rc = lib.mlp2_run_noalloc(M, H, F, int(act), DTYPE_BF16, _ptr(X), _ptr(W1), _ptr(W2), _ptr(Y), sp, int(mode))
    if rc != OK:
        raise Mlp2Error(rc, "mlp2_run_noalloc")


class ChainPlan:
    """A plan for the GEMM chain ``Z_l = act(Z_{l-1} @ W_l)``, ``Y = Z_{L-1} @ W_L`` (dims = [D_0, ..., D_L])."""

    def __init__(self, M: int, dims, act: int):
        import torch

        self.lib = load()
        self.M, self.dims, self.act = int(M), [int(d) for d in dims], int(act)
        self.L = len(self.dims) - 1
        self.device = torch.device("cuda", torch.cuda.current_device())
        arr = (ctypes.c_int64 * len(self.dims))(*self.dims)
        h = self.lib.mlp2_chain_plan(self.M, self.L, arr, self.act, DTYPE_BF16)
        if not h:
            raise Mlp2Error(self.lib.mlp2_last_error(), "mlp2_chain_plan")
        self.handle = ctypes.c_void_p(h)

    def close(self):
        if getattr(self, "handle", None):
            self.lib.mlp2_chain_destroy(self.handle)
            self.handle = None

    def __del__(self):  # pragma: no cover - best effort
        try:
            self.close()
        except Exception:
            pass

    def run(self, X, Ws, Y, mode, stream=None) -> None:
        """Enqueue one evaluation on ``stream`` (default: torch's current stream)."""
        import torch

        if len(Ws) != self.L:
            raise ValueError(f"expected {self.L} weights")
        _check_tensor(X, "X", self.M * self.dims[0], self.device)
        for l, W in enumerate(Ws):
            _check_tensor(W, f"W{l + 1}", self.dims[l] * self.dims[l + 1], self.device)
        _check_tensor(Y, "Y", self.M * self.dims[-1], self.device)
        mode = MODES.get(mode, mode)
        if stream is None:
            stream = torch.cuda.current_stream(self.device)
        sp = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
        ptrs = (ctypes.c_void_p * self.L)(*[_ptr(W) for W in Ws])
        rc = self.lib.mlp2_chain_run(self.handle, _ptr(X), ptrs, _ptr(Y), sp, int(mode))
        if rc != OK:
            raise Mlp2Error(rc, "mlp2_chain_run")

    def check(self) -> int:
        return self.lib.mlp2_chain_check(self.handle)

    def grid(self) -> int:
        return int(self.lib.mlp2_chain_grid(self.handle))

    def attach_trace(self, buffer, records_per_group: int) -> None:
        """Attach a device int64 tensor as the timing-trace buffer (trace builds only)."""
        rc = self.lib.mlp2_chain_trace_attach(self.handle, _ptr(buffer), int(records_per_group))
        if rc != OK:
            raise Mlp2Error(rc, "mlp2_chain_trace_attach")

    def set_spin_limit(self, polls: int) -> None:
        rc = self.lib.mlp2_chain_set_spin_limit(self.handle, int(polls))
        if rc != OK:
            raise Mlp2Error(rc, "mlp2_chain_set_spin_limit")


def _stream(stream, device) -> int:
    import torch

    if stream is None:
        stream = torch.cuda.current_stream(device)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _dtype_code(dtype) -> int:
    import torch

    codes = {torch.bfloat16: DTYPE_BF16, torch.float32: DTYPE_F32}
    if dtype not in codes:
        raise TypeError(f"{dtype} is not supported: bfloat16 or float32")
    return codes[dtype]


def _check_shape(t, name, shape, dtype, device, rows=False):
    """``t`` is a ``dtype`` tensor of ``shape`` on ``device``; contiguous, or with ``rows`` a matrix of contiguous rows."""
    if t.dtype == dtype and t.shape == shape and t.device == device and t.is_contiguous():
        return  # (the smallest calls last no longer than a dozen such checks)
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, is {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} must live on {device}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, has {tuple(t.shape)}")
    if rows:
        if (t.shape[1] > 1 and t.stride(1) != 1) or (t.shape[0] > 1 and t.stride(0) < t.shape[1]):
            raise ValueError(f"{name}'s rows must be contiguous and apart from each other")
    else:
        raise ValueError(f"{name} must be contiguous")


def _row_stride(t) -> int:
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


class _Owned:
    """A plan handle, freed with its object."""

    _name = ""

    def _create(self, *args):
        import torch

        self.lib = load()
        self.device = torch.device("cuda", torch.cuda.current_device())
        self._bf16, self._f32 = torch.bfloat16, torch.float32
        # torch's own call for the current stream's handle; torch.cuda.current_stream() makes an object of it first
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        h = getattr(self.lib, f"mlp2_{self._name}_plan")(*args)
        if not h:
            raise Mlp2Error(self.lib.mlp2_last_error(), f"mlp2_{self._name}_plan")
        self.handle = ctypes.c_void_p(h)

    def close(self):
        if getattr(self, "handle", None):
            getattr(self.lib, f"mlp2_{self._name}_destroy")(self.handle)
            self.handle = None

    def __del__(self):  # pragma: no cover - best effort
        try:
            self.close()
        except Exception:
            pass

    def _on(self, stream) -> int:
        if stream is None and self._raw_stream is not None:
            return self._raw_stream(self.device.index)
        return _stream(stream, self.device)

    def _done(self, rc, call):
        if rc != OK:
            raise Mlp2Error(rc, f"mlp2_{self._name}_{call}")


class TrainPlan(_Owned):
    """Training of ``Y = act(X @ W1) @ W2`` with up to ``max_rows`` rows a call, on the current device.

    ``W1`` is ``[H, F]``, for SwiGLU ``[2, H, F]``; ``forward`` also writes the
    pre-activations ``P`` (``[M, F]`` or ``[2, M, F]``) that ``backward`` takes.
    A leading 1 in ``W1``, ``P`` and ``dW1`` of an MLP without gate is accepted.
    """

    _name = "train"

    def __init__(self, max_rows: int, H: int, F: int, act: int):
        self.max_rows, self.H, self.F, self.act = int(max_rows), int(H), int(F), int(act)
        self._create(self.max_rows, self.H, self.F, self.act, DTYPE_BF16)

    def _check(self, t, name, *shape):
        lead = 2 if self.act == ACT_SWIGLU else 1
        if name in ("W1", "P", "dW1") and (lead == 2 or t.dim() == 3):
            shape = (lead,) + shape
        _check_shape(t, name, shape, self._bf16, self.device)

    def forward(self, X, W1, W2, P, Y, stream=None) -> None:
        """Enqueue ``P = X @ W1`` and ``Y = act(P) @ W2`` on ``stream`` (default: torch's current stream)."""
        M, H, F = int(X.shape[0]), self.H, self.F
        for t, name, shape in ((X, "X", (M, H)), (W1, "W1", (H, F)), (W2, "W2", (F, H)), (P, "P", (M, F)), (Y, "Y", (M, H))):
            self._check(t, name, *shape)
        self._done(self.lib.mlp2_train_forward(self.handle, M, _ptr(X), _ptr(W1), _ptr(W2), _ptr(P), _ptr(Y),
                                               self._on(stream)), "forward")

    def backward(self, dY, X, W1, W2, P, dX=None, dW1=None, dW2=None, stream=None) -> None:
        """Enqueue the gradients that are asked for (None: not computed)."""
        M, H, F = int(X.shape[0]), self.H, self.F
        for t, name, shape in ((dY, "dY", (M, H)), (X, "X", (M, H)), (W1, "W1", (H, F)), (W2, "W2", (F, H)), (P, "P", (M, F)),
                               (dX, "dX", (M, H)), (dW1, "dW1", (H, F)), (dW2, "dW2", (F, H))):
            if t is not None or not name.startswith(("dX", "dW")):
                self._check(t, name, *shape)
        if M == 0 and dX is not None and dW1 is None and dW2 is None:
            return  # (an empty tensor's pointer is null, which the library takes for a gradient that is not asked for)
        self._done(self.lib.mlp2_train_backward(self.handle, M, _ptr(dY), _ptr(X), _ptr(W1), _ptr(W2), _ptr(P), _ptr(dX),
                                                _ptr(dW1), _ptr(dW2), self._on(stream)), "backward")


class NormPlan(_Owned):
    """Layer norm over rows of ``H`` elements, up to ``max_rows`` rows a call, on the current device.

    ``x_dtype`` is the type of ``X`` and ``dX``, ``y_dtype`` (default: the same)
    that of ``Y`` and ``dY``; everything else is float32.  Matrices may have any
    row stride, and may be columns of one buffer.
    """

    _name = "norm"

    def __init__(self, max_rows: int, H: int, x_dtype=None, y_dtype=None):
        import torch

        self.max_rows, self.H = int(max_rows), int(H)
        self.x_dtype = torch.bfloat16 if x_dtype is None else x_dtype
        self.y_dtype = self.x_dtype if y_dtype is None else y_dtype
        self._create(self.max_rows, self.H, _dtype_code(self.x_dtype), _dtype_code(self.y_dtype))

    def _vector(self, t, name, n):
        if t is not None:
            _check_shape(t, name, (n,), self._f32, self.device)

    def forward(self, X, weight, bias, Y, mean=None, rstd=None, eps=1e-5, stream=None) -> None:
        """Enqueue ``Y = (X - mean) * rstd * weight + bias`` (None: no weight, no bias, statistics not written)."""
        M, H = X.shape[0], self.H
        _check_shape(X, "X", (M, H), self.x_dtype, self.device, rows=True)
        _check_shape(Y, "Y", (M, H), self.y_dtype, self.device, rows=True)
        self._vector(weight, "weight", H)
        self._vector(bias, "bias", H)
        self._vector(mean, "mean", M)
        self._vector(rstd, "rstd", M)
        self._done(self.lib.mlp2_norm_forward(self.handle, M, _ptr(X), _row_stride(X), _ptr(weight), _ptr(bias), float(eps),
                                              _ptr(Y), _row_stride(Y), _ptr(mean), _ptr(rstd),
                                              self._on(stream)), "forward")

    def backward(self, dY, X, weight, mean, rstd, dX, dweight=None, dbias=None, stream=None) -> None:
        """Enqueue the gradients of X, and of weight and bias where asked for."""
        M, H = X.shape[0], self.H
        _check_shape(dY, "dY", (M, H), self.y_dtype, self.device, rows=True)
        _check_shape(X, "X", (M, H), self.x_dtype, self.device, rows=True)
        _check_shape(dX, "dX", (M, H), self.x_dtype, self.device, rows=True)
        self._vector(weight, "weight", H)
        self._vector(mean, "mean", M)
        self._vector(rstd, "rstd", M)
        self._vector(dweight, "dweight", H)
        self._vector(dbias, "dbias", H)
        self._done(self.lib.mlp2_norm_backward(self.handle, M, _ptr(dY), _row_stride(dY), _ptr(X), _row_stride(X), _ptr(weight),
                                               _ptr(mean), _ptr(rstd), _ptr(dX), _row_stride(dX), _ptr(dweight), _ptr(dbias),
                                               self._on(stream)), "backward")


#: The quintic of the Muon optimiser: five steps bring singular values of (0.003, 1] to about (0.7, 1.2).
ORTHO_COEFFS = (3.4445, -4.7750, 2.0315)


class OrthoPlan(_Owned):
    """Newton-Schulz orthogonalisation of ``count`` matrices ``[rows, cols]`` at a time, on the current device."""

    _name = "ortho"

    def __init__(self, count: int, rows: int, cols: int, dtype=None):
        import torch

        self.shape = (int(count), int(rows), int(cols))
        self.dtype = torch.float32 if dtype is None else dtype
        self._create(*self.shape, _dtype_code(self.dtype))

    def run(self, G, O, steps: int = 5, coeffs=ORTHO_COEFFS, eps: float = 1e-7, stream=None) -> None:
        """Enqueue ``steps`` steps on the matrices G (``[count, rows, cols]``; ``[rows, cols]`` for one) into the bf16 O.

        ``coeffs``: three numbers for every step, or ``steps`` triples."""
        flat = [float(v) for c in coeffs for v in (c if hasattr(c, "__len__") else (c,))]
        if len(flat) == 3:
            flat = flat * int(steps)
        if len(flat) != 3 * int(steps):
            raise ValueError(f"coeffs must hold 3 or {3 * int(steps)} numbers")
        for t, name, dtype in ((G, "G", self.dtype), (O, "O", self._bf16)):
            _check_shape(t, name, self.shape[1:] if self.shape[0] == 1 and t.dim() == 2 else self.shape, dtype, self.device)
        arr = (ctypes.c_float * len(flat))(*flat)
        self._done(self.lib.mlp2_ortho_run(self.handle, _ptr(G), _ptr(O), int(steps), arr, float(eps),
                                           self._on(stream)), "run")
