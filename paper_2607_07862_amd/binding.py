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
DTYPE_BF16, DTYPE_F32, DTYPE_MXFP4 = 0, 1, 2
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
    "mlp2_mx_quantize",
    "mlp2_mx_plan",
    "mlp2_mx_product",
    "mlp2_mx_destroy",
    "mlp2_moe_plan",
    "mlp2_moe_forward",
    "mlp2_moe_experts",
    "mlp2_moe_destroy",
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
    for name in ("train", "norm", "ortho", "mx", "moe"):
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
    lib.mlp2_mx_quantize.restype = ctypes.c_int
    lib.mlp2_mx_quantize.argtypes = [I64, I64, I64, ctypes.c_int, P, ctypes.c_int, I64, I64, P, P, P, P]
    lib.mlp2_mx_plan.argtypes = [I64, I64, I64, ctypes.c_int, ctypes.c_int]
    lib.mlp2_mx_product.restype = ctypes.c_int
    lib.mlp2_mx_product.argtypes = [P, I64] + [P] * 6
    lib.mlp2_moe_plan.argtypes = [I64, I64, I64, I64, I64, ctypes.c_int, ctypes.c_int]
    lib.mlp2_moe_forward.restype = ctypes.c_int
    lib.mlp2_moe_forward.argtypes = [P, I64, P, P, ctypes.c_int] + [P] * 8
    lib.mlp2_moe_experts.restype = ctypes.c_int
    lib.mlp2_moe_experts.argtypes = [P, I64] + [P] * 9
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


_dtype_codes = {}


def _dtype_code(dtype) -> int:
    if not _dtype_codes:
        import torch

        _dtype_codes.update({torch.bfloat16: DTYPE_BF16, torch.float32: DTYPE_F32})
    if dtype not in _dtype_codes:
        raise TypeError(f"{dtype} is not supported: bfloat16 or float32")
    return _dtype_codes[dtype]


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


_calls = None


def _torch_calls():
    """torch's own calls for the current device and its current stream's handle, and bfloat16: the smallest calls last no longer than
    the objects that torch.cuda's functions make of them."""
    global _calls
    if _calls is None:
        import torch

        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
        _calls = (getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device), raw, torch.bfloat16)
    return _calls


def _lib_of():
    return _lib if _lib is not None else load()


def _mx_shapes(rows, K, count):
    groups = -(-K // 128)
    return (count, rows, 64 * groups), (count, groups, rows, 4)


class MxMatrix:
    """``count`` matrices ``[rows, K]`` in MXFP4, K contiguous, on the current device (uninitialised).

    ``codes`` is uint8 ``[count, rows, Kp / 2]`` and ``scales`` uint8 ``[count, Kp / 128, rows, 4]``, Kp being K rounded up to a
    multiple of 128 (the format: ``include/mlp2.h``).  ``mx_quantize`` fills them."""

    def __init__(self, rows: int, K: int, count: int = 1):
        import torch

        self.rows, self.K, self.count = int(rows), int(K), int(count)
        codes, scales = _mx_shapes(self.rows, self.K, self.count)
        self.device = torch.device("cuda", torch.cuda.current_device())
        self.codes = torch.empty(codes, dtype=torch.uint8, device=self.device)
        self.scales = torch.empty(scales, dtype=torch.uint8, device=self.device)

    @classmethod
    def of(cls, codes, scales, K: int) -> "MxMatrix":
        """The matrices that these two tensors hold (not copied).

        Arrays of unpadded rows, codes ``[count, rows, K / 2]`` and one scale after the other ``[count, rows, K / 32]``, become these
        with ``G = -(-K // 128)`` and ``pad = torch.nn.functional.pad``::

            codes = pad(codes, (0, 64 * G - K // 2))
            scales = pad(scales, (0, 4 * G - K // 32)).view(count, rows, G, 4).transpose(1, 2).contiguous()
        """
        import torch

        if codes.dim() != 3:
            raise ValueError(f"codes must have three dimensions, has {codes.dim()}")
        self = cls.__new__(cls)
        self.rows, self.K, self.count = int(codes.shape[1]), int(K), int(codes.shape[0])
        self.device, self.codes, self.scales = codes.device, codes, scales
        if self.device.type != "cuda":
            raise ValueError("codes must live on a GPU")
        want = _mx_shapes(self.rows, self.K, self.count)
        _check_shape(codes, "codes", want[0], torch.uint8, self.device)
        _check_shape(scales, "scales", want[1], torch.uint8, self.device)
        return self


def _check_mx(m, name, rows, K, count, device):
    if not isinstance(m, MxMatrix):
        raise TypeError(f"{name} must be an MxMatrix")
    if m.device != device:
        raise ValueError(f"{name} must live on {device}")
    if (m.rows, m.K, m.count) != (rows, K, count):
        raise ValueError(f"{name} must hold {count} matrices [{rows}, {K}], holds {m.count} of [{m.rows}, {m.K}]")


def mx_quantize(X, out: MxMatrix, values=None, down: bool = False, stream=None) -> None:
    """Enqueue the quantisation of X, bf16 or float32 ``[rows, cols]`` or ``[count, rows, cols]``, into ``out``.

    Blocks of 32 lie along a row, so that ``out`` holds ``[rows, K = cols]``, or with ``down`` down a column: the library's weights
    ``[K, N]`` become ``[N, K]``.  X's rows must be contiguous, at any distance; its matrices may be columns of one buffer.
    ``values`` (bf16, X's shape, contiguous) receives what the codes stand for."""
    device = X.device
    current, raw_stream, bf16 = _torch_calls()
    code = _dtype_code(X.dtype)
    shape, strides = tuple(X.shape), X.stride()
    if len(shape) not in (2, 3):
        raise ValueError(f"X must have two or three dimensions, has {len(shape)}")
    if device.type != "cuda" or device.index != current():
        raise ValueError("X must live on the current device")
    rows, cols = shape[-2:]
    count = shape[0] if len(shape) == 3 else 1
    _check_mx(out, "out", cols if down else rows, rows if down else cols, count, device)
    if values is not None:
        _check_shape(values, "values", shape, bf16, device)
    ld = strides[-2] if rows > 1 else cols
    matrix = strides[0] if count > 1 else rows * ld
    behind = count <= 1 or matrix >= (rows - 1) * ld + cols
    if (cols > 1 and strides[-1] != 1) or ld < cols or not (behind or matrix >= cols and (count - 1) * matrix + cols <= ld):
        raise ValueError("X's rows must be contiguous and apart from each other")
    stream = raw_stream(device.index) if stream is None else _stream(stream, device)
    rc = _lib_of().mlp2_mx_quantize(count, rows, cols, 1 if down else 0, _ptr(X), code, ld, matrix, _ptr(out.codes), _ptr(out.scales),
                                    _ptr(values), stream)
    if rc != OK:
        raise Mlp2Error(rc, "mlp2_mx_quantize")


class MxPlan(_Owned):
    """``Y = act(A @ W.T)`` of MXFP4 matrices A ``[M <= max_rows, K]`` and W ``[N, K]`` (SwiGLU: two of them, gate and up), on the
    current device; ``y_dtype`` is bfloat16 (default) or float32."""

    _name = "mx"

    def __init__(self, max_rows: int, N: int, K: int, act: int = ACT_IDENTITY, y_dtype=None):
        import torch

        self.max_rows, self.N, self.K, self.act = int(max_rows), int(N), int(K), int(act)
        self.y_dtype = torch.bfloat16 if y_dtype is None else y_dtype
        self._create(self.max_rows, self.N, self.K, self.act, _dtype_code(self.y_dtype))

    def product(self, A: MxMatrix, W: MxMatrix, Y, stream=None) -> None:
        """Enqueue the product on ``stream`` (default: torch's current stream)."""
        M = int(Y.shape[0])
        _check_shape(Y, "Y", (M, self.N), self.y_dtype, self.device)
        _check_mx(A, "A", M, self.K, 1, self.device)
        _check_mx(W, "W", self.N, self.K, 2 if self.act == ACT_SWIGLU else 1, self.device)
        self._done(self.lib.mlp2_mx_product(self.handle, M, _ptr(A.codes), _ptr(A.scales), _ptr(W.codes), _ptr(W.scales), _ptr(Y),
                                            self._on(stream)), "product")


class MoePlan(_Owned):
    """A mixture-of-experts layer for up to ``max_tokens`` tokens: the best ``k`` of ``E`` experts of each, two-layer MLPs.

    ``w_dtype``: bfloat16, W1 ``[E, H, F]`` (SwiGLU ``[E, 2, H, F]``) and W2 ``[E, F, H]``, or ``"mxfp4"``, W1 an ``MxMatrix`` of E
    (SwiGLU 2 E) matrices ``[F, K = H]`` and W2 one of E matrices ``[H, K = F]``, as ``mx_quantize(..., down=True)`` makes them."""

    _name = "moe"

    def __init__(self, max_tokens: int, H: int, F: int, E: int, k: int, act: int = ACT_SWIGLU, w_dtype=None):
        import torch

        self.max_tokens, self.H, self.F, self.E, self.k, self.act = int(max_tokens), int(H), int(F), int(E), int(k), int(act)
        self.mx = isinstance(w_dtype, str) and w_dtype == "mxfp4"
        if not self.mx and w_dtype not in (None, torch.bfloat16):
            raise TypeError(f'{w_dtype} is not supported: bfloat16 or "mxfp4"')
        self._i32 = torch.int32
        self._create(self.max_tokens, self.H, self.F, self.E, self.k, self.act, DTYPE_MXFP4 if self.mx else DTYPE_BF16)

    def _check(self, X, W1, W2, Y, ids, gates):
        T, H, F, E = int(X.shape[0]), self.H, self.F, self.E
        gated = self.act == ACT_SWIGLU
        _check_shape(X, "X", (T, H), self._bf16, self.device)
        _check_shape(Y, "Y", (T, H), self._bf16, self.device)
        _check_shape(ids, "ids", (T, self.k), self._i32, self.device)
        _check_shape(gates, "gates", (T, self.k), self._f32, self.device)
        if self.mx:
            _check_mx(W1, "W1", F, H, 2 * E if gated else E, self.device)
            _check_mx(W2, "W2", H, F, E, self.device)
            return T, (_ptr(W1.codes), _ptr(W1.scales), _ptr(W2.codes), _ptr(W2.scales))
        if isinstance(W1, MxMatrix) or isinstance(W2, MxMatrix):
            raise TypeError("W1 and W2 must be bfloat16 tensors")
        _check_shape(W1, "W1", (E, 2, H, F) if gated else (E, 1, H, F) if W1.dim() == 4 else (E, H, F), self._bf16, self.device)
        _check_shape(W2, "W2", (E, F, H), self._bf16, self.device)
        return T, (_ptr(W1), 0, _ptr(W2), 0)

    def forward(self, X, Wr, W1, W2, Y, ids, gates, stream=None) -> None:
        """Enqueue the whole layer: ids ``[T, k]`` (int32) and gates ``[T, k]`` (float32) from the router's weight Wr ``[H, E]``
        (bfloat16 or float32), then Y."""
        T, w = self._check(X, W1, W2, Y, ids, gates)
        code = _dtype_code(Wr.dtype)
        _check_shape(Wr, "Wr", (self.H, self.E), Wr.dtype, self.device)
        self._done(self.lib.mlp2_moe_forward(self.handle, T, _ptr(X), _ptr(Wr), code, *w, _ptr(Y), _ptr(ids), _ptr(gates),
                                             self._on(stream)), "forward")

    def experts(self, X, ids, gates, W1, W2, Y, stream=None) -> None:
        """Enqueue the experts and their weighted sum for the caller's ids (outside ``[0, E)``: an empty slot) and gates."""
        T, w = self._check(X, W1, W2, Y, ids, gates)
        self._done(self.lib.mlp2_moe_experts(self.handle, T, _ptr(X), _ptr(ids), _ptr(gates), *w, _ptr(Y), self._on(stream)), "experts")
