"""Thin ctypes binding of libqmm.so (the C ABI declared in include/qmm.h).

Argument marshalling only (of the shortest hot-path calls in the extension csrc/qmm_py.c,
of the others here): every step of every product runs in the CUDA kernels of the library.  PyTorch is used for device memory and streams.  There
is no CPU fallback: if the shared library cannot be loaded, or a call fails,
an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
import threading

import torch

Q4 = 4
Q5 = 5
Q6 = 6
Q8 = 8

# scores of a router
SOFTMAX = 0
SIGMOID = 1

# microscaled 4-bit floating point (the number of a format is its block length) and element types
MXFP4 = 32
NVFP4 = 16
DTYPES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqmm.so")
_lock = threading.Lock()
_lib = None

STATUS_NAMES = {
    0: "QMM_OK", 1: "QMM_ERR_INVALID_ARG", 2: "QMM_ERR_SHAPE", 3: "QMM_ERR_ALIGNMENT",
    4: "QMM_ERR_WORKSPACE", 5: "QMM_ERR_UNSUPPORTED", 6: "QMM_ERR_CUDA", 7: "QMM_ERR_DEVICE_TIMEOUT",
    8: "QMM_ERR_BAD_WEIGHTS",
}

# every symbol include/qmm.h declares
EXPORTS = (
    "qmm_last_error", "qmm_version", "qmm_canonical_bytes", "qmm_packed_bytes", "qmm_pack",
    "qmm_dequant", "qmm_gemv_workspace_bytes", "qmm_gemv", "qmm_gemm_workspace_bytes", "qmm_gemm",
    "qmm_moe_workspace_bytes", "qmm_moe", "qmm_moe_route", "qmm_status_check", "qmm_gemv_static", "qmm_gemv_batch", "qmm_gemm_batch",
    "qmm_gemv_gate_up", "qmm_packed_check", "qmm_debug_config", "qmm_debug_wait_give_up",
    "qmm_chain_plan_bytes", "qmm_chain_workspace_bytes", "qmm_chain_build", "qmm_chain_run",
    "qmm_mx_bytes", "qmm_mx_pack", "qmm_mx_quantize", "qmm_mx_dequantize", "qmm_mx_gemm_workspace_bytes", "qmm_mx_gemm",
    "qmm_mx_linear_workspace_bytes", "qmm_mx_linear", "qmm_expert_sort_workspace_bytes", "qmm_expert_sort", "qmm_expert_gather",
    "qmm_expert_combine", "qmm_expert_combine_grad", "qmm_mx_experts_bytes", "qmm_mx_quantize_experts", "qmm_mx_experts_gate_up",
    "qmm_mx_experts_gemm", "qmm_mx_moe_workspace_bytes", "qmm_mx_moe",
    "qmm_expert_route", "qmm_expert_route_grad", "qmm_rms_norm", "qmm_rms_norm_grad_workspace_bytes", "qmm_rms_norm_grad",
    "qmm_rows_quantize", "qmm_rows_dequantize", "qmm_lora_workspace_bytes", "qmm_lora", "qmm_lora_grad",
)


class QmmError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("%s: %s" % (STATUS_NAMES.get(status, status), message))
        self.status = status
        self.message = message


class GemvProblem(ctypes.Structure):
    _fields_ = [("packed", ctypes.c_void_p), ("x_fp16", ctypes.c_void_p), ("y_fp16", ctypes.c_void_p),
                ("N", ctypes.c_int64), ("K", ctypes.c_int64)]


class GemmProblem(ctypes.Structure):
    _fields_ = [("packed", ctypes.c_void_p), ("X_fp16", ctypes.c_void_p), ("Y_fp16", ctypes.c_void_p),
                ("N", ctypes.c_int64), ("K", ctypes.c_int64), ("ldx", ctypes.c_int64), ("ldy", ctypes.c_int64)]


class ChainStage(ctypes.Structure):
    _fields_ = [("op", ctypes.c_int32), ("x_stage", ctypes.c_int32), ("x_offset", ctypes.c_int64),
                ("x_fp16", ctypes.c_void_p), ("packed", ctypes.c_void_p), ("packed_up", ctypes.c_void_p),
                ("N", ctypes.c_int64), ("K", ctypes.c_int64), ("y_fp16", ctypes.c_void_p)]


class ChainInfo(ctypes.Structure):
    _fields_ = [("magic", ctypes.c_int32), ("fmt", ctypes.c_int32), ("stages", ctypes.c_int32), ("grid", ctypes.c_int32),
                ("threads", ctypes.c_int32), ("smem_bytes", ctypes.c_int32), ("plan_bytes", ctypes.c_uint64),
                ("ws_bytes", ctypes.c_uint64), ("plan", ctypes.c_void_p), ("ws", ctypes.c_void_p)]


CHAIN_LINEAR = 0
CHAIN_GATE_UP_SILU = 1


class MoeArgs(ctypes.Structure):
    _fields_ = [
        ("T", ctypes.c_int32), ("H", ctypes.c_int32), ("I", ctypes.c_int32), ("E", ctypes.c_int32),
        ("topk", ctypes.c_int32), ("fmt", ctypes.c_int32),
        ("logits", ctypes.c_void_p), ("X", ctypes.c_void_p),
        ("w_gate", ctypes.c_void_p), ("w_up", ctypes.c_void_p), ("w_down", ctypes.c_void_p),
        ("out", ctypes.c_void_p),
        ("topk_idx", ctypes.c_void_p), ("topk_w", ctypes.c_void_p),
        ("perm", ctypes.c_void_p), ("expert_offsets", ctypes.c_void_p),
        ("dbg_H", ctypes.c_void_p), ("dbg_D", ctypes.c_void_p),
        ("w_router", ctypes.c_void_p), ("router_logits", ctypes.c_void_p),
    ]


class MxMoeArgs(ctypes.Structure):
    _fields_ = [
        ("T", ctypes.c_int32), ("H", ctypes.c_int32), ("I", ctypes.c_int32), ("E", ctypes.c_int32), ("topk", ctypes.c_int32),
        ("fmt", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("X", ctypes.c_void_p), ("ldx", ctypes.c_int64), ("idx", ctypes.c_void_p), ("weights", ctypes.c_void_p),
        ("w_gate", ctypes.c_void_p), ("w_up", ctypes.c_void_p), ("w_down", ctypes.c_void_p),
        ("x_scale", ctypes.c_void_p), ("h_scale", ctypes.c_void_p), ("gate_scale", ctypes.c_void_p),
        ("up_scale", ctypes.c_void_p), ("down_scale", ctypes.c_void_p),
        ("out", ctypes.c_void_p), ("ldo", ctypes.c_int64), ("rows_f32", ctypes.c_int32),
    ]


class LoraArgs(ctypes.Structure):
    _fields_ = [
        ("T", ctypes.c_int32), ("n", ctypes.c_int32), ("r", ctypes.c_int32), ("dtype", ctypes.c_int32), ("x_format", ctypes.c_int32),
        ("K", ctypes.c_int64), ("N", ctypes.c_int64), ("X", ctypes.c_void_p), ("ldx", ctypes.c_int64), ("x_scale", ctypes.c_void_p),
        ("idx", ctypes.c_void_p), ("order", ctypes.c_void_p), ("offsets", ctypes.c_void_p), ("units", ctypes.c_void_p),
        ("A", ctypes.c_void_p), ("B", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("S", ctypes.c_void_p),
        ("Y0", ctypes.c_void_p), ("ldy0", ctypes.c_int64), ("Y", ctypes.c_void_p), ("ldy", ctypes.c_int64),
        ("dY", ctypes.c_void_p), ("lddy", ctypes.c_int64), ("dX0", ctypes.c_void_p), ("lddx0", ctypes.c_int64),
        ("dX", ctypes.c_void_p), ("lddx", ctypes.c_int64), ("dA", ctypes.c_void_p), ("dB", ctypes.c_void_p),
    ]


def lib() -> ctypes.CDLL:
    """Load libqmm.so (building it with nvcc first if it is not there)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(LIB_PATH):
                from . import _build
                _build.build_library()
            L = ctypes.CDLL(LIB_PATH)
            i64, vp, ci, sz = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
            L.qmm_last_error.restype = ctypes.c_char_p
            L.qmm_last_error.argtypes = []
            L.qmm_version.restype = ci
            L.qmm_canonical_bytes.restype = sz
            L.qmm_canonical_bytes.argtypes = [ci, i64, i64]
            L.qmm_packed_bytes.restype = sz
            L.qmm_packed_bytes.argtypes = [ci, i64, i64]
            L.qmm_pack.argtypes = [ci, vp, i64, i64, vp, vp]
            L.qmm_dequant.argtypes = [ci, vp, i64, i64, vp, vp]
            L.qmm_gemv_workspace_bytes.restype = sz
            L.qmm_gemv_workspace_bytes.argtypes = [ci, i64, i64]
            L.qmm_gemv.argtypes = [ci, vp, i64, i64, vp, vp, vp, sz, vp]
            L.qmm_gemv_static.argtypes = [ci, vp, i64, i64, vp, vp, vp]
            L.qmm_gemv_gate_up.argtypes = [ci, vp, vp, i64, i64, vp, vp, vp]
            L.qmm_gemv_batch.argtypes = [ci, ctypes.POINTER(GemvProblem), ci, vp]
            L.qmm_gemm_batch.argtypes = [ci, ctypes.POINTER(GemmProblem), ci, i64, vp]
            L.qmm_gemm_workspace_bytes.restype = sz
            L.qmm_gemm_workspace_bytes.argtypes = [ci, i64, i64, i64]
            L.qmm_gemm.argtypes = [ci, vp, i64, i64, vp, i64, vp, i64, i64, vp, sz, vp]
            L.qmm_moe_workspace_bytes.restype = sz
            L.qmm_moe_workspace_bytes.argtypes = [ctypes.POINTER(MoeArgs)]
            L.qmm_moe.argtypes = [ctypes.POINTER(MoeArgs), vp, sz, vp]
            L.qmm_moe_route.argtypes = [ctypes.POINTER(MoeArgs), vp, sz, vp]
            L.qmm_status_check.argtypes = [vp, vp]
            L.qmm_chain_plan_bytes.restype = sz
            L.qmm_chain_plan_bytes.argtypes = [ci, ctypes.POINTER(ChainStage), ci]
            L.qmm_chain_workspace_bytes.restype = sz
            L.qmm_chain_workspace_bytes.argtypes = [ci, ctypes.POINTER(ChainStage), ci]
            L.qmm_chain_build.argtypes = [ci, ctypes.POINTER(ChainStage), ci, vp, sz, vp, sz, ctypes.POINTER(ChainInfo), vp]
            L.qmm_chain_run.argtypes = [ctypes.POINTER(ChainInfo), vp]
            i32 = ctypes.c_int32
            for name in ("qmm_mx_bytes", "qmm_mx_gemm_workspace_bytes", "qmm_mx_linear_workspace_bytes", "qmm_expert_sort_workspace_bytes",
                         "qmm_mx_experts_bytes", "qmm_mx_moe_workspace_bytes", "qmm_rms_norm_grad_workspace_bytes", "qmm_lora_workspace_bytes"):
                getattr(L, name).restype = sz
            L.qmm_mx_bytes.argtypes = [ci, i64, i64]
            L.qmm_mx_pack.argtypes = [ci, vp, vp, i64, i64, vp, vp]
            L.qmm_mx_quantize.argtypes = [ci, ci, vp, i64, i64, i64, vp, vp, vp]
            L.qmm_mx_dequantize.argtypes = [ci, vp, i64, i64, vp, ci, vp, i64, vp]
            L.qmm_mx_gemm_workspace_bytes.argtypes = [ci, i64, i64, i64]
            L.qmm_mx_gemm.argtypes = [ci, vp, i64, vp, i64, i64, vp, vp, ci, vp, i64, vp, sz, vp]
            L.qmm_mx_linear_workspace_bytes.argtypes = [ci, i64, i64, i64]
            L.qmm_mx_linear.argtypes = [ci, ci, vp, i64, i64, vp, i64, i64, vp, vp, vp, i64, vp, sz, vp]
            L.qmm_expert_sort_workspace_bytes.argtypes = [i32, i32, i32]
            L.qmm_expert_sort.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, vp, sz, vp]
            L.qmm_expert_gather.argtypes = [ci, vp, i64, i32, i32, i64, vp, vp, vp, vp, i64, vp]
            L.qmm_expert_combine.argtypes = [ci, vp, i64, i32, i32, i64, vp, vp, vp, i64, vp]
            L.qmm_expert_combine_grad.argtypes = [ci, vp, i64, vp, i64, i32, i32, i64, vp, vp, vp, vp, i64, vp, vp]
            L.qmm_mx_experts_bytes.argtypes = [ci, i32, i32, i32, i64]
            L.qmm_mx_quantize_experts.argtypes = [ci, ci, vp, i64, i32, i32, i32, i64, vp, vp, vp, vp, vp, vp, vp]
            L.qmm_mx_experts_gate_up.argtypes = [ci, vp, i32, i32, i32, vp, vp, vp, vp, i64, i64, vp, vp, vp, vp, vp, vp, vp]
            L.qmm_mx_experts_gemm.argtypes = [ci, vp, i32, i32, i32, vp, vp, vp, i64, i64, vp, vp, ci, vp, i64, vp, vp]
            L.qmm_mx_moe_workspace_bytes.argtypes = [ctypes.POINTER(MxMoeArgs)]
            L.qmm_mx_moe.argtypes = [ctypes.POINTER(MxMoeArgs), vp, sz, vp]
            L.qmm_expert_route.argtypes = [ci, vp, i64, i32, i32, i32, ci, vp, i32, i32, i32, i32, ctypes.c_float, vp, vp, vp]
            L.qmm_expert_route_grad.argtypes = [ci, vp, vp, i64, vp, i32, i32, i32, ci, i32, ctypes.c_float, vp, i64, vp]
            L.qmm_rms_norm.argtypes = [ci, vp, i64, vp, i64, vp, ctypes.c_float, i64, i64, vp, i64, vp, i64, ci, vp, i64, vp, vp]
            L.qmm_rms_norm_grad_workspace_bytes.argtypes = [i64, i64]
            L.qmm_rms_norm_grad.argtypes = [ci, vp, i64, vp, i64, vp, ctypes.c_float, i64, i64, vp, i64, vp, i64, vp, vp, sz, vp]
            L.qmm_rows_quantize.argtypes = [ci, vp, i64, i64, i64, ci, vp, i64, vp, vp]
            L.qmm_rows_dequantize.argtypes = [ci, vp, i64, vp, i64, i64, ci, vp, i64, vp]
            L.qmm_lora_workspace_bytes.argtypes = [i32, i32, i32]
            L.qmm_lora.argtypes = [ctypes.POINTER(LoraArgs), vp, sz, vp]
            L.qmm_lora_grad.argtypes = [ctypes.POINTER(LoraArgs), vp, sz, vp]
            L.qmm_packed_check.argtypes = [ci, vp, i64, i64, vp, vp]
            L.qmm_debug_config.argtypes = [ctypes.c_char_p, ctypes.c_char_p]
            L.qmm_debug_wait_give_up.argtypes = [vp, i64, vp]
            _lib = L
    return _lib


_ext = None


def _native():
    """The extension that marshals the shortest calls (0.5 us instead of 3 us of a call), built first if it is not there."""
    global _ext
    if _ext is None:
        lib()
        from . import _build
        with _lock:
            if not os.path.exists(_build.EXT):
                _build.build_extension()
        from . import _qmm_py
        _ext = _qmm_py
    return _ext


_layer_ext = None


def _layer():
    """The same for the router, the norm and the adapters."""
    global _layer_ext
    if _layer_ext is None:
        lib()
        from . import _build
        with _lock:
            if not os.path.exists(_build.LAYER_EXT):
                _build.build_extension()
        from . import _qmm_layer_py
        _layer_ext = _qmm_layer_py
    return _layer_ext


def last_error() -> str:
    return lib().qmm_last_error().decode("utf-8", "replace")


def _check(status: int):
    if status != 0:
        raise QmmError(status, last_error())


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    """Handle of the current stream of the current device (without a Stream object: 0.3 us instead of 3.3 us per call)."""
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _dp(t):
    return 0 if t is None else t.data_ptr()


def _nbytes(t) -> int:
    return 0 if t is None else t.numel() * t.element_size()


def version() -> int:
    return lib().qmm_version()


def canonical_bytes(fmt: int, N: int, K: int) -> int:
    return lib().qmm_canonical_bytes(fmt, N, K)


def packed_bytes(fmt: int, N: int, K: int) -> int:
    n = lib().qmm_packed_bytes(fmt, N, K)
    if n == 0:
        raise QmmError(5, last_error())
    return n


def pack(fmt: int, canonical: torch.Tensor, N: int, K: int, out: torch.Tensor | None = None) -> torch.Tensor:
    """canonical: uint8 CUDA tensor of canonical_bytes(fmt,N,K) bytes -> packed uint8 tensor."""
    assert canonical.is_cuda and canonical.dtype == torch.uint8 and canonical.is_contiguous()
    assert canonical.numel() == canonical_bytes(fmt, N, K)
    if out is None:
        out = torch.empty(packed_bytes(fmt, N, K), dtype=torch.uint8, device=canonical.device)
    _check(lib().qmm_pack(fmt, canonical.data_ptr(), N, K, out.data_ptr(), _stream()))
    return out


def dequant(fmt: int, packed: torch.Tensor, N: int, K: int) -> torch.Tensor:
    out = torch.empty((N, K), dtype=torch.float32, device=packed.device)
    _check(lib().qmm_dequant(fmt, packed.data_ptr(), N, K, out.data_ptr(), _stream()))
    return out


def gemv_workspace_bytes(fmt: int, N: int, K: int) -> int:
    return lib().qmm_gemv_workspace_bytes(fmt, N, K)


def gemv(fmt: int, packed: torch.Tensor, N: int, K: int, x: torch.Tensor,
         y: torch.Tensor | None = None, ws: torch.Tensor | None = None) -> torch.Tensor:
    """y = W x.  x: fp16 [K] CUDA tensor; returns fp16 [N]."""
    assert x.is_cuda and x.dtype == torch.float16 and x.numel() == K and x.is_contiguous()
    if y is None:
        y = torch.empty(N, dtype=torch.float16, device=x.device)
    if ws is None:
        need = gemv_workspace_bytes(fmt, N, K)
        ws = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
    _check(lib().qmm_gemv(fmt, packed.data_ptr(), N, K, x.data_ptr(), y.data_ptr(), _dp(ws), _nbytes(ws), _stream()))
    return y


def gemv_batch_problems(problems):
    """problems: iterable of (packed, N, K, x, y) tensors -> ctypes array for gemv_batch (keeps the tensors alive)."""
    problems = list(problems)
    arr = (GemvProblem * len(problems))()
    for i, (packed, N, K, x, y) in enumerate(problems):
        assert x.dtype == torch.float16 and x.numel() == K and y.dtype == torch.float16 and y.numel() == N
        arr[i] = GemvProblem(packed.data_ptr(), x.data_ptr(), y.data_ptr(), N, K)
    arr._keep = problems
    return arr


def gemv_batch(fmt: int, problems) -> None:
    """All products y_i = W_i x_i of the list in one launch.  `problems` is the array made by
    gemv_batch_problems (build it once and reuse it: the call only reads it)."""
    _check(lib().qmm_gemv_batch(fmt, problems, len(problems), _stream()))


def gemm_batch_problems(problems):
    """problems: iterable of (packed, N, K, X [M, K], Y [M, N]) tensors -> ctypes array for gemm_batch (keeps
    the tensors alive).  Row strides may exceed K / N; every X and Y has the same number of rows."""
    problems = list(problems)
    arr = (GemmProblem * len(problems))()
    for i, (packed, N, K, X, Y) in enumerate(problems):
        assert X.dtype == torch.float16 and X.dim() == 2 and X.shape[1] == K and X.stride(1) == 1
        assert Y.dtype == torch.float16 and Y.dim() == 2 and Y.shape == (X.shape[0], N) and Y.stride(1) == 1
        M = X.shape[0]
        arr[i] = GemmProblem(packed.data_ptr(), X.data_ptr(), Y.data_ptr(), N, K,
                             X.stride(0) if M > 1 else max(K, X.stride(0)), Y.stride(0) if M > 1 else max(N, Y.stride(0)))
    arr._keep = problems
    arr._M = problems[0][3].shape[0] if problems else 0
    return arr


def gemm_batch(fmt: int, problems) -> None:
    """All products Y_i = X_i W_i^T (M <= 8 rows each) of the list in one launch.  `problems` is the array
    made by gemm_batch_problems (build it once and reuse it: the call only reads it)."""
    _check(lib().qmm_gemm_batch(fmt, problems, len(problems), problems._M, _stream()))


GEMV_STATIC_SCRATCH_BYTES = 1 << 20


def gemv_gate_up(fmt: int, packed_gate: torch.Tensor, packed_up: torch.Tensor, N: int, K: int, x: torch.Tensor,
                 h: torch.Tensor | None = None) -> torch.Tensor:
    """h = fp16(silu(W_gate x) * (W_up x)) in one launch (both products kept in fp32 until the end)."""
    assert x.is_cuda and x.dtype == torch.float16 and x.numel() == K and x.is_contiguous()
    if h is None:
        h = torch.empty(N, dtype=torch.float16, device=x.device)
    assert h.is_cuda and h.dtype == torch.float16 and h.numel() == N and h.is_contiguous()
    _check(lib().qmm_gemv_gate_up(fmt, packed_gate.data_ptr(), packed_up.data_ptr(), N, K, x.data_ptr(), h.data_ptr(), _stream()))
    return h


def gemv_static(fmt: int, packed: torch.Tensor, N: int, K: int, x: torch.Tensor, y: torch.Tensor) -> torch.Tensor:
    """y = W x through qmm_gemv_static: no workspace argument and no allocation anywhere.

    For callers that may not allocate device memory when they need the product (memory
    budget already handed out, allocator calls forbidden after start-up, no tolerance for
    the device-wide synchronisation an allocation implies).  The split-K scratch is a fixed
    array inside the library (GEMV_STATIC_SCRATCH_BYTES per GPU); shapes that need more
    raise QmmError (QMM_ERR_WORKSPACE).  `y` must be provided by the caller.  All calls on a
    device share that scratch: keep them on one stream.  Make the first call on each device
    outside any stream capture.
    """
    assert x.is_cuda and x.dtype == torch.float16 and x.numel() == K and x.is_contiguous()
    assert y.is_cuda and y.dtype == torch.float16 and y.numel() == N and y.is_contiguous()
    _check(lib().qmm_gemv_static(fmt, packed.data_ptr(), N, K, x.data_ptr(), y.data_ptr(), _stream()))
    return y


def gemm_workspace_bytes(fmt: int, M: int, N: int, K: int) -> int:
    return lib().qmm_gemm_workspace_bytes(fmt, M, N, K)


def gemm(fmt: int, packed: torch.Tensor, N: int, K: int, X: torch.Tensor,
         Y: torch.Tensor | None = None, ws: torch.Tensor | None = None) -> torch.Tensor:
    """Y = X W^T.  X: fp16 [M,K] (row stride >= K); returns fp16 [M,N]."""
    assert X.is_cuda and X.dtype == torch.float16 and X.dim() == 2 and X.shape[1] == K and X.stride(1) == 1
    M = X.shape[0]
    if Y is None:
        Y = torch.empty((M, N), dtype=torch.float16, device=X.device)
    assert Y.stride(1) == 1
    if ws is None:
        ws = torch.zeros(max(gemm_workspace_bytes(fmt, M, N, K), 256), dtype=torch.uint8, device=X.device)
    _check(lib().qmm_gemm(fmt, packed.data_ptr(), N, K, X.data_ptr(), X.stride(0) if M > 1 else max(K, X.stride(0)),
                          Y.data_ptr(), Y.stride(0) if M > 1 else max(N, Y.stride(0)), M,
                          ws.data_ptr(), _nbytes(ws), _stream()))
    return Y


def moe_args(fmt, T, H, I, E, topk, logits, X, w_gate, w_up, w_down, out,
             topk_idx=None, topk_w=None, perm=None, expert_offsets=None, dbg_H=None, dbg_D=None,
             w_router=None, router_logits=None) -> MoeArgs:
    a = MoeArgs(T, H, I, E, topk, fmt, _dp(logits), _dp(X), _dp(w_gate), _dp(w_up), _dp(w_down), _dp(out),
                _dp(topk_idx), _dp(topk_w), _dp(perm), _dp(expert_offsets), _dp(dbg_H), _dp(dbg_D),
                _dp(w_router), _dp(router_logits))
    # the struct holds raw device pointers only: keep the tensors alive as long as the struct
    a._keep = (logits, X, w_gate, w_up, w_down, out, topk_idx, topk_w, perm, expert_offsets, dbg_H, dbg_D, w_router, router_logits)
    return a


def moe_workspace_bytes(args: MoeArgs) -> int:
    n = lib().qmm_moe_workspace_bytes(ctypes.byref(args))
    if n == 0:
        raise QmmError(5, last_error())
    return n


def moe(args: MoeArgs, ws: torch.Tensor) -> None:
    _check(lib().qmm_moe(ctypes.byref(args), ws.data_ptr(), _nbytes(ws), _stream()))


def moe_route(args: MoeArgs, ws: torch.Tensor) -> None:
    _check(lib().qmm_moe_route(ctypes.byref(args), ws.data_ptr(), _nbytes(ws), _stream()))


def status_check(ws: torch.Tensor) -> None:
    _check(lib().qmm_status_check(ws.data_ptr(), _stream()))


class Chain:
    """A planned list of decode products (qmm_chain_build); run() is the one-launch hot-path call.

    stages: list of dicts with keys op, packed, N, K and either x (fp16 CUDA tensor) or x_stage (+ x_offset);
    optional packed_up (gate/up stages) and y (fp16 CUDA tensor receiving a plain copy of the output).
    The object keeps every tensor it refers to alive; the plan and workspace tensors are attributes."""

    def __init__(self, fmt: int, stages):
        self.fmt = fmt
        self._keep = []
        arr = (ChainStage * len(stages))()
        for i, s in enumerate(stages):
            x, y, up = s.get("x"), s.get("y"), s.get("packed_up")
            if x is not None:
                assert x.is_cuda and x.dtype == torch.float16 and x.is_contiguous() and x.numel() == s["K"]
            if y is not None:
                assert y.is_cuda and y.dtype == torch.float16 and y.is_contiguous() and y.numel() == s["N"]
            arr[i] = ChainStage(s.get("op", CHAIN_LINEAR), -1 if x is not None else s["x_stage"], s.get("x_offset", 0),
                                _dp(x), s["packed"].data_ptr(), _dp(up), s["N"], s["K"], _dp(y))
            self._keep.append((x, y, up, s["packed"]))
        self.stages = arr
        L = lib()
        plan_bytes = L.qmm_chain_plan_bytes(fmt, arr, len(arr))
        ws_bytes = L.qmm_chain_workspace_bytes(fmt, arr, len(arr))
        if plan_bytes == 0 or ws_bytes == 0:
            raise QmmError(1, last_error())
        self.plan = torch.empty(plan_bytes, dtype=torch.uint8, device="cuda")
        self.ws = torch.empty(ws_bytes, dtype=torch.uint8, device="cuda")
        self.info = ChainInfo()
        _check(L.qmm_chain_build(fmt, arr, len(arr), self.plan.data_ptr(), plan_bytes, self.ws.data_ptr(), ws_bytes,
                                 ctypes.byref(self.info), _stream()))

    def run(self) -> None:
        _check(lib().qmm_chain_run(ctypes.byref(self.info), _stream()))


# ---- microscaled 4-bit floating point

def _rows2d(t: torch.Tensor, what: str):
    """(pointer, row pitch, rows, columns) of a 2-D CUDA tensor whose rows are contiguous."""
    assert t.is_cuda and t.dim() == 2, "%s: 2-D CUDA tensor" % what
    rows, cols = t.shape
    ld, inner = t.stride()
    assert inner == 1 or cols <= 1, "%s: rows must be contiguous" % what
    return t.data_ptr(), ld if rows > 1 or ld > cols else cols, rows, cols


def _counts(*n) -> None:
    """Counts are 32-bit in the library (ctypes would cut larger ones)."""
    assert max(n) < 1 << 31 and min(n) >= -(1 << 31), "a count past 32 bits: %s" % (n,)


_one_gpu = None


def _on_device(now, *tensors) -> None:
    """CUDA tensors of another device than `now` (None: the current one, where a kernel runs) are refused.  A tensor may be None; with one GPU there is no other."""
    global _one_gpu
    if _one_gpu is None:
        _one_gpu = torch.cuda.device_count() == 1
    if _one_gpu:
        return
    if now is None:
        now = torch.cuda.current_device()
    for t in tensors:
        assert t is None or t.get_device() == now, "tensor on device %d, device %d is wanted" % (t.get_device(), now)


def _mx_need(fmt: int, rows: int, K: int) -> int:
    """mx_bytes, for the two formats without a call into the library: the size that a packed argument has to have."""
    if fmt != MXFP4 and fmt != NVFP4:
        return lib().qmm_mx_bytes(fmt, rows, K)
    return ((rows + 127) >> 7) * ((K + 255) >> 8) * (16384 + 32768 // fmt)


def _scalar(t, n: int = 1) -> int:
    """Pointer of n fp32 tensor scales (None: 0)."""
    if t is None:
        return 0
    assert t.is_cuda and t.dtype == torch.float32 and t.numel() == n and t.is_contiguous()
    return t.data_ptr()


def _operand(t: torch.Tensor, need: int, what: str, rows: int = 1) -> int:
    """Pointer of a packed operand of at least `need` bytes (without rows nothing is touched)."""
    if rows == 0:
        return 0
    assert t.is_cuda and t.dtype == torch.uint8 and t.is_contiguous()
    if need == 0:
        raise QmmError(1, last_error())
    assert t.numel() >= need, "%s: %d bytes, %d needed" % (what, t.numel(), need)
    return t.data_ptr()


def _workspace(need: int, device, ws: torch.Tensor | None) -> torch.Tensor:
    """ws, or a new workspace with its header zeroed (callers on a hot path keep one)."""
    if need == 0:
        raise QmmError(1, last_error())
    if ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device=device)
        ws[:1024].zero_()
    assert ws.is_cuda and ws.is_contiguous(), "workspace: a contiguous CUDA tensor is wanted"
    return ws


def _status(t) -> int:
    """Pointer of a status word in device memory (None: 0)."""
    if t is None:
        return 0
    assert t.is_cuda and t.is_contiguous() and _nbytes(t) >= 4, "status: a word in CUDA memory is wanted"
    return t.data_ptr()


def mx_bytes(fmt: int, rows: int, K: int) -> int:
    return lib().qmm_mx_bytes(fmt, rows, K)


def mx_pack(fmt: int, codes: torch.Tensor, scales: torch.Tensor, K: int, out: torch.Tensor | None = None) -> torch.Tensor:
    """Canonical codes uint8 [rows, ceil(K/B) B/2] and scales uint8 [rows, ceil(K/B)] (B = fmt, the block length) -> packed operand."""
    rows, blocks = codes.shape[0], -(-K // fmt)
    assert codes.is_cuda and codes.dtype == torch.uint8 and codes.is_contiguous() and codes.shape == (rows, blocks * fmt // 2)
    assert scales.is_cuda and scales.dtype == torch.uint8 and scales.is_contiguous() and scales.shape == (rows, blocks)
    need = mx_bytes(fmt, rows, K)
    if out is None:
        out = torch.empty(need, dtype=torch.uint8, device=codes.device)
    _on_device(None, codes, scales, out)
    _check(lib().qmm_mx_pack(fmt, codes.data_ptr(), scales.data_ptr(), rows, K, _operand(out, need, "out", rows), _stream()))
    return out


def mx_quantize(fmt: int, x: torch.Tensor, out: torch.Tensor | None = None, tensor_scale: torch.Tensor | None = None) -> torch.Tensor:
    """x [rows, K] (fp16, bf16 or fp32; any row stride) -> packed operand, uint8."""
    if out is None:
        out = torch.empty(lib().qmm_mx_bytes(fmt, x.shape[0], x.shape[1]), dtype=torch.uint8, device=x.device)
    _check((_ext or _native()).mx_quantize(fmt, x, out, tensor_scale))
    return out


def mx_dequantize(fmt: int, packed: torch.Tensor, rows: int, K: int, out: torch.Tensor | None = None,
                  tensor_scale: torch.Tensor | None = None, dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """Packed operand -> the values it stands for, [rows, K] of out's type (or `dtype`)."""
    if out is None:
        out = torch.empty((rows, K), dtype=dtype, device=packed.device)
    assert out.shape == (rows, K)
    _check((_ext or _native()).mx_dequantize(fmt, packed, out, tensor_scale))
    return out


def mx_gemm_workspace_bytes(fmt: int, M: int, N: int, K: int) -> int:
    return lib().qmm_mx_gemm_workspace_bytes(fmt, M, N, K)


def mx_gemm(fmt: int, a: torch.Tensor, M: int, w: torch.Tensor, N: int, K: int, Y: torch.Tensor | None = None,
            a_scale: torch.Tensor | None = None, w_scale: torch.Tensor | None = None, ws: torch.Tensor | None = None,
            dtype: torch.dtype = torch.float16) -> torch.Tensor:
    """Y [M, N] = a w^T with both operands packed; Y's type, or `dtype` where Y is None."""
    L = lib()
    if Y is None:
        Y = torch.empty((M, N), dtype=dtype, device=a.device)
    ptr, ld, r, c = _rows2d(Y, "Y")
    assert (r, c) == (M, N)
    ws = _workspace(L.qmm_mx_gemm_workspace_bytes(fmt, M, N, K), a.device, ws)
    _on_device(None, a, w, Y, a_scale, w_scale, ws)
    _check(L.qmm_mx_gemm(fmt, _operand(a, _mx_need(fmt, M, K), "a", M), M, _operand(w, _mx_need(fmt, N, K), "w"), N, K,
                         _scalar(a_scale), _scalar(w_scale), DTYPES[Y.dtype], ptr, ld, ws.data_ptr(), _nbytes(ws), _stream()))
    return Y


def mx_linear_workspace_bytes(fmt: int, M: int, N: int, K: int) -> int:
    return lib().qmm_mx_linear_workspace_bytes(fmt, M, N, K)


def mx_linear(fmt: int, X: torch.Tensor, w: torch.Tensor, N: int, Y: torch.Tensor | None = None, x_scale: torch.Tensor | None = None,
              w_scale: torch.Tensor | None = None, ws: torch.Tensor | None = None) -> torch.Tensor:
    """Y [M, N] = quantised(X) w^T: X [M, K] as it comes (fp16, bf16 or fp32), w packed [N, K]; Y has X's type."""
    if Y is None:
        Y = torch.empty((X.shape[0], N), dtype=X.dtype, device=X.device)
    if ws is None:
        ws = _workspace(lib().qmm_mx_linear_workspace_bytes(fmt, X.shape[0], N, X.shape[1]), X.device, ws)
    _check((_ext or _native()).mx_linear(fmt, X, w, N, Y, x_scale, w_scale, ws))
    return Y


# ---- tokens sorted by expert and back

class ExpertPlan:
    """Where each (token, slot) pair of a router's choice goes in expert order (qmm_expert_sort fills it; buffers are kept
    and may be refilled; before the first sort every pair counts as dropped).  order, place [T * topk], offsets, units [E + 1]:
    int32 views of one buffer."""

    def __init__(self, T: int, topk: int, E: int, device="cuda", fill: bool = True):
        _counts(T, topk, E, T * topk)
        P = T * topk
        self.T, self.topk, self.E = T, topk, E
        self.buf = torch.empty(2 * P + 2 * (E + 1), dtype=torch.int32, device=device)
        self.device = self.buf.get_device()
        self.order, self.place, self.offsets, self.units = self.buf.split([P, P, E + 1, E + 1])
        if fill:                                           # (a sort follows at once otherwise)
            self.buf[: 2 * P].fill_(-1)
            self.buf[2 * P:].zero_()
        base = self.buf.data_ptr()
        self.ptrs = (base, base + 4 * P, base + 8 * P, base + 8 * P + 4 * (E + 1))         # order, place, offsets, units
        self.ws_bytes = lib().qmm_expert_sort_workspace_bytes(T, topk, E)
        self.ws = torch.empty(self.ws_bytes, dtype=torch.uint8, device=device) if self.ws_bytes else None
        self.ws_ptr = _dp(self.ws)


def expert_sort(idx: torch.Tensor, E: int, out: ExpertPlan | None = None) -> ExpertPlan:
    """idx [T, topk] int32: experts of each token, values outside [0, E) dropped -> ExpertPlan."""
    T, topk = idx.shape
    if out is None:
        out = ExpertPlan(T, topk, E, idx.device, fill=False)
    assert out.T == T and out.topk == topk and out.E == E
    order, place, offsets, units = out.ptrs
    _check((_ext or _native()).expert_sort(idx, E, order, place, offsets, units, out.ws_ptr, out.ws_bytes, out.device))
    return out


def expert_gather(x: torch.Tensor, plan: ExpertPlan, weights: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """xs [T * topk, H]: row place[p] = (weights[p] *) x[p // topk]; rows past the last pair are zero."""
    if out is None:
        out = torch.empty((plan.T * plan.topk, x.shape[1]), dtype=x.dtype, device=x.device)
    _check((_ext or _native()).expert_gather(x, plan.T, plan.topk, plan.ptrs[0], plan.ptrs[1], plan.device, weights, out))
    return out


def expert_combine(ys: torch.Tensor, plan: ExpertPlan, weights: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """y [T, H] = sum over a token's pairs of (weights[p] *) ys[place[p]]."""
    if out is None:
        out = torch.empty((plan.T, ys.shape[1]), dtype=ys.dtype, device=ys.device)
    _check((_ext or _native()).expert_combine(ys, plan.T, plan.topk, plan.ptrs[1], plan.device, weights, out))
    return out


def expert_combine_grad(dy: torch.Tensor, ys: torch.Tensor, plan: ExpertPlan, weights: torch.Tensor, dys: torch.Tensor | None = None,
                        dw: torch.Tensor | None = None):
    """Gradients of expert_combine: (dys [T * topk, H], dw [T, topk] fp32)."""
    if dys is None:
        dys = torch.empty((plan.T * plan.topk, dy.shape[1]), dtype=dy.dtype, device=dy.device)
    if dw is None:
        dw = torch.empty((plan.T, plan.topk), dtype=torch.float32, device=dy.device)
    _check((_ext or _native()).expert_combine_grad(dy, ys, plan.T, plan.topk, plan.ptrs[0], plan.ptrs[1], plan.device, weights, dys, dw))
    return dys, dw


def expert_gather_grad(dxs: torch.Tensor, plan: ExpertPlan, weights: torch.Tensor | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """Gradient of expert_gather with respect to x: the sum over a token's pairs of (weights[p] *) dxs[place[p]]."""
    return expert_combine(dxs, plan, weights, out)


# ---- experts' products on microscaled operands

def mx_experts_bytes(fmt: int, T: int, topk: int, E: int, K: int) -> int:
    _counts(fmt, T, topk, E)
    return lib().qmm_mx_experts_bytes(fmt, T, topk, E, K)


def mx_quantize_experts(fmt: int, x: torch.Tensor, idx: torch.Tensor, plan: ExpertPlan, out: torch.Tensor | None = None,
                        tensor_scale: torch.Tensor | None = None) -> torch.Tensor:
    """x [T, K] quantised once per token and stored at the row of each of its pairs (rows grouped by expert)."""
    xp, ldx, T, K = _rows2d(x, "x")
    assert T == plan.T and idx.is_cuda and idx.dtype == torch.int32 and idx.is_contiguous() and idx.shape == (T, plan.topk)
    need = mx_experts_bytes(fmt, T, plan.topk, plan.E, K)
    if out is None:
        out = torch.empty(need, dtype=torch.uint8, device=x.device)
    _on_device(None, x, idx, plan.buf, out, tensor_scale)
    _check(lib().qmm_mx_quantize_experts(fmt, DTYPES[x.dtype], xp, ldx, T, plan.topk, plan.E, K, idx.data_ptr(), plan.ptrs[1], plan.ptrs[2],
                                         plan.ptrs[3], _scalar(tensor_scale), _operand(out, need, "out", T), _stream()))
    return out


def mx_experts_gate_up(fmt: int, a: torch.Tensor, plan: ExpertPlan, w_gate: torch.Tensor, w_up: torch.Tensor, N: int, K: int,
                       h: torch.Tensor | None = None, a_scale=None, gate_scale=None, up_scale=None, h_scale=None, status=None) -> torch.Tensor:
    """Packed rows [., K] -> packed rows [., N]: silu(W_gate[e] a) * (W_up[e] a), quantised from fp32."""
    T, topk, E = plan.T, plan.topk, plan.E
    each, need = E * mx_bytes(fmt, N, K), mx_experts_bytes(fmt, T, topk, E, N)
    if h is None:
        h = torch.empty(need, dtype=torch.uint8, device=a.device)
    _on_device(None, a, plan.buf, w_gate, w_up, h, a_scale, gate_scale, up_scale, h_scale, status)
    _check(lib().qmm_mx_experts_gate_up(fmt, _operand(a, mx_experts_bytes(fmt, T, topk, E, K), "a", T), T, topk, E, plan.ptrs[2], plan.ptrs[3],
                                        _operand(w_gate, each, "w_gate"), _operand(w_up, each, "w_up"), N, K, _scalar(a_scale),
                                        _scalar(gate_scale, E), _scalar(up_scale, E), _scalar(h_scale), _operand(h, need, "h", T), _status(status), _stream()))
    return h


def mx_experts_gemm(fmt: int, a: torch.Tensor, plan: ExpertPlan, w: torch.Tensor, N: int, K: int, Y: torch.Tensor | None = None,
                    a_scale=None, w_scale=None, status=None, dtype: torch.dtype = torch.float16) -> torch.Tensor:
    """Packed rows [., K] -> Y [T * topk, N] in sorted order: row r of expert e = W[e] a[r]."""
    T, topk, E = plan.T, plan.topk, plan.E
    if Y is None:
        Y = torch.empty((T * topk, N), dtype=dtype, device=a.device)
    yp, ldy, r, c = _rows2d(Y, "Y")
    assert (r, c) == (T * topk, N)
    _on_device(None, a, plan.buf, w, Y, a_scale, w_scale, status)
    _check(lib().qmm_mx_experts_gemm(fmt, _operand(a, mx_experts_bytes(fmt, T, topk, E, K), "a", T), T, topk, E, plan.ptrs[2], plan.ptrs[3],
                                     _operand(w, E * mx_bytes(fmt, N, K), "w"), N, K, _scalar(a_scale), _scalar(w_scale, E), DTYPES[Y.dtype],
                                     yp, ldy, _status(status), _stream()))
    return Y


def mx_moe_args(fmt: int, X, idx, weights, w_gate, w_up, w_down, I: int, E: int, out, x_scale=None, gate_scale=None, up_scale=None,
                down_scale=None, h_scale=None, rows_dtype: torch.dtype | None = None) -> MxMoeArgs:
    """Arguments of mx_moe_run: build once and reuse while the tensors stay where they are (the struct keeps them alive).
    rows_dtype: type of the experts' rows on their way to the weighted sum, X's (default) or torch.float32."""
    xp, ldx, T, H = _rows2d(X, "X")
    op, ldo, r, c = _rows2d(out, "out")
    topk = idx.shape[1]
    _counts(T, H, I, E, topk)
    assert idx.is_cuda and idx.dtype == torch.int32 and idx.is_contiguous() and idx.shape[0] == T
    assert weights.is_cuda and weights.dtype == torch.float32 and weights.is_contiguous() and weights.shape == idx.shape
    assert (r, c) == (T, H) and out.dtype == X.dtype
    assert rows_dtype in (None, X.dtype, torch.float32), "rows_dtype: X's type or torch.float32"
    gu, dn = E * _mx_need(fmt, I, H), E * _mx_need(fmt, H, I)
    a = MxMoeArgs(T, H, I, E, topk, fmt, DTYPES[X.dtype], xp, ldx, idx.data_ptr(), weights.data_ptr(), _operand(w_gate, gu, "w_gate"),
                  _operand(w_up, gu, "w_up"), _operand(w_down, dn, "w_down"), _scalar(x_scale), _scalar(h_scale), _scalar(gate_scale, E),
                  _scalar(up_scale, E), _scalar(down_scale, E), op, ldo, int(rows_dtype is torch.float32))
    a._keep = (X, idx, weights, w_gate, w_up, w_down, out, x_scale, gate_scale, up_scale, down_scale, h_scale)
    _on_device(X.get_device(), *a._keep)
    return a


def mx_moe_workspace_bytes(args: MxMoeArgs) -> int:
    return lib().qmm_mx_moe_workspace_bytes(ctypes.byref(args))


def mx_moe_run(args: MxMoeArgs, ws: torch.Tensor) -> None:
    assert ws.is_cuda and ws.is_contiguous(), "workspace: a contiguous CUDA tensor is wanted"
    _on_device(None, ws, *getattr(args, "_keep", ())[:1])
    _check(lib().qmm_mx_moe(ctypes.byref(args), ws.data_ptr(), _nbytes(ws), _stream()))


def mx_moe(fmt: int, X, idx, weights, w_gate, w_up, w_down, I: int, E: int, out=None, ws=None, **scales) -> torch.Tensor:
    """A routed feed-forward layer in 4 bits: out [T, H] from X [T, H], idx / weights [T, topk] and E packed matrices of each kind
    (scales: x_scale, h_scale, and [E] gate_scale, up_scale, down_scale for NVFP4; rows_dtype as in mx_moe_args)."""
    if out is None:
        out = torch.empty_like(X, memory_format=torch.contiguous_format)
    args = mx_moe_args(fmt, X, idx, weights, w_gate, w_up, w_down, I, E, out, **scales)
    if ws is None:
        ws = _workspace(mx_moe_workspace_bytes(args), X.device, None)
    mx_moe_run(args, ws)
    return out


# ---- a router's choice

def expert_route(logits: torch.Tensor, topk: int, scores: int = SOFTMAX, bias: torch.Tensor | None = None, groups: int = 1, top_groups: int | None = None,
                 group_top: int = 1, renormalize: bool = True, scale: float = 1.0, idx: torch.Tensor | None = None, weights: torch.Tensor | None = None):
    """logits [T, E] (fp16, bf16 or fp32) -> (idx [T, topk] int32, weights [T, topk] fp32): what expert_sort, expert_combine and mx_moe take.
    scores SOFTMAX or SIGMOID; bias [E] fp32 counts for the choice alone; of `groups` groups of experts, valued by their group_top (1 or 2) best, top_groups
    (default: all) are open.  Experts whose logit is -inf are not chosen: slots left over have idx -1 and weight 0."""
    T, E = logits.shape
    if idx is None:
        idx = torch.empty((T, topk), dtype=torch.int32, device=logits.device)
    if weights is None:
        weights = torch.empty((T, topk), dtype=torch.float32, device=logits.device)
    assert idx.shape == (T, topk) and weights.shape == (T, topk), "idx and weights: [T, topk]"
    _check((_layer_ext or _layer()).expert_route(logits, topk, scores, bias, groups, groups if top_groups is None else top_groups, group_top, 1 if renormalize else 0, scale,
                                                 idx, weights))
    return idx, weights


def expert_route_grad(dweights: torch.Tensor, logits: torch.Tensor, idx: torch.Tensor, scores: int = SOFTMAX, renormalize: bool = True, scale: float = 1.0,
                      out: torch.Tensor | None = None) -> torch.Tensor:
    """Gradient of expert_route's weights with respect to the logits: dweights [T, topk] (as expert_combine_grad gives it) -> [T, E] of the logits' type."""
    if out is None:
        out = torch.empty_like(logits, memory_format=torch.contiguous_format)
    T, topk = idx.shape
    assert logits.shape[0] == T and dweights.shape == (T, topk), "dweights and idx [T, topk], logits [T, E]"
    _check((_layer_ext or _layer()).expert_route_grad(dweights, logits, idx, topk, scores, 1 if renormalize else 0, scale, out))
    return out


# ---- root-mean-square norm, rows of 8 bits

def rms_norm(x: torch.Tensor, weight: torch.Tensor | None = None, eps: float = 1e-6, residual: torch.Tensor | None = None, h: torch.Tensor | None = None,
             y: torch.Tensor | None = None):
    """(y, h): h = x + residual (x itself without one), y = h / sqrt(mean(h^2) + eps) * weight, all [rows, K] of one type; any row strides.  h may be x or residual."""
    if y is None:
        y = torch.empty_like(x, memory_format=torch.contiguous_format)
    if h is None and residual is not None:
        h = torch.empty_like(x, memory_format=torch.contiguous_format)
    _check((_layer_ext or _layer()).rms_norm(x, weight, eps, residual, h, y, None, None))
    return y, x if h is None else h


def rms_norm_rows(x: torch.Tensor, weight: torch.Tensor | None = None, eps: float = 1e-6, residual: torch.Tensor | None = None, h: torch.Tensor | None = None,
                  codes: torch.Tensor | None = None, scales: torch.Tensor | None = None, y: torch.Tensor | None = None, dtype: torch.dtype = torch.float8_e4m3fn):
    """(codes, scales, h): the same norm into rows of 8 bits (torch.float8_e4m3fn or torch.int8) with one fp32 scale per row; also into y where it is given."""
    if codes is None:
        codes = torch.empty(x.shape, dtype=dtype, device=x.device)
    if scales is None:
        scales = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
    if h is None and residual is not None:
        h = torch.empty_like(x, memory_format=torch.contiguous_format)
    _check((_layer_ext or _layer()).rms_norm(x, weight, eps, residual, h, y, codes, scales))
    return codes, scales, x if h is None else h


def rms_norm_grad_workspace_bytes(rows: int, K: int) -> int:
    return lib().qmm_rms_norm_grad_workspace_bytes(rows, K)


def rms_norm_grad(dy: torch.Tensor, h: torch.Tensor, weight: torch.Tensor | None = None, eps: float = 1e-6, dh: torch.Tensor | None = None, dx: torch.Tensor | None = None,
                  dweight: torch.Tensor | None = None, ws: torch.Tensor | None = None, want_dweight: bool = True):
    """(dx, dweight fp32 [K]): gradients of rms_norm for dy at y and dh (optional) at h; dx is that of x and of the residual."""
    if dx is None:
        dx = torch.empty_like(h, memory_format=torch.contiguous_format)
    if dweight is None and want_dweight:
        dweight = torch.empty(h.shape[1], dtype=torch.float32, device=h.device)
    if ws is None and dweight is not None:
        ws = torch.empty(rms_norm_grad_workspace_bytes(*h.shape), dtype=torch.uint8, device=h.device)
    _check((_layer_ext or _layer()).rms_norm_grad(dy, h, weight, eps, dh, dx, dweight, ws))
    return dx, dweight


def rows_quantize(x: torch.Tensor, codes: torch.Tensor | None = None, scales: torch.Tensor | None = None, dtype: torch.dtype = torch.float8_e4m3fn):
    """x [rows, K] -> (codes of 8 bits [rows, K], scales fp32 [rows]): what lora takes as x, and what a training program keeps of x for lora_grad."""
    if codes is None:
        codes = torch.empty(x.shape, dtype=dtype, device=x.device)
    if scales is None:
        scales = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
    _check((_layer_ext or _layer()).rows_quantize(x, codes, scales))
    return codes, scales


def rows_dequantize(codes: torch.Tensor, scales: torch.Tensor, out: torch.Tensor | None = None, dtype: torch.dtype = torch.float32) -> torch.Tensor:
    """Rows of 8 bits -> the values that they stand for, of out's type (or `dtype`)."""
    if out is None:
        out = torch.empty(codes.shape, dtype=dtype, device=codes.device)
    _check((_layer_ext or _layer()).rows_dequantize(codes, scales, out))
    return out


# ---- low-rank adapters beside a shared projection

LORA_ROWS_WITHOUT_WORKSPACE = 512                          # the library's bound: a forward pass of up to so many rows sorts nothing


def lora_workspace_bytes(T: int, n: int, r: int) -> int:
    _counts(T, n, r)
    need = lib().qmm_lora_workspace_bytes(T, n, r)
    if need == 0:
        raise QmmError(1, last_error())
    return need


def _lora_plan(plan: ExpertPlan | None, T: int, n: int):
    """Addresses of a plan's order, offsets and units, and its device; zeros without one."""
    if plan is None:
        return 0, 0, 0, 0
    assert plan.T == T and plan.topk == 1 and plan.E == n, "plan: of idx [T, 1] and n adapters"
    return plan.ptrs[0], plan.ptrs[2], plan.ptrs[3], plan.device


def lora(x: torch.Tensor, idx: torch.Tensor, a: torch.Tensor, b: torch.Tensor, y0: torch.Tensor | None, scale: torch.Tensor | None = None,
         x_scale: torch.Tensor | None = None, s: torch.Tensor | None = None, plan: ExpertPlan | None = None, ws: torch.Tensor | None = None,
         out: torch.Tensor | None = None) -> torch.Tensor:
    """out [T, N] = y0 + scale[idx] * b[idx] (a[idx] x): adapters a [n, r, K], b [n, N, r] beside a projection's output y0 (None: zeros; out may be y0).
    x [T, K] of the adapters' type, or rows of 8 bits with x_scale.  idx [T] int32, outside [0, n): no adapter.  s [T, r] fp32 receives a[idx] x, which lora_grad takes.
    plan: expert_sort(idx.view(-1, 1), n), for programs that use one for many projections."""
    T = x.shape[0]
    if out is None:
        out = torch.empty((T, b.shape[1]), dtype=b.dtype, device=x.device)
    if ws is None and T > LORA_ROWS_WITHOUT_WORKSPACE:
        ws = torch.empty(lora_workspace_bytes(T, a.shape[0], a.shape[1]), dtype=torch.uint8, device=x.device)
    _check((_layer_ext or _layer()).lora(x, x_scale, idx, a, b, scale, *_lora_plan(plan, T, a.shape[0]), s, y0, out, ws))
    return out


def lora_grad(dy: torch.Tensor, x: torch.Tensor | None, s: torch.Tensor | None, idx: torch.Tensor, a: torch.Tensor, b: torch.Tensor, dx0: torch.Tensor | None = None,
              scale: torch.Tensor | None = None, x_scale: torch.Tensor | None = None, plan: ExpertPlan | None = None, ws: torch.Tensor | None = None,
              dx: torch.Tensor | None | bool = None, da: torch.Tensor | None | bool = None, db: torch.Tensor | None | bool = None):
    """(dx, da, db): dx [T, K] = dx0 (None: zeros) + the adapters' part, of dy's type; da, db fp32 in a's and b's shapes.  x: as in lora, 16-bit or 8-bit rows.
    dx, da or db False: not wanted (da needs x, db needs s)."""
    T, n, r = dy.shape[0], a.shape[0], a.shape[1]

    def out(t, shape, dtype):
        return None if t is False else torch.empty(shape, dtype=dtype, device=dy.device) if t is None else t
    dx, da, db = out(dx, (T, a.shape[2]), dy.dtype), out(da, a.shape, torch.float32), out(db, b.shape, torch.float32)
    if ws is None:
        ws = torch.empty(lora_workspace_bytes(T, n, r), dtype=torch.uint8, device=dy.device)
    _check((_layer_ext or _layer()).lora_grad(x, x_scale, idx, a, b, scale, *_lora_plan(plan, T, n), s, dy, dx0, dx, da, db, ws))
    return dx, da, db


def packed_check(fmt: int, packed: torch.Tensor, N: int, K: int, ws: torch.Tensor) -> None:
    """Enqueue the plausibility check of a packed buffer; status_check(ws) reports the outcome."""
    _check(lib().qmm_packed_check(fmt, packed.data_ptr(), N, K, ws.data_ptr(), _stream()))


def debug_config(name: str | None, value: str | None = None) -> None:
    """Set (or with value None clear) a debug knob; name None resets all of them."""
    enc = lambda v: None if v is None else str(v).encode()
    _check(lib().qmm_debug_config(enc(name), enc(value)))


def debug_wait_give_up(ws: torch.Tensor, limit_cycles: int) -> None:
    _check(lib().qmm_debug_wait_give_up(ws.data_ptr(), int(limit_cycles), _stream()))
