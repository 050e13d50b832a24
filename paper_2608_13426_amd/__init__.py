"""Python binding of librmm (Reduced Matrix Multiplication on MI355X).

Thin ctypes layer over the C-ABI declared in ``include/rmm.h``: it reads
sizes and strides off torch tensors, passes raw device pointers and the
current HIP stream, and raises ``RmmError`` on a non-zero status.  Every
step of the computation runs in librmm's gfx950 kernels; torch only owns the
device memory and the stream.  Importing this package fails loudly when
``librmm.so`` has not been built (``python paper_2608_13426_amd/build.py``).
"""
from __future__ import annotations

import ctypes
import os
import struct

import torch

__all__ = [
    "RmmError", "LIB_PATH", "lib", "RMM_F32", "RMM_BF16", "RMM_OP_SCORE",
    "RMM_OP_SELECT", "RMM_OP_LINEAR", "RMM_OP_ATTENTION", "RMM_OP_PV", "rmm_retained_count",
    "rmm_workspace_size", "rmm_reduced_pv",
    "rmm_status_string", "rmm_score", "rmm_select", "rmm_reduced_gemm",
    "rmm_reduced_qk", "rmm_linear", "rmm_score_kmajor", "rmm_reduced_gemm_kmajor",
    "rmm_reduced_attention", "rmm_reduced_gemv", "rmm_gemv_workspace_size", "rmm_select_tokens",
    "rmm_linear_noalloc", "rmm_noalloc_scratch_bytes", "rmm_rmsnorm_kmajor",
    "rmm_rmsnorm_kmajor_workspace_size", "rmm_attention_weights_kmajor",
    "rmm_attention_weights_kmajor_workspace_size", "rmm_reduced_pv_kmajor", "rmm_decode_step",
    "rmm_decode_step_workspace_size", "rmm_decode_products", "rmm_decode_products_shared",
    "rmm_decode_products_shared_workspace_size", "rmm_decode_step_shared", "DecodeGroup",
    "rmm_reduced_qk_rowstats",
    "rmm_attention_weights_kmajor_rowstats", "RMM_CACHE_BF", "RMM_CACHE_MX", "Rope", "rope_tables", "KvCache",
    "kv_cache", "rmm_qk_norm_rope", "rmm_qk_norm_rope_workspace_size", "rmm_kv_append", "rmm_kv_gather",
    "rmm_paged_attention", "rmm_paged_attention_workspace_size", "EXPORTED_SYMBOLS",
]

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "librmm.so")

RMM_F32, RMM_BF16 = 0, 1
RMM_OP_SCORE, RMM_OP_SELECT, RMM_OP_LINEAR, RMM_OP_ATTENTION, RMM_OP_PV = 0, 1, 2, 3, 4
RMM_CACHE_BF, RMM_CACHE_MX = 0, 1

_p = ctypes.c_void_p
_i64 = ctypes.c_int64


class DecodeGroup(ctypes.Structure):
    """rmm_decode_group_t: one projection group of a decode step."""
    _fields_ = [("X", _p), ("W", _p), ("idx", _p), ("Y", _p), ("K", _i64), ("N", _i64),
                ("k", _i64), ("ldx", _i64), ("ldw", _i64), ("ldy", _i64)]


class _Heads(ctypes.Structure):
    """rmm_heads_t"""
    _fields_ = [("data", _p), ("n", _i64), ("batch_stride", _i64), ("token_stride", _i64),
                ("head_stride", _i64)]


class _RopeTables(ctypes.Structure):
    """rmm_rope_t"""
    _fields_ = [("cos", _p), ("sin", _p), ("n_pos", _i64), ("rot", _i64), ("interleaved", ctypes.c_int)]


class _KvCacheC(ctypes.Structure):
    """rmm_kv_cache_t"""
    _fields_ = [("type", ctypes.c_int), ("k", _p), ("v", _p), ("k_scale", _p), ("v_scale", _p),
                ("n_pages", _i64), ("page_size", _i64), ("Hkv", _i64), ("D", _i64), ("k_stride", _i64),
                ("v_stride", _i64), ("k_scale_stride", _i64), ("v_scale_stride", _i64)]


# these structs are only read by the library: the binding passes each packed into bytes
_HEADS_BYTES, _ROPE_BYTES = struct.Struct("@Pqqqq"), struct.Struct("@PPqqi4x")
assert _HEADS_BYTES.size == ctypes.sizeof(_Heads) and _ROPE_BYTES.size == ctypes.sizeof(_RopeTables)

_SIGS = {
    "rmm_retained_count": (_i64, [ctypes.c_double, _i64]),
    "rmm_workspace_size": (ctypes.c_size_t, [ctypes.c_int, _i64, _i64, _i64, _i64]),
    "rmm_score": (ctypes.c_int, [_p, ctypes.c_int, _i64, _i64, _i64, _i64, _p, _p,
                                 ctypes.c_size_t, _p]),
    "rmm_select": (ctypes.c_int, [_p, _i64, _i64, _i64, _p, _p]),
    "rmm_reduced_gemm": (ctypes.c_int, [_p, _p, _p, ctypes.c_int, _i64, _i64, _i64, _i64,
                                        _i64, _i64, _i64, _p, _i64, _p]),
    "rmm_gemv_workspace_size": (ctypes.c_size_t, [_i64, _i64, _i64, _i64]),
    "rmm_select_tokens": (ctypes.c_int, [_p, ctypes.c_int, _i64, _i64, _i64, _i64, _p, _p]),
    "rmm_reduced_gemv": (ctypes.c_int, [_p, _p, _p, ctypes.c_int, _i64, _i64, _i64, _i64,
                                        _i64, _i64, _i64, _p, _i64, _p, ctypes.c_size_t, _p]),
    "rmm_reduced_qk": (ctypes.c_int, [_p, _p, _p, ctypes.c_int, _i64, _i64, _i64, _i64, _i64,
                                      _i64, _i64, ctypes.c_float, ctypes.c_int, _p, _p]),
    "rmm_linear": (ctypes.c_int, [_p, _p, ctypes.c_double, ctypes.c_int, _i64, _i64, _i64,
                                  _i64, _i64, _i64, _p, _i64, _p, _p, ctypes.c_size_t, _p]),
    "rmm_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "rmm_noalloc_scratch_bytes": (ctypes.c_size_t, []),
    "rmm_rmsnorm_kmajor_workspace_size": (ctypes.c_size_t, [_i64, _i64, _i64]),
    "rmm_attention_weights_kmajor_workspace_size": (ctypes.c_size_t, [_i64, _i64, _i64, _i64]),
    "rmm_attention_weights_kmajor": (ctypes.c_int, [_p, _i64, _i64, _i64, _i64, _i64, ctypes.c_int,
                                                    _p, _i64, _p, _p, ctypes.c_size_t, _p]),
    "rmm_reduced_qk_rowstats": (ctypes.c_int, [_p, _p, _p, _i64, _i64, _i64, _i64, _i64, _i64, _i64,
                                               ctypes.c_float, ctypes.c_int, _p, _p, _p, _p]),
    "rmm_attention_weights_kmajor_rowstats": (ctypes.c_int, [_p, _i64, _i64, _i64, _i64, _i64,
                                                             ctypes.c_int, _p, _p, _p, _i64, _p, _p,
                                                             ctypes.c_size_t, _p]),
    "rmm_decode_step_workspace_size": (ctypes.c_size_t, [ctypes.POINTER(DecodeGroup), ctypes.c_int,
                                                         _i64]),
    "rmm_decode_step": (ctypes.c_int, [ctypes.POINTER(DecodeGroup), ctypes.c_int, _i64, _p,
                                       ctypes.c_size_t, _p]),
    "rmm_decode_products": (ctypes.c_int, [ctypes.POINTER(DecodeGroup), ctypes.c_int, _i64, _p,
                                       ctypes.c_size_t, _p]),
    "rmm_decode_products_shared_workspace_size": (ctypes.c_size_t, [ctypes.POINTER(DecodeGroup),
                                                                    ctypes.c_int, _i64]),
    "rmm_decode_products_shared": (ctypes.c_int, [ctypes.POINTER(DecodeGroup), ctypes.c_int, _i64,
                                                  _p, ctypes.c_size_t, _p]),
    "rmm_decode_step_shared": (ctypes.c_int, [ctypes.POINTER(DecodeGroup), ctypes.c_int, _i64, _p,
                                              ctypes.c_size_t, _p]),
    "rmm_reduced_pv_kmajor": (ctypes.c_int, [_p, _p, _p, _i64, _i64, _i64, _i64, _i64, _i64, _i64,
                                             _i64, ctypes.c_int, _p, _p]),
    "rmm_rmsnorm_kmajor": (ctypes.c_int, [_p, _p, ctypes.c_float, _i64, _i64, _i64, _i64, _p, _i64,
                                          _p, _p, ctypes.c_size_t, _p]),
    "rmm_linear_noalloc": (ctypes.c_int, [_p, _p, ctypes.c_double, ctypes.c_int, _i64, _i64, _i64,
                                          _i64, _i64, _i64, _p, _i64, _p, _p]),
    "rmm_score_kmajor": (ctypes.c_int, [_p, _i64, _i64, _i64, _i64, _p, _p, _i64, _p,
                                        ctypes.c_size_t, _p]),
    "rmm_reduced_gemm_kmajor": (ctypes.c_int, [_p, _p, _p, _i64, _i64, _i64, _i64, _i64, _i64,
                                               _i64, _p, _i64, _p]),
    "rmm_reduced_attention": (ctypes.c_int, [_p, _p, _p, _p, ctypes.c_int, _i64, _i64, _i64, _i64,
                                             _i64, _i64, _i64, ctypes.c_float, ctypes.c_int, _p,
                                             _p, ctypes.c_size_t, _p]),
    "rmm_reduced_pv": (ctypes.c_int, [_p, _p, ctypes.c_int, _i64, _i64, _i64, _i64, _i64, _i64,
                                      _i64, _i64, _p, _p, _p, ctypes.c_size_t, _p]),
    "rmm_attention_kmajor_workspace_size": (ctypes.c_size_t, [_i64, _i64, _i64, _i64, _i64, _i64]),
    "rmm_gemm_swiglu_workspace_size": (ctypes.c_size_t, [_i64, _i64, _i64]),
    "rmm_check_indices": (ctypes.c_int, [_p, _i64, _i64, _i64, _p, _p]),
    "rmm_reduced_gemm_swiglu_kmajor": (ctypes.c_int, [_p, _p, _p, _i64, _i64, _i64, _i64, _i64,
                                                      _i64, _i64, _p, _i64, _p, _p,
                                                      ctypes.c_size_t, _p]),
    "rmm_reduced_attention_kmajor": (ctypes.c_int, [_p, _p, _p, _p, ctypes.c_int, _i64, _i64, _i64,
                                                    _i64, _i64, _i64, _i64, ctypes.c_float,
                                                    ctypes.c_int, _p, _i64, _p, _p, ctypes.c_size_t,
                                                    _p]),
    "rmm_qk_norm_rope_workspace_size": (ctypes.c_size_t, [_i64, _i64, _i64, _i64]),
    "rmm_qk_norm_rope": (ctypes.c_int, [ctypes.c_int, _i64, _i64, _i64, _p, _p, _p, _p, _p, _p,
                                        ctypes.c_float, _p, _p, _p, _p, ctypes.c_size_t, _p]),
    "rmm_kv_append": (ctypes.c_int, [_i64, _p, _p, _p, _p, _p, _p, _p, _p, ctypes.c_float, _p, _p,
                                     _p]),
    "rmm_kv_gather": (ctypes.c_int, [_p, _p, _i64, _p, _p, _p]),
    "rmm_paged_attention_workspace_size": (ctypes.c_size_t, [_i64, _i64, _i64, _i64, _i64]),
    "rmm_paged_attention": (ctypes.c_int, [_i64, _p, _p, _p, _i64, _i64, _p, _i64, _p, _p, _i64,
                                           ctypes.c_float, ctypes.c_int, _p, _p, ctypes.c_size_t, _p]),
}
EXPORTED_SYMBOLS = tuple(_SIGS)


class RmmError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn} failed: {rmm_status_string(status)} (status {status})")


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"librmm.so is missing at {LIB_PATH}; build it with "
                          "`python paper_2608_13426_amd/build.py`")
    handle = ctypes.CDLL(LIB_PATH)
    for name, (res, args) in _SIGS.items():
        fn = getattr(handle, name)
        fn.restype = res
        fn.argtypes = args
    return handle


lib = _load()


# ---------------------------------------------------------------- helpers

def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return RMM_BF16
    if t.dtype == torch.float32:
        return RMM_F32
    raise TypeError(f"unsupported dtype {t.dtype}; librmm takes bfloat16 or float32")


def _dev(*ts: torch.Tensor) -> torch.device:
    d = ts[0].device
    for t in ts:
        if t.device.type != "cuda":
            raise ValueError("librmm tensors must live on the GPU")
        if t.device != d:
            raise ValueError("all tensors must be on one device")
    return d


def _stream(device: torch.device, stream) -> int:
    if stream is None:
        return torch.cuda.current_stream(device).cuda_stream
    if stream.device != device:
        raise ValueError("the stream must be one of the tensors' device")
    return stream.cuda_stream


def _ptr(t):
    return None if t is None else t.data_ptr()


def _scratch(n: int, device: torch.device, stream, dtype=torch.uint8) -> torch.Tensor:
    """n elements for a call on `stream` (None: the current one), from that stream's
    pool: a block that the pool hands out again is then still in use at most by
    earlier work of the same stream, which the call follows."""
    if stream is None:
        return torch.empty(max(n, 1), dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(max(n, 1), dtype=dtype, device=device)


def _rows(t: torch.Tensor, name: str):
    """View a [U, M, K] or [M, K] tensor as U units of M rows with stride ldx."""
    if t.dim() == 2:
        t3 = t.unsqueeze(0)
    elif t.dim() == 3:
        t3 = t
    else:
        raise ValueError(f"{name} must be 2-D or 3-D")
    U, M, K = t3.shape
    if t3.stride(2) != 1:
        raise ValueError(f"{name} rows must be contiguous")
    ldx = t3.stride(1)
    if U > 1 and t3.stride(0) != M * ldx:
        raise ValueError(f"{name} units must be packed (stride M*ldx)")
    return U, M, K, ldx


def _check(fn: str, status: int):
    if status != 0:
        raise RmmError(fn, status)


# ---------------------------------------------------------------- C-ABI

def rmm_retained_count(r: float, K: int) -> int:
    """k = ceil(r*K) (Sec. 3.2); -1 for r outside (0, 1] or K < 1."""
    return int(lib.rmm_retained_count(float(r), int(K)))


def rmm_workspace_size(op: int, B: int, M: int, K: int, k: int = 0) -> int:
    return int(lib.rmm_workspace_size(int(op), int(B), int(M), int(K), int(k)))


def rmm_status_string(status: int) -> str:
    return lib.rmm_status_string(int(status)).decode()


def rmm_score(X: torch.Tensor, energy: torch.Tensor, workspace: torch.Tensor | None = None,
              stream=None) -> torch.Tensor:
    """Column energies of each unit of X ([B, M, K] or [M, K]) into float64 energy [B, K]."""
    B, M, K, ldx = _rows(X, "X")
    d = _dev(X, energy)
    if energy.dtype != torch.float64 or energy.numel() != B * K or not energy.is_contiguous():
        raise ValueError("energy must be a contiguous float64 tensor of B*K elements")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check("rmm_score", lib.rmm_score(X.data_ptr(), _dtype_code(X), B, M, K, ldx,
                                      energy.data_ptr(), _ptr(workspace), ws_bytes,
                                      _stream(d, stream)))
    return energy


def rmm_score_kmajor(X: torch.Tensor, energy: torch.Tensor, Xt: torch.Tensor,
                     workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Energies of each unit of bf16 X [B, M, K] plus its K-major copy Xt [B, K, ldxt]."""
    B, M, K, ldx = _rows(X, "X")
    d = _dev(X, energy, Xt)
    if energy.dtype != torch.float64 or energy.numel() != B * K or not energy.is_contiguous():
        raise ValueError("energy must be a contiguous float64 tensor of B*K elements")
    Bt, Kt, Mt, ldxt = _rows(Xt, "Xt")
    if (Bt, Kt, Mt) != (B, K, M) or Xt.dtype != X.dtype:
        raise ValueError("Xt must be [B, K, M] (a view with row stride ldxt) of X's dtype")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check("rmm_score_kmajor", lib.rmm_score_kmajor(
        X.data_ptr(), B, M, K, ldx, energy.data_ptr(), Xt.data_ptr(), ldxt, _ptr(workspace),
        ws_bytes, _stream(d, stream)))
    return energy


def rmm_select(energy: torch.Tensor, k: int, idx: torch.Tensor, stream=None) -> torch.Tensor:
    """TopK (ascending int32 indices) of each unit's energies.

    energy holds B units of K float64 energies ([B, K], or flat); idx holds
    B*k int32 slots, from which B is read.
    """
    d = _dev(energy, idx)
    k = int(k)
    if energy.dtype != torch.float64 or not energy.is_contiguous():
        raise ValueError("energy must be contiguous float64")
    if idx.dtype != torch.int32 or not idx.is_contiguous() or k < 1 or idx.numel() % k:
        raise ValueError("idx must be a contiguous int32 tensor of B*k elements")
    B = idx.numel() // k
    if B < 1 or energy.numel() % B:
        raise ValueError("energy must hold B*K values")
    K = energy.numel() // B
    _check("rmm_select", lib.rmm_select(energy.data_ptr(), B, K, k, idx.data_ptr(),
                                        _stream(d, stream)))
    return idx


def rmm_reduced_gemm(X: torch.Tensor, W: torch.Tensor, idx: torch.Tensor, Y: torch.Tensor,
                     stream=None) -> torch.Tensor:
    """Y[b] = X[b][:, I_b] @ W[I_b, :] for X [B, M, K], W [K, N], idx [B, k], Y [B, M, N]."""
    B, M, K, ldx = _rows(X, "X")
    d = _dev(X, W, idx, Y)
    if W.dim() != 2 or W.shape[0] != K or W.stride(1) != 1:
        raise ValueError("W must be [K, N] with contiguous rows")
    N, ldw = W.shape[1], W.stride(0)
    By, My, Ny, ldy = _rows(Y, "Y")
    if (By, My, Ny) != (B, M, N):
        raise ValueError("Y must be [B, M, N]")
    if not (X.dtype == W.dtype == Y.dtype):
        raise TypeError("X, W and Y must share one dtype")
    if idx.dtype != torch.int32 or not idx.is_contiguous() or idx.numel() % B:
        raise ValueError("idx must be contiguous int32 [B, k]")
    k = idx.numel() // B
    _check("rmm_reduced_gemm", lib.rmm_reduced_gemm(
        X.data_ptr(), W.data_ptr(), idx.data_ptr(), _dtype_code(X), B, M, N, K, k, ldx, ldw,
        Y.data_ptr(), ldy, _stream(d, stream)))
    return Y


def rmm_check_indices(idx: torch.Tensor, K: int, bad: torch.Tensor | None = None,
                      stream=None) -> torch.Tensor:
    """Per unit of idx [B, k]: 0 if its list is strictly ascending within
    [0, K), else 1 + the first position that breaks it (int32 [B])."""
    if idx.dim() == 1:
        idx = idx.unsqueeze(0)
    if idx.dtype != torch.int32 or not idx.is_contiguous() or idx.dim() != 2:
        raise ValueError("idx must be contiguous int32 [B, k]")
    B, k = idx.shape
    if bad is None:
        bad = _scratch(B, idx.device, stream, torch.int32)[:B]
        if stream is not None:              # the caller reads it on the current one
            bad.record_stream(torch.cuda.current_stream(idx.device))
    d = _dev(idx, bad)
    if bad.dtype != torch.int32 or bad.numel() != B or not bad.is_contiguous():
        raise ValueError("bad must be contiguous int32 [B]")
    _check("rmm_check_indices", lib.rmm_check_indices(idx.data_ptr(), B, k, int(K), bad.data_ptr(),
                                                      _stream(d, stream)))
    return bad


def rmm_select_tokens(X: torch.Tensor, k: int, idx: torch.Tensor, stream=None) -> torch.Tensor:
    """TopK of X[b][j]^2 per row of X [B, K] (or [B, 1, K]: one token per unit),
    ascending, into idx (int32, B*k)."""
    if X.dim() == 3:
        if X.shape[1] != 1:
            raise ValueError("X must hold one token per unit")
        X = X[:, 0, :]
    if X.dim() != 2 or X.stride(1) != 1:
        raise ValueError("X must be [B, K] with contiguous rows")
    B, K = X.shape
    d = _dev(X, idx)
    if idx.dtype != torch.int32 or not idx.is_contiguous() or idx.numel() != B * k:
        raise ValueError("idx must be contiguous int32 with B*k elements")
    _check("rmm_select_tokens", lib.rmm_select_tokens(
        X.data_ptr(), _dtype_code(X), B, K, X.stride(0), int(k), idx.data_ptr(), _stream(d, stream)))
    return idx


def rmm_gemv_workspace_size(B: int, M: int, N: int, k: int) -> int:
    return int(lib.rmm_gemv_workspace_size(int(B), int(M), int(N), int(k)))


def rmm_reduced_gemv(X: torch.Tensor, W: torch.Tensor, idx: torch.Tensor, Y: torch.Tensor,
                     workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """Decode-step form of rmm_reduced_gemm (M <= 8 rows per unit, bf16):
    Y[b] = X[b][:, I_b] @ W[I_b, :]; `workspace` (uint8,
    rmm_gemv_workspace_size(B, M, N, k) bytes) is allocated here when not given."""
    B, M, K, ldx = _rows(X, "X")
    d = _dev(X, W, idx, Y)
    if W.dim() != 2 or W.shape[0] != K or W.stride(1) != 1:
        raise ValueError("W must be [K, N] with contiguous rows")
    N, ldw = W.shape[1], W.stride(0)
    By, My, Ny, ldy = _rows(Y, "Y")
    if (By, My, Ny) != (B, M, N):
        raise ValueError("Y must be [B, M, N]")
    if not (X.dtype == W.dtype == Y.dtype):
        raise TypeError("X, W and Y must share one dtype")
    if idx.dtype != torch.int32 or not idx.is_contiguous() or idx.numel() % B:
        raise ValueError("idx must be contiguous int32 [B, k]")
    k = idx.numel() // B
    if workspace is None:
        need = rmm_gemv_workspace_size(B, M, N, k)
        workspace = _scratch(need, d, stream)
    ws_bytes = workspace.numel() * workspace.element_size()
    _check("rmm_reduced_gemv", lib.rmm_reduced_gemv(
        X.data_ptr(), W.data_ptr(), idx.data_ptr(), _dtype_code(X), B, M, N, K, k, ldx, ldw,
        Y.data_ptr(), ldy, workspace.data_ptr(), ws_bytes, _stream(d, stream)))
    return Y


def rmm_reduced_gemm_kmajor(Xt: torch.Tensor, W: torch.Tensor, idx: torch.Tensor,
                            Y: torch.Tensor, stream=None) -> torch.Tensor:
    """Y[b] = X[b][:, I_b] @ W[I_b, :] from the K-major copy Xt [B, K, M]."""
    B, K, M, ldxt = _rows(Xt, "Xt")
    d = _dev(Xt, W, idx, Y)
    if W.dim() != 2 or W.shape[0] != K or W.stride(1) != 1:
        raise ValueError("W must be [K, N] with contiguous rows")
    N, ldw = W.shape[1], W.stride(0)
    By, My, Ny, ldy = _rows(Y, "Y")
    if (By, My, Ny) != (B, M, N):
        raise ValueError("Y must be [B, M, N]")
    if not (Xt.dtype == W.dtype == Y.dtype == torch.bfloat16):
        raise TypeError("Xt, W and Y must be bfloat16")
    if idx.dtype != torch.int32 or not idx.is_contiguous() or idx.numel() % B:
        raise ValueError("idx must be contiguous int32 [B, k]")
    k = idx.numel() // B
    _check("rmm_reduced_gemm_kmajor", lib.rmm_reduced_gemm_kmajor(
        Xt.data_ptr(), W.data_ptr(), idx.data_ptr(), B, M, N, K, k, ldxt, ldw, Y.data_ptr(),
        ldy, _stream(d, stream)))
    return Y


def swiglu_weight_layout(Wg: torch.Tensor, Wu: torch.Tensor) -> torch.Tensor:
    """The gate and up weights [K, F] as rmm_reduced_gemm_swiglu_kmajor reads
    them: [K, 2F] in 128-column blocks, gate then up of the same 128 channels
    (a column permutation, made once at load time)."""
    if Wg.shape != Wu.shape or Wg.dim() != 2 or Wg.shape[1] % 128:
        raise ValueError("Wg and Wu must be [K, F] with F a multiple of 128")
    K, F = Wg.shape
    return torch.stack([Wg.reshape(K, F // 128, 128), Wu.reshape(K, F // 128, 128)],
                       dim=2).reshape(K, 2 * F).contiguous()


def rmm_gemm_swiglu_workspace_size(B: int, M: int, F: int) -> int:
    return int(lib.rmm_gemm_swiglu_workspace_size(B, M, F))


def rmm_reduced_gemm_swiglu_kmajor(Xt: torch.Tensor, Wgu: torch.Tensor, idx: torch.Tensor,
                                   Ht: torch.Tensor, energy: torch.Tensor,
                                   workspace: torch.Tensor | None = None,
                                   stream=None) -> torch.Tensor:
    """The reduced gate|up product from the K-major copy Xt [B, K, M] with the
    SwiGLU epilogue: writes the down projection's K-major input Ht [B, F, M]
    (rows of stride ldht >= M) and its column energies energy float64 [B, F].
    Wgu [K, 2F] in the layout of swiglu_weight_layout; idx [B, k]."""
    B, K, M, ldxt = _rows(Xt, "Xt")
    if Ht.dim() == 2:
        Ht = Ht.unsqueeze(0)
    if energy.dim() == 1:
        energy = energy.unsqueeze(0)
    d = _dev(Xt, Wgu, idx, Ht, energy)
    if Wgu.dim() != 2 or Wgu.shape[0] != K or Wgu.stride(1) != 1 or Wgu.shape[1] % 2:
        raise ValueError("Wgu must be [K, 2F] with contiguous rows")
    F, ldw = Wgu.shape[1] // 2, Wgu.stride(0)
    if Ht.shape[0] != B or Ht.shape[1] != F or Ht.shape[2] != M:
        raise ValueError("Ht must be [B, F, M]")
    if Ht.stride(2) != 1 or (B > 1 and Ht.stride(0) != F * Ht.stride(1)):
        raise ValueError("Ht rows must be contiguous, with one row stride ldht")
    if tuple(energy.shape) != (B, F) or not energy.is_contiguous() or energy.dtype != torch.float64:
        raise ValueError("energy must be contiguous float64 [B, F]")
    if not (Xt.dtype == Wgu.dtype == Ht.dtype == torch.bfloat16):
        raise TypeError("Xt, Wgu and Ht must be bfloat16")
    if idx.dtype != torch.int32 or not idx.is_contiguous() or idx.numel() % B:
        raise ValueError("idx must be contiguous int32 [B, k]")
    k = idx.numel() // B
    if workspace is None:
        workspace = _scratch(rmm_gemm_swiglu_workspace_size(B, M, F), d, stream)
    ws_bytes = workspace.numel() * workspace.element_size()
    _check("rmm_reduced_gemm_swiglu_kmajor", lib.rmm_reduced_gemm_swiglu_kmajor(
        Xt.data_ptr(), Wgu.data_ptr(), idx.data_ptr(), B, M, F, K, k, ldxt, ldw, Ht.data_ptr(),
        Ht.stride(1), energy.data_ptr(), workspace.data_ptr(), ws_bytes, _stream(d, stream)))
    return Ht


def rmm_reduced_qk(Q: torch.Tensor, Kc: torch.Tensor, idx: torch.Tensor, S: torch.Tensor,
                   causal: bool = True, scale: float | None = None, stream=None) -> torch.Tensor:
    """Reduced scores for Q [batch, H, Lq, D], Kc [batch, Hkv, Lk, D], idx [batch, H, k]."""
    if Q.dim() == 3:
        Q, Kc, S = Q.unsqueeze(0), Kc.unsqueeze(0), S.unsqueeze(0)
    batch, H, Lq, D = Q.shape
    bk, Hkv, Lk, Dk = Kc.shape
    d = _dev(Q, Kc, idx, S)
    if bk != batch or Dk != D:
        raise ValueError("Kc must be [batch, Hkv, Lk, D]")
    if tuple(S.shape) != (batch, H, Lq, Lk):
        raise ValueError("S must be [batch, H, Lq, Lk]")
    for t, n in ((Q, "Q"), (Kc, "Kc"), (S, "S"), (idx, "idx")):
        if not t.is_contiguous():
            raise ValueError(f"{n} must be contiguous")
    if not (Q.dtype == Kc.dtype == S.dtype):
        raise TypeError("Q, Kc and S must share one dtype")
    if idx.dtype != torch.int32 or idx.numel() % (batch * H):
        raise ValueError("idx must be int32 [batch, H, k]")
    k = idx.numel() // (batch * H)
    if scale is None:
        scale = D ** -0.5
    _check("rmm_reduced_qk", lib.rmm_reduced_qk(
        Q.data_ptr(), Kc.data_ptr(), idx.data_ptr(), _dtype_code(Q), batch, H, Hkv, Lq, Lk, D,
        k, float(scale), 1 if causal else 0, S.data_ptr(), _stream(d, stream)))
    return S


def rmm_reduced_qk_rowstats(Q: torch.Tensor, Kc: torch.Tensor, idx: torch.Tensor, S: torch.Tensor,
                            row_max: torch.Tensor, row_rinv: torch.Tensor, causal: bool = True,
                            scale: float | None = None, stream=None) -> torch.Tensor:
    """rmm_reduced_qk (bf16) that also writes each score row's softmax
    statistics: row_max and row_rinv, float32 [batch*H*Lq]."""
    if Q.dim() != 4 or Kc.dim() != 4 or S.dim() != 4:
        raise ValueError("Q, Kc and S must be 4-D")
    batch, H, Lq, D = Q.shape
    bk, Hkv, Lk, Dk = Kc.shape
    d = _dev(Q, Kc, idx, S, row_max, row_rinv)
    if bk != batch or Dk != D or tuple(S.shape) != (batch, H, Lq, Lk):
        raise ValueError("shapes: Q [b, H, Lq, D], Kc [b, Hkv, Lk, D], S [b, H, Lq, Lk]")
    for t, n in ((Q, "Q"), (Kc, "Kc"), (S, "S"), (idx, "idx")):
        if not t.is_contiguous():
            raise ValueError(f"{n} must be contiguous")
    if not (Q.dtype == Kc.dtype == S.dtype == torch.bfloat16):
        raise TypeError("Q, Kc and S must be bfloat16")
    for t, n in ((row_max, "row_max"), (row_rinv, "row_rinv")):
        if t.dtype != torch.float32 or t.numel() != batch * H * Lq or not t.is_contiguous():
            raise ValueError(f"{n} must be contiguous float32 [batch*H*Lq]")
    if idx.dtype != torch.int32 or idx.numel() % (batch * H):
        raise ValueError("idx must be int32 [batch, H, k]")
    k = idx.numel() // (batch * H)
    if scale is None:
        scale = D ** -0.5
    _check("rmm_reduced_qk_rowstats", lib.rmm_reduced_qk_rowstats(
        Q.data_ptr(), Kc.data_ptr(), idx.data_ptr(), batch, H, Hkv, Lq, Lk, D, k, float(scale),
        1 if causal else 0, S.data_ptr(), row_max.data_ptr(), row_rinv.data_ptr(), _stream(d, stream)))
    return S


def rmm_reduced_attention(Q: torch.Tensor, Kc: torch.Tensor, V: torch.Tensor, idx: torch.Tensor,
                          O: torch.Tensor, causal: bool = True, scale: float | None = None,
                          workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """softmax(reduced scores + mask) V for Q [batch, H, Lq, D], Kc and V
    [batch, Hkv, Lk, D], idx [batch, H, k]; writes O [batch, H, Lq, D].
    `workspace` (uint8, rmm_workspace_size(RMM_OP_ATTENTION, batch*H, Lk, D, k)
    bytes) is allocated here when not given."""
    if Q.dim() == 3:
        Q, Kc, V, O = Q.unsqueeze(0), Kc.unsqueeze(0), V.unsqueeze(0), O.unsqueeze(0)
    batch, H, Lq, D = Q.shape
    bk, Hkv, Lk, Dk = Kc.shape
    d = _dev(Q, Kc, V, idx, O)
    if bk != batch or Dk != D:
        raise ValueError("Kc must be [batch, Hkv, Lk, D]")
    if tuple(V.shape) != (batch, Hkv, Lk, D):
        raise ValueError("V must be [batch, Hkv, Lk, D]")
    if tuple(O.shape) != (batch, H, Lq, D):
        raise ValueError("O must be [batch, H, Lq, D]")
    for t, n in ((Q, "Q"), (Kc, "Kc"), (V, "V"), (O, "O"), (idx, "idx")):
        if not t.is_contiguous():
            raise ValueError(f"{n} must be contiguous")
    if not (Q.dtype == Kc.dtype == V.dtype == O.dtype):
        raise TypeError("Q, Kc, V and O must share one dtype")
    if idx.dtype != torch.int32 or idx.numel() % (batch * H):
        raise ValueError("idx must be int32 [batch, H, k]")
    k = idx.numel() // (batch * H)
    if scale is None:
        scale = D ** -0.5
    if workspace is None:
        workspace = _scratch(rmm_workspace_size(RMM_OP_ATTENTION, batch * H, Lk, D, k), d, stream)
    ws_bytes = workspace.numel() * workspace.element_size()
    _check("rmm_reduced_attention", lib.rmm_reduced_attention(
        Q.data_ptr(), Kc.data_ptr(), V.data_ptr(), idx.data_ptr(), _dtype_code(Q), batch, H, Hkv,
        Lq, Lk, D, k, float(scale), 1 if causal else 0, O.data_ptr(), workspace.data_ptr(),
        ws_bytes, _stream(d, stream)))
    return O


def rmm_attention_kmajor_workspace_size(batch: int, H: int, Lq: int, Lk: int, D: int,
                                        k: int) -> int:
    return int(lib.rmm_attention_kmajor_workspace_size(batch, H, Lq, Lk, D, k))


def rmm_reduced_attention_kmajor(Q: torch.Tensor, Kc: torch.Tensor, V: torch.Tensor,
                                 idx: torch.Tensor, Ot: torch.Tensor, energy: torch.Tensor,
                                 causal: bool = True, scale: float | None = None,
                                 workspace: torch.Tensor | None = None,
                                 stream=None) -> torch.Tensor:
    """The reduced attention block of rmm_reduced_attention, written as the
    output projection's K-major input Ot [batch, H*D, ldot] (a view whose
    rows have stride ldot >= Lq) with that input's column energies
    energy float64 [batch, H*D].  `workspace` (uint8,
    rmm_attention_kmajor_workspace_size(...) bytes, 256-byte aligned) is
    allocated here when not given."""
    if Q.dim() == 3:
        Q, Kc, V = Q.unsqueeze(0), Kc.unsqueeze(0), V.unsqueeze(0)
    if Ot.dim() == 2:
        Ot = Ot.unsqueeze(0)
    if energy.dim() == 1:
        energy = energy.unsqueeze(0)
    batch, H, Lq, D = Q.shape
    bk, Hkv, Lk, Dk = Kc.shape
    d = _dev(Q, Kc, V, idx, Ot, energy)
    if bk != batch or Dk != D:
        raise ValueError("Kc must be [batch, Hkv, Lk, D]")
    if tuple(V.shape) != (batch, Hkv, Lk, D):
        raise ValueError("V must be [batch, Hkv, Lk, D]")
    if Ot.shape[0] != batch or Ot.shape[1] != H * D or Ot.shape[2] < Lq:
        raise ValueError("Ot must be [batch, H*D, >= Lq]")
    if Ot.stride(2) != 1 or Ot.stride(0) != Ot.shape[1] * Ot.stride(1):
        raise ValueError("Ot rows must be contiguous, with one row stride ldot")
    if tuple(energy.shape) != (batch, H * D) or not energy.is_contiguous() or \
            energy.dtype != torch.float64:
        raise ValueError("energy must be contiguous float64 [batch, H*D]")
    for t, n in ((Q, "Q"), (Kc, "Kc"), (V, "V"), (idx, "idx")):
        if not t.is_contiguous():
            raise ValueError(f"{n} must be contiguous")
    if not (Q.dtype == Kc.dtype == V.dtype == Ot.dtype):
        raise TypeError("Q, Kc, V and Ot must share one dtype")
    if idx.dtype != torch.int32 or idx.numel() % (batch * H):
        raise ValueError("idx must be int32 [batch, H, k]")
    k = idx.numel() // (batch * H)
    if scale is None:
        scale = D ** -0.5
    if workspace is None:
        workspace = _scratch(rmm_attention_kmajor_workspace_size(batch, H, Lq, Lk, D, k), d, stream)
    ws_bytes = workspace.numel() * workspace.element_size()
    _check("rmm_reduced_attention_kmajor", lib.rmm_reduced_attention_kmajor(
        Q.data_ptr(), Kc.data_ptr(), V.data_ptr(), idx.data_ptr(), _dtype_code(Q), batch, H, Hkv,
        Lq, Lk, D, k, float(scale), 1 if causal else 0, Ot.data_ptr(), Ot.stride(1),
        energy.data_ptr(), workspace.data_ptr(), ws_bytes, _stream(d, stream)))
    return Ot


def rmm_reduced_pv(P: torch.Tensor, V: torch.Tensor, kt: int, O: torch.Tensor,
                   idx_out: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                   stream=None) -> torch.Tensor:
    """Token-axis reduced value product (Sec. 3.3): per query head u, the kt
    tokens with the largest column norms of P[u] and O[u] = P[u][:, T] @
    V[kv(u)][T, :].  P: [batch, H, Lq, Lk] (rows contiguous, any row stride),
    V: [batch, Hkv, Lk, D] contiguous, O: [batch, H, Lq, D] contiguous;
    `idx_out` (int32 [batch*H*kt]) receives the token sets when given."""
    if P.dim() != 4 or V.dim() != 4 or O.dim() != 4:
        raise ValueError("P, V and O must be 4-D")
    batch, H, Lq, Lk = P.shape
    if P.stride(3) != 1 or P.stride(1) != Lq * P.stride(2) or P.stride(0) != H * P.stride(1):
        raise ValueError("P must be [batch, H, Lq, Lk] with contiguous rows and packed rows")
    ldp = P.stride(2)
    if V.shape[0] != batch or V.shape[2] != Lk or not V.is_contiguous():
        raise ValueError("V must be contiguous [batch, Hkv, Lk, D]")
    Hkv, D = V.shape[1], V.shape[3]
    if tuple(O.shape) != (batch, H, Lq, D) or not O.is_contiguous():
        raise ValueError("O must be contiguous [batch, H, Lq, D]")
    d = _dev(P, V, O)
    if not (P.dtype == V.dtype == O.dtype):
        raise TypeError("P, V and O must share one dtype")
    if idx_out is not None and (idx_out.dtype != torch.int32 or idx_out.numel() != batch * H * kt
                                or not idx_out.is_contiguous()):
        raise ValueError("idx_out must be contiguous int32 [batch*H*kt]")
    if workspace is None:
        workspace = _scratch(rmm_workspace_size(RMM_OP_PV, batch * H, Lq, Lk, kt), d, stream)
    ws_bytes = workspace.numel() * workspace.element_size()
    _check("rmm_reduced_pv", lib.rmm_reduced_pv(
        P.data_ptr(), V.data_ptr(), _dtype_code(P), batch, H, Hkv, Lq, Lk, D, ldp, int(kt),
        O.data_ptr(), _ptr(idx_out), workspace.data_ptr(), ws_bytes, _stream(d, stream)))
    return O


def rmm_linear(X: torch.Tensor, W: torch.Tensor, r: float, Y: torch.Tensor,
               idx_out: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
               stream=None) -> torch.Tensor:
    """Fused score -> select -> gathered GEMM at retention ratio r."""
    B, M, K, ldx = _rows(X, "X")
    d = _dev(X, W, Y)
    if W.dim() != 2 or W.shape[0] != K or W.stride(1) != 1:
        raise ValueError("W must be [K, N] with contiguous rows")
    N, ldw = W.shape[1], W.stride(0)
    By, My, Ny, ldy = _rows(Y, "Y")
    if (By, My, Ny) != (B, M, N):
        raise ValueError("Y must be [B, M, N]")
    if not (X.dtype == W.dtype == Y.dtype):
        raise TypeError("X, W and Y must share one dtype")
    k = rmm_retained_count(r, K)
    if idx_out is not None and (idx_out.dtype != torch.int32 or idx_out.numel() != B * max(k, 0)
                                or not idx_out.is_contiguous()):
        raise ValueError("idx_out must be contiguous int32 [B, k]")
    if workspace is None:
        workspace = _scratch(rmm_workspace_size(RMM_OP_LINEAR, B, M, K, k), d, stream)
    ws_bytes = workspace.numel() * workspace.element_size()
    _check("rmm_linear", lib.rmm_linear(
        X.data_ptr(), W.data_ptr(), float(r), _dtype_code(X), B, M, N, K, ldx, ldw,
        Y.data_ptr(), ldy, _ptr(idx_out), workspace.data_ptr(), ws_bytes, _stream(d, stream)))
    return Y


def rmm_noalloc_scratch_bytes() -> int:
    return int(lib.rmm_noalloc_scratch_bytes())


def rmm_linear_noalloc(X: torch.Tensor, W: torch.Tensor, r: float, Y: torch.Tensor,
                       idx_out: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """rmm_linear with the library's fixed scratch instead of a workspace:
    neither this wrapper nor the call allocates device memory (usable under
    HIP graph capture).  Calls that overlap in time on one GPU race."""
    B, M, K, ldx = _rows(X, "X")
    d = _dev(X, W, Y)
    if W.dim() != 2 or W.shape[0] != K or W.stride(1) != 1:
        raise ValueError("W must be [K, N] with contiguous rows")
    N, ldw = W.shape[1], W.stride(0)
    By, My, Ny, ldy = _rows(Y, "Y")
    if (By, My, Ny) != (B, M, N):
        raise ValueError("Y must be [B, M, N]")
    if not (X.dtype == W.dtype == Y.dtype):
        raise TypeError("X, W and Y must share one dtype")
    k = rmm_retained_count(r, K)
    if idx_out is not None and (idx_out.dtype != torch.int32 or idx_out.numel() != B * max(k, 0)
                                or not idx_out.is_contiguous()):
        raise ValueError("idx_out must be contiguous int32 [B, k]")
    _check("rmm_linear_noalloc", lib.rmm_linear_noalloc(
        X.data_ptr(), W.data_ptr(), float(r), _dtype_code(X), B, M, N, K, ldx, ldw,
        Y.data_ptr(), ldy, _ptr(idx_out), _stream(d, stream)))
    return Y


def rmm_rmsnorm_kmajor_workspace_size(B: int, M: int, K: int) -> int:
    return int(lib.rmm_rmsnorm_kmajor_workspace_size(int(B), int(M), int(K)))


def rmm_rmsnorm_kmajor(X: torch.Tensor, gamma: torch.Tensor, eps: float, Xt: torch.Tensor,
                       energy: torch.Tensor, workspace: torch.Tensor | None = None,
                       stream=None) -> torch.Tensor:
    """RMSNorm of X [B, M, K] (or [M, K]) with weight gamma [K], written
    K-major into Xt [B, K, M] (row stride Xt.stride(-2)) with the column
    energies of the normalised rows in energy (float64 [B*K])."""
    B, M, K, ldx = _rows(X, "X")
    d = _dev(X, gamma, Xt, energy)
    Bt, Kt, Mt, ldxt = _rows(Xt, "Xt")
    if (Bt, Kt, Mt) != (B, K, M):
        raise ValueError("Xt must be [B, K, M]")
    if gamma.numel() != K or not gamma.is_contiguous():
        raise ValueError("gamma must be a contiguous [K] tensor")
    if not (X.dtype == gamma.dtype == Xt.dtype == torch.bfloat16):
        raise TypeError("X, gamma and Xt must be bfloat16")
    if energy.dtype != torch.float64 or energy.numel() != B * K or not energy.is_contiguous():
        raise ValueError("energy must be contiguous float64 [B*K]")
    if workspace is None:
        workspace = _scratch(rmm_rmsnorm_kmajor_workspace_size(B, M, K), d, stream)
    ws_bytes = workspace.numel() * workspace.element_size()
    _check("rmm_rmsnorm_kmajor", lib.rmm_rmsnorm_kmajor(
        X.data_ptr(), gamma.data_ptr(), float(eps), B, M, K, ldx, Xt.data_ptr(), ldxt,
        energy.data_ptr(), workspace.data_ptr(), ws_bytes, _stream(d, stream)))
    return Xt


def rmm_attention_weights_kmajor_workspace_size(batch: int, H: int, Lq: int, Lk: int) -> int:
    return int(lib.rmm_attention_weights_kmajor_workspace_size(batch, H, Lq, Lk))


def rmm_attention_weights_kmajor(S: torch.Tensor, Pt: torch.Tensor, energy: torch.Tensor,
                                 causal: bool = True, workspace: torch.Tensor | None = None,
                                 stream=None, row_max: torch.Tensor | None = None,
                                 row_rinv: torch.Tensor | None = None) -> torch.Tensor:
    """Softmax weights of the scores S [batch, H, Lq, Lk] written K-major into
    Pt [batch, H, Lk, Lq] (row stride Pt.stride(-2)), with their token
    energies (float64 [batch*H*Lk]).  With row_max and row_rinv (float32
    [batch*H*Lq], e.g. from rmm_reduced_qk_rowstats) the weights use those
    row statistics (rmm_attention_weights_kmajor_rowstats)."""
    if S.dim() != 4 or Pt.dim() != 4:
        raise ValueError("S and Pt must be 4-D")
    batch, H, Lq, Lk = S.shape
    d = _dev(S, Pt, energy)
    if tuple(Pt.shape) != (batch, H, Lk, Lq):
        raise ValueError("Pt must be [batch, H, Lk, Lq]")
    if S.stride(3) != 1 or S.stride(1) != Lq * S.stride(2) or S.stride(0) != H * Lq * S.stride(2):
        raise ValueError("S rows must be contiguous and its heads packed")
    if Pt.stride(3) != 1 or Pt.stride(1) != Lk * Pt.stride(2) or Pt.stride(0) != H * Lk * Pt.stride(2):
        raise ValueError("Pt rows must be contiguous and its heads packed")
    if not (S.dtype == Pt.dtype == torch.bfloat16):
        raise TypeError("S and Pt must be bfloat16")
    if energy.dtype != torch.float64 or energy.numel() != batch * H * Lk or not energy.is_contiguous():
        raise ValueError("energy must be contiguous float64 [batch*H*Lk]")
    if workspace is None:
        workspace = _scratch(rmm_attention_weights_kmajor_workspace_size(batch, H, Lq, Lk), d, stream)
    ws_bytes = workspace.numel() * workspace.element_size()
    if (row_max is None) != (row_rinv is None):
        raise ValueError("give both row_max and row_rinv, or neither")
    if row_max is None:
        _check("rmm_attention_weights_kmajor", lib.rmm_attention_weights_kmajor(
            S.data_ptr(), batch, H, Lq, Lk, S.stride(2), 1 if causal else 0, Pt.data_ptr(),
            Pt.stride(2), energy.data_ptr(), workspace.data_ptr(), ws_bytes, _stream(d, stream)))
        return Pt
    _dev(S, row_max, row_rinv)
    for t, n in ((row_max, "row_max"), (row_rinv, "row_rinv")):
        if t.dtype != torch.float32 or t.numel() != batch * H * Lq or not t.is_contiguous():
            raise ValueError(f"{n} must be contiguous float32 [batch*H*Lq]")
    _check("rmm_attention_weights_kmajor_rowstats", lib.rmm_attention_weights_kmajor_rowstats(
        S.data_ptr(), batch, H, Lq, Lk, S.stride(2), 1 if causal else 0, row_max.data_ptr(),
        row_rinv.data_ptr(), Pt.data_ptr(), Pt.stride(2), energy.data_ptr(), workspace.data_ptr(),
        ws_bytes, _stream(d, stream)))
    return Pt


def rmm_reduced_pv_kmajor(Pt: torch.Tensor, V: torch.Tensor, idx: torch.Tensor, O: torch.Tensor,
                          causal: bool = True, stream=None) -> torch.Tensor:
    """O[b, h] = Pt[b, h][T, :]^T V[b, h // (H/Hkv)][T, :] with the token sets
    idx [batch*H, kt] (ascending)."""
    if Pt.dim() != 4 or V.dim() != 4 or O.dim() != 4:
        raise ValueError("Pt, V and O must be 4-D")
    batch, H, Lk, Lq = Pt.shape
    _, Hkv, Lkv, D = V.shape
    d = _dev(Pt, V, idx, O)
    if Lkv != Lk or tuple(O.shape) != (batch, H, Lq, D) or H % Hkv:
        raise ValueError("shapes: Pt [b, H, Lk, Lq], V [b, Hkv, Lk, D], O [b, H, Lq, D]")
    if Pt.stride(3) != 1 or Pt.stride(1) != Lk * Pt.stride(2) or Pt.stride(0) != H * Lk * Pt.stride(2):
        raise ValueError("Pt rows must be contiguous and its heads packed")
    if not (V.is_contiguous() and O.is_contiguous()):
        raise ValueError("V and O must be contiguous")
    if not (Pt.dtype == V.dtype == O.dtype == torch.bfloat16):
        raise TypeError("Pt, V and O must be bfloat16")
    if idx.dtype != torch.int32 or not idx.is_contiguous() or idx.numel() % (batch * H):
        raise ValueError("idx must be contiguous int32 [batch*H, kt]")
    kt = idx.numel() // (batch * H)
    _check("rmm_reduced_pv_kmajor", lib.rmm_reduced_pv_kmajor(
        Pt.data_ptr(), V.data_ptr(), idx.data_ptr(), batch, H, Hkv, Lq, Lk, D, kt, Pt.stride(2),
        1 if causal else 0, O.data_ptr(), _stream(d, stream)))
    return O


def _decode_groups(groups):
    """[(X [B, K], W [K, N], k, idx [B*k] int32, Y [B, N])] -> ctypes array, B."""
    arr = (DecodeGroup * len(groups))()
    B = None
    for i, (X, W, k, idx, Y) in enumerate(groups):
        if X.dim() != 2 or W.dim() != 2 or Y.dim() != 2:
            raise ValueError("X [B, K], W [K, N] and Y [B, N] must be 2-D")
        if B is None:
            B = X.shape[0]
        if X.shape[0] != B or Y.shape[0] != B or W.shape[0] != X.shape[1] or Y.shape[1] != W.shape[1]:
            raise ValueError("group shapes disagree: X [B, K], W [K, N], Y [B, N]")
        if X.stride(1) != 1 or W.stride(1) != 1 or Y.stride(1) != 1:
            raise ValueError("rows must be contiguous")
        if not (X.dtype == W.dtype == Y.dtype == torch.bfloat16):
            raise TypeError("X, W and Y must be bfloat16")
        if idx.dtype != torch.int32 or idx.numel() != B * k or not idx.is_contiguous():
            raise ValueError("idx must be contiguous int32 [B*k]")
        _dev(X, W, idx, Y)
        arr[i] = DecodeGroup(X.data_ptr(), W.data_ptr(), idx.data_ptr(), Y.data_ptr(), X.shape[1],
                             W.shape[1], int(k), X.stride(0), W.stride(0), Y.stride(0))
    return arr, B


def rmm_decode_step_workspace_size(groups) -> int:
    arr, B = _decode_groups(groups)
    return int(lib.rmm_decode_step_workspace_size(arr, len(groups), B))


def rmm_decode_products(groups, workspace: torch.Tensor | None = None, stream=None):
    """For each group (X [B, K], W [K, N], k, idx [B*k], Y [B, N]) with idx
    holding caller-made ascending sets: Y = the reduced product; all groups
    in two launches (rmm_decode_step without its selection)."""
    arr, B = _decode_groups(groups)
    d = groups[0][0].device
    need = int(lib.rmm_decode_step_workspace_size(arr, len(groups), B))
    if workspace is None and need > 0:
        workspace = _scratch(need, d, stream)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check("rmm_decode_products", lib.rmm_decode_products(arr, len(groups), B, _ptr(workspace),
                                                          ws_bytes, _stream(d, stream)))


def rmm_decode_products_shared_workspace_size(groups) -> int:
    arr, B = _decode_groups(groups)
    return int(lib.rmm_decode_products_shared_workspace_size(arr, len(groups), B))


def rmm_decode_products_shared(groups, workspace: torch.Tensor | None = None, stream=None):
    """The same products as rmm_decode_products (B <= 32 sequences), reading
    each weight row that some sequence keeps once for the whole batch; equal
    to it within rounding."""
    arr, B = _decode_groups(groups)
    d = groups[0][0].device
    if workspace is None:
        need = int(lib.rmm_decode_products_shared_workspace_size(arr, len(groups), B))
        workspace = _scratch(need, d, stream)
    ws_bytes = workspace.numel() * workspace.element_size()
    _check("rmm_decode_products_shared",
           lib.rmm_decode_products_shared(arr, len(groups), B, _ptr(workspace), ws_bytes,
                                          _stream(d, stream)))


def rmm_decode_step_shared(groups, workspace: torch.Tensor | None = None, stream=None):
    """For each group (X [B, K], W [K, N], k, idx [B*k], Y [B, N]), B <= 32:
    idx = each token's TopK (as rmm_decode_step), Y = the shared-rows
    products over those sets (rmm_decode_products_shared)."""
    arr, B = _decode_groups(groups)
    d = groups[0][0].device
    if workspace is None:
        need = int(lib.rmm_decode_products_shared_workspace_size(arr, len(groups), B))
        workspace = _scratch(need, d, stream)
    ws_bytes = workspace.numel() * workspace.element_size()
    _check("rmm_decode_step_shared",
           lib.rmm_decode_step_shared(arr, len(groups), B, _ptr(workspace), ws_bytes, _stream(d, stream)))


def rmm_decode_step(groups, workspace: torch.Tensor | None = None, stream=None):
    """For each group (X [B, K], W [K, N], k, idx [B*k], Y [B, N]): idx = the
    TopK of each token's squared activations, Y = the reduced product; all
    groups in three launches."""
    arr, B = _decode_groups(groups)
    d = groups[0][0].device
    need = int(lib.rmm_decode_step_workspace_size(arr, len(groups), B))
    if workspace is None and need > 0:
        workspace = _scratch(need, d, stream)
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check("rmm_decode_step", lib.rmm_decode_step(arr, len(groups), B, _ptr(workspace), ws_bytes,
                                                  _stream(d, stream)))


# ------------------------------------------- rotation and the paged cache
#
# A decode step makes these calls once per layer on small tensors, so the
# binding reads each tensor's sizes and strides once and builds no objects
# that it does not pass on.

def rope_tables(n_pos: int, rot: int, theta: float = 10000.0, device="cuda"):
    """(cos, sin) float32 [n_pos, rot/2] of the angles pos * theta^(-2i/rot),
    evaluated in float64 (made once at load time)."""
    if rot < 2 or rot % 2 or n_pos < 1:
        raise ValueError("rot must be even and positive, n_pos at least 1")
    f = float(theta) ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot)
    a = torch.arange(n_pos, dtype=torch.float64, device=device)[:, None] * f
    return a.cos().float(), a.sin().float()


class Rope:
    """The position rotation of a model: cos and sin tables (float32 [n_pos,
    rot/2]); pairs (i, i + rot/2), or (2i, 2i + 1) when interleaved."""

    def __init__(self, cos: torch.Tensor, sin: torch.Tensor, interleaved: bool = False):
        if cos.dim() != 2 or cos.shape != sin.shape:
            raise ValueError("cos and sin must be [n_pos, rot/2]")
        if cos.dtype != torch.float32 or sin.dtype != torch.float32:
            raise TypeError("cos and sin must be float32")
        if not (cos.is_contiguous() and sin.is_contiguous()):
            raise ValueError("cos and sin must be contiguous")
        _dev(cos, sin)
        self.cos, self.sin, self.interleaved = cos, sin, bool(interleaved)
        self._c = _ROPE_BYTES.pack(cos.data_ptr(), sin.data_ptr(), cos.shape[0], 2 * cos.shape[1],
                                   int(self.interleaved))


class KvCache:
    """A paged key/value cache over caller-made tensors (pages may be strided,
    each page contiguous): bf16 k, v [n_pages, Hkv, page_size, D]; or MXFP4
    uint8 k, v [n_pages, Hkv, page_size, D/2] with uint8 k_scale, v_scale
    [n_pages, Hkv, page_size, D/32]."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor | None = None,
                 v_scale: torch.Tensor | None = None):
        mx = k.dtype == torch.uint8
        if k.dtype != v.dtype or k.dtype not in (torch.bfloat16, torch.uint8):
            raise TypeError("k and v must both be bfloat16, or both uint8 (MXFP4 codes)")
        if (k_scale is None) != (not mx) or (v_scale is None) != (not mx):
            raise ValueError("an MXFP4 cache takes k_scale and v_scale, a bf16 cache neither")
        if k.dim() != 4 or k.shape != v.shape:
            raise ValueError("k and v must be [n_pages, Hkv, page_size, row]")
        n_pages, Hkv, page_size, row = k.shape
        D = 2 * row if mx else row
        held = (k, v, k_scale, v_scale) if mx else (k, v)
        for t in held[2:]:
            if t.dtype != torch.uint8 or tuple(t.shape) != (n_pages, Hkv, page_size, D // 32):
                raise ValueError("scales must be uint8 [n_pages, Hkv, page_size, D/32]")
        for t in held:
            if t.stride(3) != 1 or t.stride(2) != t.shape[3] or \
                    (Hkv > 1 and t.stride(1) != page_size * t.shape[3]):
                raise ValueError("each page must be contiguous")
        self.device = _dev(*held)
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.n_pages, self.Hkv, self.page_size, self.D, self.mx = n_pages, Hkv, page_size, D, mx
        strides = [t.stride(0) * t.element_size() for t in held] + [0, 0]
        self._c = bytes(_KvCacheC(RMM_CACHE_MX if mx else RMM_CACHE_BF, k.data_ptr(), v.data_ptr(), _ptr(k_scale),
                                  _ptr(v_scale), n_pages, page_size, Hkv, D, *strides[:4]))


def kv_cache(n_pages: int, Hkv: int, page_size: int, D: int, mx: bool = False, device="cuda") -> KvCache:
    """A cache of zeros: bf16, or MXFP4 with mx."""
    if not mx:
        return KvCache(*(torch.zeros(n_pages, Hkv, page_size, D, dtype=torch.bfloat16, device=device)
                         for _ in range(2)))
    return KvCache(*(torch.zeros(n_pages, Hkv, page_size, w, dtype=torch.uint8, device=device)
                     for w in (D // 2, D // 2, D // 32, D // 32)))


def _device_index(*ts) -> int:
    """The one GPU that the given tensors (None: not given) live on."""
    d = -1
    for t in ts:
        if t is not None:
            i = t.get_device()
            if i < 0:
                raise ValueError("librmm tensors must live on the GPU")
            if d < 0:
                d = i
            elif i != d:
                raise ValueError("all tensors must be on one device")
    return d


def _heads(t: torch.Tensor, shape, dtype, name: str, what: str, batched: bool = False, head_first: bool = False):
    """rmm_heads_t of [T, heads, D] (batched: [batch, L, heads, D], or with
    head_first [batch, heads, L, D]), checked; strides of axes of one entry are
    never used."""
    if t.shape != shape:
        raise ValueError(f"{name} must be {what}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}")
    st = t.stride()
    if st[-1] != 1:
        raise ValueError(f"{name} must have contiguous heads")
    if not batched:
        return _HEADS_BYTES.pack(t.data_ptr(), shape[1], 0, st[0] if shape[0] > 1 else 0, st[1] if shape[1] > 1 else 0)
    tok, head = (2, 1) if head_first else (1, 2)
    return _HEADS_BYTES.pack(t.data_ptr(), shape[head], st[0] if shape[0] > 1 else 0, st[tok] if shape[tok] > 1 else 0,
                             st[head] if shape[head] > 1 else 0)


def _vec(t: torch.Tensor | None, n: int, dtype, name: str):
    if t is None:
        return None
    if t.dtype != dtype or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {n} elements")
    return t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda device: torch.cuda.current_stream(device).cuda_stream)


def _run(fn: str, device: int, stream, *args):
    """The call on `device`, on its current stream unless one is given."""
    if stream is None:
        s = _raw_stream(device)
    else:
        s = _stream(torch.device("cuda", device), stream)
    if torch.cuda.current_device() == device:
        status = getattr(lib, fn)(*args, s)
    else:
        with torch.cuda.device(device):
            status = getattr(lib, fn)(*args, s)
    if status != 0:
        raise RmmError(fn, status)



def _positions(rope, positions, T: int):
    if rope is None:
        return None
    if positions is None:
        raise ValueError("a rotation needs positions")
    return _vec(positions, T, torch.int32, "positions")


def rmm_qk_norm_rope_workspace_size(batch: int, H: int, L: int, D: int) -> int:
    return int(lib.rmm_qk_norm_rope_workspace_size(int(batch), int(H), int(L), int(D)))


def rmm_qk_norm_rope(Q: torch.Tensor | None, Qo: torch.Tensor | None, positions: torch.Tensor | None = None,
                     rope: Rope | None = None, K: torch.Tensor | None = None, Ko: torch.Tensor | None = None,
                     gamma_q: torch.Tensor | None = None, gamma_k: torch.Tensor | None = None, eps: float = 1e-6,
                     energy: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                     stream=None) -> torch.Tensor:
    """Per-head RMSNorm (with gamma_q, gamma_k [D]) and position rotation of Q
    [batch, L, H, D] into Qo [batch, H, L, D], and of K [batch, L, Hkv, D] into Ko
    [batch, Hkv, L, D]; any strides with contiguous heads (slices of a
    projection's rows, transposed views); Q and Qo, or K and Ko, may be left out
    (None).  positions: int32 [batch*L].  energy
    (float64 [batch*H*D]) receives the column energies of each head of Qo.
    `workspace` (uint8, rmm_qk_norm_rope_workspace_size(...) bytes) is allocated
    here when energy is wanted and it is not given."""
    if (Q is None) != (Qo is None) or (K is None) != (Ko is None) or (Q is None and K is None) or \
            (Q is not None and Q.dim() != 4) or (K is not None and K.dim() != 4):
        raise ValueError("Q must be [batch, L, H, D] and K [batch, L, Hkv, D]; Q and Qo, K and Ko come together")
    if Q is None and energy is not None:
        raise ValueError("the energies are the queries'")
    x = K if Q is None else Q
    batch, L, H, D = x.shape
    dt = x.dtype
    code = _dtype_code(x)
    q = qo = None
    if Q is not None:
        q = _heads(Q, (batch, L, H, D), dt, "Q", "[batch, L, H, D]", True)
        qo = _heads(Qo, (batch, H, L, D), dt, "Qo", "[batch, H, L, D]", True, True)
    k = ko = None
    if K is not None:
        Hkv = K.shape[2]
        k = _heads(K, (batch, L, Hkv, D), dt, "K", "[batch, L, Hkv, D]", True)
        ko = _heads(Ko, (batch, Hkv, L, D), dt, "Ko", "[batch, Hkv, L, D]", True, True)
    d = _device_index(Q, Qo, K, Ko, gamma_q, gamma_k, None if rope is None else rope.cos, positions, energy, workspace)
    ws_bytes = 0
    if energy is not None:
        if workspace is None:
            workspace = _scratch(rmm_qk_norm_rope_workspace_size(batch, H, L, D), Q.device, stream)
        ws_bytes = workspace.numel() * workspace.element_size()
    _run("rmm_qk_norm_rope", d, stream, code, batch, L, D, q, qo, k, ko, _vec(gamma_q, D, dt, "gamma_q"),
         _vec(gamma_k, D, dt, "gamma_k"), eps, None if rope is None else rope._c,
         _positions(rope, positions, batch * L), _vec(energy, batch * H * D, torch.float64, "energy"),
         _ptr(workspace), ws_bytes)
    return Ko if Q is None else Qo


def rmm_kv_append(K: torch.Tensor, V: torch.Tensor, slots: torch.Tensor, cache: KvCache,
                  positions: torch.Tensor | None = None, rope: Rope | None = None,
                  gamma_k: torch.Tensor | None = None, eps: float = 1e-6, Q: torch.Tensor | None = None,
                  Qo: torch.Tensor | None = None, gamma_q: torch.Tensor | None = None, stream=None) -> KvCache:
    """Appends K and V [T, Hkv, D] (bf16) at the slots (int32 [T]: page *
    page_size + place, all different; outside the cache, e.g. -1: not appended), K normed
    (gamma_k) and rotated (rope, positions int32 [T]) on the way; with Q and Qo
    [T, H, D] the tokens' queries are normed (gamma_q) and rotated in the same
    launch."""
    if (Q is None) != (Qo is None) or K.dim() != 3 or (Q is not None and Q.dim() != 3):
        raise ValueError("K and V must be [T, Hkv, D], Q and Qo (together) [T, H, D]")
    T, D, bf = K.shape[0], cache.D, torch.bfloat16
    q = qo = None
    if Q is not None:
        shape = (T, Q.shape[1], D)
        q, qo = _heads(Q, shape, bf, "Q", "[T, H, D]"), _heads(Qo, shape, bf, "Qo", "[T, H, D]")
    shape = (T, cache.Hkv, D)
    d = _device_index(K, V, slots, cache.k, Q, Qo, gamma_q, gamma_k, None if rope is None else rope.cos, positions)
    _run("rmm_kv_append", d, stream, T, _heads(K, shape, bf, "K", "[T, Hkv, D] of the cache's Hkv and D"),
         _heads(V, shape, bf, "V", "[T, Hkv, D] of the cache's Hkv and D"), _vec(slots, T, torch.int32, "slots"),
         cache._c, _vec(gamma_k, D, bf, "gamma_k"), q, qo, _vec(gamma_q, D, bf, "gamma_q"), eps,
         None if rope is None else rope._c, _positions(rope, positions, T))
    return cache


def rmm_kv_gather(cache: KvCache, slots: torch.Tensor, K: torch.Tensor, V: torch.Tensor, stream=None):
    """Reads the tokens at the slots (int32 [T]) back into bf16 K and V [T, Hkv,
    D] (any strides with contiguous heads; zeros for a slot outside the cache)."""
    T = slots.numel()
    shape = (T, cache.Hkv, cache.D)
    _run("rmm_kv_gather", _device_index(K, V, slots, cache.k), stream, cache._c,
         _vec(slots, T, torch.int32, "slots"), T, _heads(K, shape, torch.bfloat16, "K", "[T, Hkv, D]"),
         _heads(V, shape, torch.bfloat16, "V", "[T, Hkv, D]"))
    return K, V


def rmm_paged_attention_workspace_size(T: int, B: int, H: int, Hkv: int, D: int) -> int:
    return int(lib.rmm_paged_attention_workspace_size(int(T), int(B), int(H), int(Hkv), int(D)))


def rmm_paged_attention(Q: torch.Tensor, cache: KvCache, page_table: torch.Tensor, lengths: torch.Tensor,
                        O: torch.Tensor, q_start: torch.Tensor | None = None, idx: torch.Tensor | None = None,
                        causal: bool = True, scale: float | None = None, workspace: torch.Tensor | None = None,
                        stream=None) -> torch.Tensor:
    """Attention of the new tokens Q [T, H, D] over the cache into O [T, H, D].
    Sequence b holds lengths[b] keys (int32 [B]) in the pages page_table[b]
    (int32 [B, max_pages], rows contiguous) and has the new tokens q_start[b] ..
    q_start[b+1]-1 (int32 [B+1]; None: one each).  Causal: they are its last ones.
    idx (int32 [T, H, k]): the dims each (token, head) keeps.  `workspace`
    (uint8, rmm_paged_attention_workspace_size(...) bytes, 256-byte aligned; the
    size is not monotonous: for several T and B the largest of theirs) is allocated
    here when not given."""
    if Q.dim() != 3:
        raise ValueError("Q must be [T, H, D]")
    T, H, _ = Q.shape
    D, bf = cache.D, torch.bfloat16
    B = lengths.numel()
    width = page_table.shape[-1]
    if page_table.dtype != torch.int32 or tuple(page_table.shape) != (B, width) or page_table.stride(1) != 1:
        raise ValueError("page_table must be int32 [B, max_pages] with contiguous rows")
    k = 0
    if idx is not None:
        n = idx.numel()
        if idx.dtype != torch.int32 or not idx.is_contiguous() or n == 0 or n % (T * H):
            raise ValueError("idx must be contiguous int32 [T, H, k]")
        k = n // (T * H)
    if scale is None:
        scale = D ** -0.5
    d = _device_index(Q, O, cache.k, page_table, lengths, q_start, idx, workspace)
    if workspace is None:
        workspace = _scratch(rmm_paged_attention_workspace_size(T, B, H, cache.Hkv, D), Q.device, stream)
    ws_bytes = workspace.numel() * workspace.element_size()
    _run("rmm_paged_attention", d, stream, T, _heads(Q, (T, H, D), bf, "Q", "[T, H, D] of the cache's D"), cache._c,
         page_table.data_ptr(), page_table.stride(0) if B > 1 else width, width,
         _vec(lengths, B, torch.int32, "lengths"), B, _vec(q_start, B + 1, torch.int32, "q_start"), _ptr(idx), k,
         float(scale), 1 if causal else 0, _heads(O, (T, H, D), bf, "O", "[T, H, D]"), workspace.data_ptr(), ws_bytes)
    return O
