"""Binding of what stands between a layer's reduced products and after the last
one: products with an epilogue, the join with the residual stream, token log
probabilities.  A decode step makes these calls once per layer on small tensors,
so each tensor's sizes and strides are read once and no objects built that are not
passed on."""
from __future__ import annotations

import ctypes
import struct
import sys

import torch

from . import RMM_BF16, RMM_F32, _device_index, _dtype_code, _i64, _p, _ptr, _rows, _run, _scratch, _vec, \
    rmm_gemv_workspace_size

_rmm = sys.modules[__package__]


class _EpilogueC(ctypes.Structure):
    """rmm_epilogue_t"""
    _fields_ = [("bias", _p), ("act", ctypes.c_int), ("residual_scale", ctypes.c_float), ("residual", _p), ("ldr", _i64)]


class _JoinC(ctypes.Structure):
    """rmm_join_t"""
    _fields_ = [("dtype", ctypes.c_int), ("stream_dtype", ctypes.c_int), ("B", _i64), ("M", _i64), ("K", _i64),
                ("Y", _p), ("ldy", _i64), ("R", _p), ("ldr", _i64), ("residual_scale", ctypes.c_float),
                ("post_norm", ctypes.c_int), ("post_gamma", _p), ("gate", _p), ("gate_unit_stride", _i64),
                ("gate_row_stride", _i64), ("pre_gamma", _p), ("eps", ctypes.c_float), ("H", _p), ("ldh", _i64),
                ("X", _p), ("ldx", _i64), ("Xt", _p), ("ldxt", _i64), ("energy", _p)]


# only read by the library: each is packed into bytes
_EPILOGUE_BYTES, _JOIN_BYTES = struct.Struct("@PifPq"), struct.Struct("@iiqqqPqPqfiPPqqPf4xPqPqPqP")
assert _EPILOGUE_BYTES.size == ctypes.sizeof(_EpilogueC) and _JOIN_BYTES.size == ctypes.sizeof(_JoinC)

_CODES = {torch.bfloat16: RMM_BF16, torch.float32: RMM_F32}
_ACTS = {None: 0, "none": 0, "relu": 1, "silu": 2, "gelu": 3, "gelu_tanh": 4}


def _unit_rows(t: torch.Tensor, shape, dtype, name: str) -> int:
    """The row stride of t, [B, M, N] (or [M, N] of one unit) of `dtype`: rows
    contiguous, units packed (M rows apart); strides of axes of one entry are
    never used."""
    if t.dtype is dtype and t.shape == shape and t.is_contiguous():
        return shape[2]
    B, M, N = shape
    if tuple(t.shape) != (B, M, N) and (B > 1 or tuple(t.shape) != (M, N)):
        raise ValueError(f"{name} must be [{B}, {M}, {N}]")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}")
    st = t.stride()
    if N > 1 and st[-1] != 1:
        raise ValueError(f"{name} rows must be contiguous")
    if M > 1:
        ld = st[-2]
        if B > 1 and st[0] != M * ld:
            raise ValueError(f"{name} units must be packed (stride M*ld)")
        return ld
    return st[0] if B > 1 else N


def _epilogue(Y: torch.Tensor, shape, bias, act, residual, residual_scale: float) -> bytes:
    if act not in _ACTS:
        raise ValueError(f"act must be one of {sorted(a for a in _ACTS if a)}")
    ldr = 0 if residual is None else _unit_rows(residual, shape, Y.dtype, "residual")
    return _EPILOGUE_BYTES.pack(_vec(bias, shape[2], Y.dtype, "bias") or 0, _ACTS[act], residual_scale,
                                _ptr(residual) or 0, ldr)


def _weights(W: torch.Tensor, K: int, dtype):
    if W.dim() != 2 or W.shape[0] != K or (W.shape[1] > 1 and W.stride(1) != 1):
        raise ValueError("W must be [K, N] with contiguous rows")
    if W.dtype != dtype:
        raise TypeError(f"W must be {dtype}")
    return W.shape[1], W.stride(0) if K > 1 else W.shape[1]


def _lists(idx: torch.Tensor, B: int) -> int:
    n = idx.numel()
    if idx.dtype != torch.int32 or not idx.is_contiguous() or n == 0 or n % B:
        raise ValueError("idx must be contiguous int32 [B, k]")
    return n // B


def rmm_reduced_gemm_epilogue(X: torch.Tensor, W: torch.Tensor, idx: torch.Tensor, Y: torch.Tensor,
                              bias: torch.Tensor | None = None, act: str | None = None,
                              residual: torch.Tensor | None = None, residual_scale: float = 1.0,
                              stream=None) -> torch.Tensor:
    """Y[b] = act(X[b][:, I_b] @ W[I_b, :] + bias) + residual_scale * residual[b] for
    X [B, M, K], W [K, N], idx [B, k], Y [B, M, N] (bf16 or fp32), evaluated in fp32
    and rounded once.  act: None, "relu", "silu", "gelu" or "gelu_tanh"; bias [N];
    residual [B, M, N], which may be Y."""
    B, M, K, ldx = _rows(X, "X")
    N, ldw = _weights(W, K, X.dtype)
    ldy = _unit_rows(Y, (B, M, N), X.dtype, "Y")
    d = _device_index(X, W, idx, Y, bias, residual)
    _run("rmm_reduced_gemm_epilogue", d, stream, X.data_ptr(), W.data_ptr(), idx.data_ptr(), _dtype_code(X), B, M, N, K,
         _lists(idx, B), ldx, ldw, Y.data_ptr(), ldy,
         _epilogue(Y, (B, M, N), bias, act, residual, residual_scale))
    return Y


def rmm_reduced_gemm_kmajor_epilogue(Xt: torch.Tensor, W: torch.Tensor, idx: torch.Tensor, Y: torch.Tensor,
                                     bias: torch.Tensor | None = None, act: str | None = None,
                                     residual: torch.Tensor | None = None, residual_scale: float = 1.0,
                                     stream=None) -> torch.Tensor:
    """rmm_reduced_gemm_epilogue from the K-major copy Xt [B, K, M] (bf16)."""
    B, K, M, ldxt = _rows(Xt, "Xt")
    N, ldw = _weights(W, K, torch.bfloat16)
    ldy = _unit_rows(Y, (B, M, N), torch.bfloat16, "Y")
    if Xt.dtype != torch.bfloat16:
        raise TypeError("Xt must be bfloat16")
    d = _device_index(Xt, W, idx, Y, bias, residual)
    _run("rmm_reduced_gemm_kmajor_epilogue", d, stream, Xt.data_ptr(), W.data_ptr(), idx.data_ptr(), B, M, N, K,
         _lists(idx, B), ldxt, ldw, Y.data_ptr(), ldy,
         _epilogue(Y, (B, M, N), bias, act, residual, residual_scale))
    return Y


def rmm_reduced_gemv_epilogue(X: torch.Tensor, W: torch.Tensor, idx: torch.Tensor, Y: torch.Tensor,
                              bias: torch.Tensor | None = None, act: str | None = None,
                              residual: torch.Tensor | None = None, residual_scale: float = 1.0,
                              workspace: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """The decode-step form of rmm_reduced_gemm_epilogue (M <= 8 rows per unit,
    bf16); `workspace` (uint8, rmm_gemv_workspace_size(B, M, N, k) bytes) is
    allocated here when not given."""
    B, M, K, ldx = _rows(X, "X")
    N, ldw = _weights(W, K, torch.bfloat16)
    ldy = _unit_rows(Y, (B, M, N), torch.bfloat16, "Y")
    if X.dtype != torch.bfloat16:
        raise TypeError("X must be bfloat16")
    k = _lists(idx, B)
    d = _device_index(X, W, idx, Y, bias, residual, workspace)
    if workspace is None:
        workspace = _scratch(rmm_gemv_workspace_size(B, M, N, k), X.device, stream)
    _run("rmm_reduced_gemv_epilogue", d, stream, X.data_ptr(), W.data_ptr(), idx.data_ptr(), B, M, N, K, k, ldx, ldw,
         Y.data_ptr(), ldy, _epilogue(Y, (B, M, N), bias, act, residual, residual_scale), workspace.data_ptr(),
         workspace.nbytes)
    return Y


def rmm_block_join_workspace_size(B: int, M: int, K: int) -> int:
    return int(_rmm.lib.rmm_block_join_workspace_size(int(B), int(M), int(K)))


def rmm_block_join(Y: torch.Tensor | None, R: torch.Tensor | None, H: torch.Tensor | None = None,
                   X: torch.Tensor | None = None, Xt: torch.Tensor | None = None, energy: torch.Tensor | None = None,
                   post_norm: bool = False, post_gamma: torch.Tensor | None = None, gate: torch.Tensor | None = None,
                   residual_scale: float = 1.0, pre_gamma: torch.Tensor | None = None, eps: float = 1e-6,
                   workspace: torch.Tensor | None = None, stream=None):
    """A block's output Y [B, M, K] (or [M, K]) joined to the residual stream R:
    y = norm(Y) * post_gamma with post_norm, else Y; H = residual_scale * R + gate * y,
    stored in the stream's type (bf16 or fp32); X = norm(H) * pre_gamma, or with Xt
    [B, K, M] and energy (float64 [B*K]) its K-major copy and column energies (bf16;
    needs H; fastest where Xt's rows lie a multiple of 64 elements apart).  gate: [K], or
    three-dimensional and broadcastable to [B, M, K], with contiguous rows of K; gammas [K]
    or None (ones).  Y or R may be None, and outputs that are not wanted.
    H may be R, X may be Y.  `workspace` (uint8, rmm_block_join_workspace_size(B, M, K)
    bytes, 256-byte aligned) is allocated here when Xt is wanted and it is not given.
    Returns H, X and Xt, those that were given."""
    some = Y if Y is not None else R
    if some is None or some.dim() not in (2, 3):
        raise ValueError("Y or R must be given, as [B, M, K] or [M, K]")
    shape = some.shape if some.dim() == 3 else (1, *some.shape)
    B, M, K = shape
    if B * M * K == 0:
        raise ValueError("Y and R must not be empty")
    sd = R.dtype if R is not None else H.dtype if H is not None else Y.dtype
    dt = Y.dtype if Y is not None else X.dtype if X is not None else torch.bfloat16 if Xt is not None else sd
    if dt not in _CODES or sd not in _CODES:
        raise TypeError("rows must be bfloat16 or float32")
    ldy = ldr = ldh = ldx = py = pr = ph = px = 0
    if Y is not None:
        ldy, py = _unit_rows(Y, shape, dt, "Y"), Y.data_ptr()
    if R is not None:
        ldr, pr = _unit_rows(R, shape, sd, "R"), R.data_ptr()
    if H is not None:
        ldh, ph = _unit_rows(H, shape, sd, "H"), H.data_ptr()
    if X is not None:
        ldx, px = _unit_rows(X, shape, dt, "X"), X.data_ptr()
    gu = gr = 0
    if gate is not None:
        if gate.dtype != dt:
            raise TypeError(f"gate must be {dt}")
        if gate.dim() not in (1, 3) or gate.shape[-1] != K or (K > 1 and gate.stride(-1) != 1) or \
                (gate.dim() == 3 and (gate.shape[0] not in (1, B) or gate.shape[1] not in (1, M))):
            raise ValueError("gate must be [K], or three-dimensional and broadcastable to [B, M, K], with contiguous rows")
        if gate.dim() == 3:
            gu = gate.stride(0) if gate.shape[0] > 1 else 0
            gr = gate.stride(1) if gate.shape[1] > 1 else 0
    ldxt, ws_bytes = 0, 0
    d = _device_index(Y, R, H, X, Xt, energy, post_gamma, gate, pre_gamma, workspace)
    if Xt is not None:
        ldxt = _unit_rows(Xt, (B, K, M), torch.bfloat16, "Xt")
        if workspace is None:
            workspace = _scratch(rmm_block_join_workspace_size(B, M, K), some.device, stream)
        ws_bytes = workspace.nbytes
    _run("rmm_block_join", d, stream,
         _JOIN_BYTES.pack(_CODES[dt], _CODES[sd], B, M, K, py, ldy, pr, ldr, residual_scale, 1 if post_norm else 0,
                          _vec(post_gamma, K, dt, "post_gamma") or 0, 0 if gate is None else gate.data_ptr(), gu, gr,
                          _vec(pre_gamma, K, dt, "pre_gamma") or 0, eps, ph, ldh, px, ldx,
                          0 if Xt is None else Xt.data_ptr(), ldxt, _vec(energy, B * K, torch.float64, "energy") or 0),
         _ptr(workspace), ws_bytes)
    return tuple(t for t in (H, X, Xt) if t is not None)


def _flat(t: torch.Tensor | None, dtype, name: str):
    """The address of a contiguous tensor whose shape has been checked."""
    if t is None:
        return None
    if t.dtype is not dtype or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor")
    return t.data_ptr()


def rmm_token_logprobs_workspace_size(T: int, V: int, top: int) -> int:
    return int(_rmm.lib.rmm_token_logprobs_workspace_size(int(T), int(V), int(top)))


def rmm_token_logprobs(logits: torch.Tensor, tokens: torch.Tensor | None = None, logp: torch.Tensor | None = None,
                       entropy: torch.Tensor | None = None, top_idx: torch.Tensor | None = None,
                       top_logp: torch.Tensor | None = None, scale: float = 1.0,
                       workspace: torch.Tensor | None = None, stream=None) -> None:
    """One pass over logits [T, V] (bf16 or fp32, rows contiguous): logp (float32) =
    the log probabilities of tokens (int32, both [T, given] or [T]; -1: 0) under
    softmax(scale * logits), entropy (float32 [T]) of that distribution, top_idx
    (int32) and top_logp (float32, both [T, top], top <= 64) its most likely tokens,
    ties to the lower one.  What is not given is not computed.  `workspace`
    (uint8, rmm_token_logprobs_workspace_size(T, V, top) bytes) is allocated here when
    not given."""
    if logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits must be [T, V] with contiguous rows")
    T, V = logits.shape
    if (tokens is None) != (logp is None) or (top_idx is None) != (top_logp is None):
        raise ValueError("tokens and logp, top_idx and top_logp come together")
    given = top = 0
    if tokens is not None:
        size = tokens.shape
        if len(size) not in (1, 2) or size[0] != T or logp.shape != size:
            raise ValueError("tokens and logp must be [T] or [T, given]")
        given = size[1] if len(size) == 2 else 1
    if top_idx is not None:
        size = top_idx.shape
        if len(size) != 2 or size[0] != T or top_logp.shape != size:
            raise ValueError("top_idx and top_logp must be [T, top]")
        top = size[1]
    d = _device_index(logits, tokens, logp, entropy, top_idx, top_logp, workspace)
    if workspace is None:
        workspace = _scratch(rmm_token_logprobs_workspace_size(T, V, top), logits.device, stream)
    i32, f32 = torch.int32, torch.float32
    _run("rmm_token_logprobs", d, stream, logits.data_ptr(), _dtype_code(logits), T, V,
         logits.stride(0) if T > 1 else V, scale, _flat(tokens, i32, "tokens"), given, _flat(logp, f32, "logp"),
         _vec(entropy, T, f32, "entropy"), top, _flat(top_idx, i32, "top_idx"), _flat(top_logp, f32, "top_logp"),
         workspace.data_ptr(), workspace.nbytes)
