"""float64 definitions of the rotation, the 4-bit format and the attention over a
paged cache, for the tests of those entry points (numpy, CPU)."""
from __future__ import annotations

import math

import numpy as np
import torch

from tests.gpu_util import U16, U32

EPS = 1e-6
GRID = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])


def bf16(x):
    """float64 array of x rounded to bf16."""
    return torch.from_numpy(np.asarray(x, dtype=np.float64)).to(torch.bfloat16).double().numpy()


def np64(t):
    return t.detach().double().cpu().numpy()


def rotate(x, gamma, pos, cos, sin, interleaved):
    """x [T, heads, D] float64 -> (normed and rotated, error bound before the
    output's rounding).  An fp32 value passes r, x r, gamma, and in a pair one
    product and one sum: at most 5 roundings of a result bounded by |u c| + |w s|
    (one more for the second-order terms)."""
    y = np.array(x, dtype=np.float64)
    if gamma is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + float(np.float32(EPS))) * gamma
    mag = np.abs(y)
    if cos is not None:
        h = cos.shape[1]
        c, s = cos[pos][:, None, :], sin[pos][:, None, :]
        a = (slice(0, 2 * h, 2), slice(1, 2 * h, 2)) if interleaved else (slice(0, h), slice(h, 2 * h))
        u, w = y[..., a[0]].copy(), y[..., a[1]].copy()
        y[..., a[0]], y[..., a[1]] = u * c - w * s, w * c + u * s
        mag[..., a[0]] = np.abs(u * c) + np.abs(w * s)
        mag[..., a[1]] = np.abs(w * c) + np.abs(u * s)
    return y, 6 * U32 * mag


def rotate_f32(x, gamma, pos, cos, sin, interleaved):
    """The same in fp32 with each product and sum rounded by itself."""
    f = np.float32
    y = np.array(x, dtype=f)
    if gamma is not None:
        y64 = y.astype(np.float64)
        r = (1 / np.sqrt((y64 * y64).sum(-1, keepdims=True) / y.shape[-1] + float(f(EPS)))).astype(f)
        y = (y * r) * gamma.astype(f)
    if cos is not None:
        h = cos.shape[1]
        c, s = cos[pos][:, None, :].astype(f), sin[pos][:, None, :].astype(f)
        a = (slice(0, 2 * h, 2), slice(1, 2 * h, 2)) if interleaved else (slice(0, h), slice(h, 2 * h))
        u, w = y[..., a[0]].copy(), y[..., a[1]].copy()
        y[..., a[0]], y[..., a[1]] = u * c - w * s, w * c + u * s
    assert y.dtype == f
    return y


def mx_round(x):
    """Values of x [..., D] after the 4-bit format: per 32 the smallest scale 2^e,
    e in -119 .. 125, at which the largest magnitude rounds to at most 6, then
    the nearest code (ties to the even one); NaN groups where x is not finite."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(*x.shape[:-1], -1, 32)
    out = np.empty_like(g)
    for i in np.ndindex(g.shape[:-1]):
        v = g[i]
        top = np.abs(v).max()
        if not np.isfinite(top):
            out[i] = np.nan
            continue
        e = -119
        if top > 0:
            e = min(max(math.frexp(top)[1] - 4, -119), 125)
            while top * 2.0 ** -e >= 7 and e < 125:
                e += 1
            while e > -119 and top * 2.0 ** (1 - e) < 7:
                e -= 1
        y = np.abs(v) * 2.0 ** -e
        d = np.abs(y[:, None] - GRID[None, :])
        near = d.min(1)
        code = np.array([min((c for c in range(8) if d[j, c] == near[j]), key=lambda c: c & 1) for j in range(32)])
        out[i] = np.copysign(GRID[code], v) * 2.0 ** e
    return out.reshape(x.shape)


def mx_values(codes, scales):
    """uint8 codes [..., D/2] and scale bytes [..., D/32] -> float64 values."""
    q = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])
    v = GRID[q & 7] * np.where(q & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (v.reshape(*scales.shape, 32) * s[..., None]).reshape(v.shape)


def history(cache, table, b, length):
    """Sequence b's (K, V) [Hkv, length, D] float64 out of a KvCache."""
    pages = table[b, :-(-length // cache.page_size)].long()
    out = []
    for t, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        x = t[pages].cpu()
        x = mx_values(x.numpy(), s[pages].cpu().numpy()) if cache.mx else np64(x)
        out.append(x.transpose(1, 0, 2, 3).reshape(cache.Hkv, len(pages) * cache.page_size, cache.D)[:, :length])
    return out


def attend(Q, K, V, n, scale, causal, idx=None):
    """(O, bound) [n, H, D] of one sequence's new tokens Q [n, H, D] over K, V
    [Hkv, L, D].  Bound: each weight carries its bf16 rounding (2^-9) and the fp32
    error of its score, (D + 4) u32 |scale| sum |q||k|, twice (numerator and sum);
    the output moves by at most 2 d max |V|, d the largest relative move of a weight, and
    is rounded to bf16."""
    _, H, D = Q.shape
    Hkv, L, _ = K.shape
    O, bound = np.zeros(Q.shape), np.zeros(Q.shape)
    for j in range(n):
        see = max(L - n + j + 1, 0) if causal else L
        if see == 0:
            continue
        for h in range(H):
            g = h // (H // Hkv)
            I = np.arange(D) if idx is None else idx[j, h]
            q, k, v = Q[j, h, I], K[g, :see][:, I], V[g, :see]
            with np.errstate(invalid="ignore", over="ignore"):
                s = scale * (k @ q)
                w = np.exp(s - s.max())
                w /= w.sum()
                O[j, h] = w @ v
                d = np.expm1(2.0 ** -9 + 2 * (D + 4) * U32 * abs(scale) * (np.abs(k) @ np.abs(q)).max())
                bound[j, h] = 2 * d * np.abs(v).max() + U16 * np.abs(O[j, h])
    return O, bound
