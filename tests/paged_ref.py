"""Attention of query rows over a key/value history in float64, with how far the
kernels' arithmetic may move it: for the tests of long sequences, where a limit on
the scale of the values would not notice a lost or doubled run of keys.

With w the exact weights of a row, the kernels use w_s (1 + t_s): t_s holds the weight's
rounding to bf16 (at most U16) and the fp32 error `eps` of its score and exponential.
  sum of the rounded weights:    O' - O = sum w_s t_s (V_s - O) / sum w_s (1 + t_s)
  sum of the unrounded weights:  the same, times a factor within U16 of 1
  fp32 sums: `steps` additions one after the other, each within U32 of sum w |V|
  the output's rounding:         U16 |O|
`limit` bounds this for every element, by |sum w t (V - O)| <= t sqrt(sum w (V - O)^2).
`rms` is the size of a row's error over its dims, all of these being independent from key
to key: a rounding to bf16 has a variance of at most U16^2 / 3, so sum w t (V - O) has one
of (U16^2 / 3 + eps^2) sum w^2 (V - O)^2, and L additions have L U32^2 sum w V^2.  Four
times that size is allowed (a sum of few weights' roundings is the same in all dims)."""
from __future__ import annotations

import torch

from tests.gpu_util import U16, U32


def attend(q, K, V, see, scale, unrounded, keep=None):
    """(O, limit [R, D], rms [R]) of query rows q [R, D] over K, V [L, D], row r over its
    first see[r] keys; keep [R, D]: the dims that its scores use.  All float64, one device."""
    R, D = q.shape
    L = K.shape[0]
    q = q if keep is None else torch.where(keep, q, 0.0)
    gone = torch.arange(L, device=q.device)[None, :] >= see[:, None]
    s = (scale * (q @ K.T)).masked_fill(gone, -float("inf"))
    none = see <= 0
    s[none] = 0.0
    w = torch.softmax(s, -1)
    w[none] = 0.0
    most = (q.abs() @ K.abs().T).masked_fill(gone, 0.0).amax(-1, keepdim=True) * abs(scale)
    O, VV = w @ V, w @ V.square()
    spread = (VV - O.square()).clamp_min(0)                    # sum w (V - O)^2
    w2 = w.square()
    var = (w2 @ V.square() - 2 * O * (w2 @ V) + O.square() * w2.sum(-1, keepdim=True)).clamp_min(0)
    eps = ((D + 4) * most + 4 * (most + 64) + 4) * U32
    t = 1.01 * (U16 + eps)
    sums = (L / 32 + 128) * U32 * VV.sqrt()
    limit = t / (1 - t) * spread.sqrt() + (t * O.abs() if unrounded else 0) + sums + 1.01 * U16 * O.abs()
    third = U16 * U16 / 3
    random = (third + eps * eps) * var + third * O.square() * (1 + (w2.sum(-1, keepdim=True) if unrounded else 0))
    rms = 4 * (random + L * U32 * U32 * VV).mean(-1).sqrt()
    return O, limit, rms


def check(got, O, limit, rms, what=""):
    """got [R, D]: every element within its limit, every row within its rms."""
    err = got - O
    assert bool(torch.isfinite(got).all()), what
    over = (err.abs() - limit).max().item()
    assert over <= 0, f"{what}: an element is {over:.3g} past its limit"
    size = err.square().mean(-1).sqrt()
    r = int((size - rms).argmax())
    assert size[r] <= rms[r], f"{what}: row {r} is off by {size[r]:.3g} (rms), {rms[r]:.3g} allowed"


def accepts(got, O, limit, rms):
    try:
        check(got, O, limit, rms)
    except AssertionError:
        return False
    return True
