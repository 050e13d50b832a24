"""float64 forms of the products with an epilogue, the join and the token log
probabilities, with bounds on what the kernels' arithmetic may differ by."""
import math

import torch

U32, U = 2.0 ** -24, {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def act64(x, name):
    if name == "relu":
        return x.clamp_min(0)
    if name == "silu":
        return x * torch.sigmoid(x)
    if name == "gelu":
        return 0.5 * x * torch.erfc(-x * math.sqrt(0.5))
    if name == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)))
    return x


def product(X, W, idx, bias, act, R, rs, out):
    """(Y, bound): X [B, M, K] rows.  fp32 sums of k exact products err by k u32
    sum|x w|, the bias adds one rounding of the sum; an activation passes errors on
    with a slope of at most 1.13 and its evaluation errs by at most 16 u32 |x|
    (2^-16 |x| where the output is bf16); the scaled residual adds two
    roundings, the output one."""
    Y, tol = [], []
    for b in range(X.shape[0]):
        i = idx.view(X.shape[0], -1)[b].long()
        x, w = X[b][:, i].double(), W[i].double()
        k = i.numel()
        s = x @ w
        mag = x.abs() @ w.abs()
        if bias is not None:
            s = s + bias.double()
        e = k * U32 * mag + U32 * s.abs()
        y = act64(s, act)
        if act not in (None, "none", "relu"):
            e = 1.13 * e + (16 * U32 if out == torch.float32 else 2.0 ** -16) * s.abs()
        if R is not None:
            y = y + rs * R[b].double()
            e = e + 2 * U32 * (abs(rs) * R[b].double().abs() + y.abs())
        Y.append(y)
        tol.append(U[out] * y.abs() + e * (1 + U[out]) + 1e-38)
    return torch.stack(Y), torch.stack(tol)


def inv_rms(x, eps):
    return 1 / (x.square().mean(-1, keepdim=True) + float(torch.tensor(eps, dtype=torch.float32))).sqrt()


def join(Y, R, post, gpost, gate, rs, eps, sd):
    """(H, bound) of the stream: r, its product, the gain, the gate, the scaled
    residual and the sum are rounded to fp32 once each, H to its type."""
    y = None
    if Y is not None:
        y = Y.double()
        if post:
            y = y * inv_rms(y, eps)
            if gpost is not None:
                y = y * gpost.double()
        if gate is not None:
            y = y * gate.double()
    rs = float(torch.tensor(rs, dtype=torch.float32))
    r = None if R is None else rs * R.double()
    h = y if r is None else r if y is None else y + r
    mag = sum(t.abs() for t in (y, r) if t is not None)
    return h, U[sd] * h.abs() + 6 * U32 * mag * (1 + U[sd]) + 1e-38


def normed(H, gpre, eps, dt):
    """(X, bound) from the stored H: r, its product and the gain, then the output's rounding."""
    x = H.double() * inv_rms(H.double(), eps)
    if gpre is not None:
        x = x * gpre.double()
    return x, (U[dt] + 4 * U32) * x.abs() + 1e-38


def order(z):
    """Whole numbers in the ranking order of logits: NaN above +inf, -0 equal to +0."""
    b = (z.float() + 0.0).view(torch.int32).long()
    k = torch.where(b < 0, b ^ 0x7FFFFFFF, b)
    return torch.where(z.isnan(), torch.full_like(k, 2 ** 32), k)


def top_tokens(z, n):
    return order(z).neg().sort(dim=1, stable=True).indices[:, :n]


def logprobs(z, scale):
    """(log p, entropy, bound on log p, bound on entropy), float64.

    With t = (z - b) scale log2 e: two roundings of t and one of the scale move a
    weight by 3 u32 |t| (and a few u32 of exp2), and so does each of up to 10 moves of b.  A lane's fp32 sum of up to V/256 + 8 terms errs by that many u32.
    The sum's relative error moves every log p, the scale's rounding log p by 2 u32 |t|;
    entropy moves by twice that of the weights times itself, and by t's own errors."""
    x = z.double() * float(torch.tensor(scale, dtype=torch.float32))
    lp = torch.log_softmax(x, 1)
    p = lp.exp()
    ent = -(torch.where(p > 0, p * lp, torch.zeros_like(p))).sum(1)
    t = (x.amax(1, keepdim=True) - x).clamp_max(1e30) * 1.4427
    mean_t = torch.where(p > 0, p * t, torch.zeros_like(p)).sum(1, keepdim=True) + 10
    rel = (3 * mean_t + z.shape[1] / 256 + 16) * U32
    return lp, ent, rel + 2 * U32 * (t + lp.abs()), (2 * rel * (ent[:, None] + mean_t * U32 + 1)).flatten() + 4 * U32 * mean_t.flatten()
