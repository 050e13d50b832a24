"""Timed cases of what stands between a layer's reduced products and after the
last one: the product with bias, activation and residual in its epilogue; the
join of a block's output with the residual stream (norms before and after, gate,
residual scale); and the log probabilities of given tokens, with the
distribution's entropy and its most likely tokens.

A case is a dict of plain values.  ``prepare`` builds on the GPU what a program
holds before the call, ``run`` makes one pass, ``exact`` evaluates the same
formulas in float64 and ``work`` counts the bytes and operations no
implementation can do without.  With ``own`` false ``run`` computes the plain
form out of elementary torch operations; with ``own`` true it calls this
package.

  product   Y = act(X[:, I] W[I, :] + bias) + s R
  join      H = s R + gate * (Y or norm(Y) gamma_post);  X = norm(H) gamma_pre
            norm(v) = v / sqrt(mean(v^2) + eps), of the stored H
  logprobs  log softmax(scale z)[token];  entropy of softmax(scale z);  the
            tokens of the largest z (ties to the lower index) with theirs

Values follow the repository's synthetic recipe: activations N(0, 1) with 1 %
of the channels scaled by 20, weights N(0, 0.02^2); logits are N(0, 2^2) with a
heavy-tailed offset per token of the vocabulary.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


# ----------------------------------------------------------------- cases

def listed():
    return [
        # one decoding token through the down projection onto its residual: latency
        dict(name="product_token", kind="product", path="few", dtype="bf16", B=1, M=1, N=4096, K=14336, r=0.5, act="none",
             bias=False, residual=True, scale=1.0),
        # five drafted tokens for each of three sequences, biased q|k|v, a set per sequence
        dict(name="product_draft", kind="product", path="few", dtype="bf16", B=3, M=5, N=6144, K=4096, r=0.5, act="silu",
             bias=True, residual=False, scale=1.0),
        # a prompt through the down projection onto its residual
        dict(name="product_prompt", kind="product", path="kmajor", dtype="bf16", B=1, M=8192, N=4096, K=14336, r=0.5,
             act="none", bias=False, residual=True, scale=1.0),
        # two prompts of odd length, an odd width, everything in the epilogue
        dict(name="product_odd", kind="product", path="kmajor", dtype="bf16", B=2, M=1001, N=4097, K=1000, r=0.61, act="gelu",
             bias=True, residual=True, scale=0.5),
        # a small fp32 layer from row-major activations
        dict(name="product_f32", kind="product", path="rows", dtype="f32", B=1, M=517, N=771, K=1024, r=0.5, act="gelu_tanh",
             bias=True, residual=True, scale=1.0),
        # one decode step of four sequences: latency
        dict(name="join_token", kind="join", out="rows", dtype="bf16", stream="bf16", B=4, M=1, K=4096, post=False, gate="none",
             scale=1.0),
        # a prompt, norms before and after, feeding a reduced projection
        dict(name="join_prompt", kind="join", out="kmajor", dtype="bf16", stream="bf16", B=1, M=8192, K=4096, post=True,
             gate="none", scale=1.0),
        # two sequences with gates of their own on an fp32 stream, 70B width
        dict(name="join_gated", kind="join", out="kmajor", dtype="bf16", stream="f32", B=2, M=1001, K=8192, post=True,
             gate="unit", scale=0.7),
        # fp32, an odd width, a gate per channel
        dict(name="join_f32", kind="join", out="rows", dtype="f32", stream="f32", B=3, M=333, K=1367, post=True, gate="channel",
             scale=1.0),
        # one decoded token's alternatives: latency
        dict(name="logprobs_token", kind="logprobs", dtype="bf16", T=1, V=128000, top=5, given=1, entropy=True, masked=0.0,
             scale=1.0),
        # a decode step of a batch in fp32, odd vocabulary in padded rows, constrained decoding at a temperature
        dict(name="logprobs_batch", kind="logprobs", dtype="f32", T=48, V=50003, top=20, given=4, entropy=True, masked=0.5,
             scale=1.25),
        # a prompt scored
        dict(name="logprobs_prompt", kind="logprobs", dtype="bf16", T=2048, V=128000, top=5, given=1, entropy=True, masked=0.0,
             scale=1.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_WIDTHS = (1024, 2048, 4096, 4096, 5120, 6144, 8192, 14336)


def draw(rng):
    kind = rng.choice(("product", "product", "join", "logprobs"))
    while True:
        if kind == "product":
            path = rng.choice(("few", "kmajor", "kmajor", "rows"))
            c = dict(kind="product", path=path, dtype="f32" if path == "rows" and rng.random() < 0.7 else "bf16",
                     B=rng.choice((1, 1, 2, 5, 16)), M=rng.randint(1, 8) if path == "few" else _log(rng, 9, 8192),
                     N=rng.choice(_WIDTHS) if rng.random() < 0.5 else _log(rng, 64, 20000),
                     K=rng.choice(_WIDTHS) if rng.random() < 0.6 else _log(rng, 64, 16000), r=rng.choice((1.0, 0.8, 0.5, 0.5, 0.25)),
                     act=rng.choice(("none", "relu", "silu", "gelu", "gelu_tanh")), bias=rng.random() < 0.6,
                     residual=rng.random() < 0.6, scale=rng.choice((1.0, 1.0, 0.5, 1.7)))
            most = 2 ** 28 if path == "few" else 8192 * 4096 * 7168 // (16 if path == "rows" else 1)
            k = math.ceil(c["r"] * c["K"])
            if c["B"] * c["M"] * c["N"] * k <= most and c["B"] * c["M"] * c["K"] <= 2 ** 28 and c["B"] * c["N"] * k <= 2 ** 31:
                return c
        elif kind == "join":
            out = rng.choice(("rows", "kmajor"))
            dtype, stream = rng.choice((("bf16", "bf16"), ("bf16", "f32")) + (() if out == "kmajor" else (("f32", "f32"),)))
            K = rng.choice(_WIDTHS) if rng.random() < 0.5 else _log(rng, 48, 16384)
            c = dict(kind="join", out=out, dtype=dtype, stream=stream, B=rng.choice((1, 1, 2, 5)), M=_log(rng, 1, 8192),
                     K=(K + 7) // 8 * 8 if out == "kmajor" else K, post=rng.random() < 0.5,
                     gate=rng.choice(("none", "none", "channel", "unit", "token")), scale=rng.choice((1.0, 1.0, 0.7)))
            if c["B"] * c["M"] * c["K"] * (2 if stream == "f32" else 1) <= 8192 * 4096:
                return c
        else:
            c = dict(kind="logprobs", dtype=rng.choice(("bf16", "f32")), T=_log(rng, 1, 4096), V=_log(rng, 500, 260000),
                     top=rng.choice((0, 1, 5, 20, 64)), given=rng.choice((0, 1, 1, 4)), entropy=rng.random() < 0.7,
                     masked=rng.choice((0.0, 0.0, 0.5, 0.99)), scale=rng.choice((1.0, 1.0, 1.25, 0.6)))
            if c["T"] * c["V"] * (2 if c["dtype"] == "f32" else 1) <= 2048 * 128000 and c["top"] + c["given"] > 0:
                return c


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _randn(g, *shape):
    return torch.randn(*shape, device=DEV, generator=g)


def _acts(g, *shape):
    """Rows of activations, 1 % of the channels large."""
    x = _randn(g, *shape)
    x[..., torch.randperm(shape[-1], device=DEV, generator=g)[:max(1, shape[-1] // 100)]] *= 20.0
    return x


def _up(n, m):
    return (n + m - 1) // m * m


def prepare(case, seed):
    c, g = case, _gen(seed)
    s = dict(case=c)
    dt = _DT[c["dtype"]]
    if c["kind"] == "product":
        B, M, N, K = c["B"], c["M"], c["N"], c["K"]
        k = max(1, math.ceil(c["r"] * K - 1e-9 * K))
        x = _acts(g, B, M, K).to(dt)
        s["idx"] = x.double().square().sum(1).topk(k, dim=1).indices.sort(dim=1).values.int().contiguous()
        if c["path"] == "kmajor":
            s["Xt"] = torch.zeros(B, K, _up(M, 8), dtype=dt, device=DEV)[:, :, :M]
            s["Xt"].copy_(x.transpose(1, 2))
        else:
            s["X"] = x
        s["W"] = torch.zeros(K, _up(N, 8), dtype=dt, device=DEV)[:, :N]
        s["W"].copy_(0.02 * _randn(g, K, N))
        s["bias"] = (0.2 * _randn(g, N)).to(dt) if c["bias"] else None
        s["R"] = _acts(g, B, M, N).to(dt) if c["residual"] else None
        s["Y"] = torch.empty(B, M, N, dtype=dt, device=DEV)
        if own and c["path"] == "few":
            import paper_2608_13426_amd as rmm
            s["ws"] = torch.empty(max(1, rmm.rmm_gemv_workspace_size(B, M, N, k)), dtype=torch.uint8, device=DEV)
        return s
    if c["kind"] == "join":
        B, M, K = c["B"], c["M"], c["K"]
        s["Y"] = _acts(g, B, M, K).to(dt)
        s["R"] = (3.0 * _acts(g, B, M, K)).to(_DT[c["stream"]])
        s["post"] = (1 + 0.1 * _randn(g, K)).to(dt) if c["post"] else None
        s["pre"] = (1 + 0.1 * _randn(g, K)).to(dt)
        shape = {"channel": (K,), "unit": (B, 1, K), "token": (B, M, K)}.get(c["gate"])
        s["gate"] = (0.5 + 0.3 * _randn(g, *shape)).to(dt) if shape else None
        s["H"] = torch.empty_like(s["R"])
        if c["out"] == "kmajor":
            s["Xt"] = torch.zeros(B, K, _up(M, 8), dtype=dt, device=DEV)[:, :, :M]
            s["e"] = torch.empty(B * K, dtype=torch.float64, device=DEV)
        else:
            s["X"] = torch.empty(B, M, K, dtype=dt, device=DEV)
        if own:
            import paper_2608_13426_amd as rmm
            s["ws"] = torch.empty(max(1, rmm.rmm_block_join_workspace_size(B, M, K)), dtype=torch.uint8, device=DEV)
        return s
    T, V = c["T"], c["V"]
    offset = 1.5 * _randn(g, V) / (0.2 + _randn(g, V).abs())
    z = torch.zeros(T, _up(V, 8), dtype=dt, device=DEV)[:, :V]
    for t0 in range(0, T, 512):                              # in pieces: the temporaries are large
        z[t0:t0 + 512] = 2.0 * _randn(g, min(512, T - t0), V) + offset.clamp(-8, 8)
    if c["masked"]:
        barred = torch.rand(V, device=DEV, generator=g) < c["masked"]
        barred[V // 2] = False
        z[:, barred] = -math.inf
    s["z"] = z
    s["tokens"] = torch.randint(0, V, (T, c["given"]), device=DEV, generator=g, dtype=torch.int32)
    s["tokens"][::3, :1] = z[::3].argmax(1, keepdim=True).int()[:, :c["given"]]
    if T > 1:
        s["tokens"][-1:, -1:] = -1                           # a padded place
    f = dict(dtype=torch.float32, device=DEV)
    s["logp"] = torch.empty(T, c["given"], **f) if c["given"] else None
    s["entropy"] = torch.empty(T, **f) if c["entropy"] else None
    s["top_idx"] = torch.empty(T, c["top"], dtype=torch.int32, device=DEV) if c["top"] else None
    s["top_logp"] = torch.empty(T, c["top"], **f) if c["top"] else None
    if own:
        import paper_2608_13426_amd as rmm
        s["ws"] = torch.empty(max(1, rmm.rmm_token_logprobs_workspace_size(T, V, c["top"])), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------ plain form

_EPS = 1e-6
_EPS32 = float(torch.tensor(_EPS, dtype=torch.float32))


def _act(x, name):
    if name == "relu":
        return torch.where(x < 0, 0 * x, x)
    if name == "silu":
        return x / (1 + (-x).exp())
    if name == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    if name == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))
    return x


def _plain_product(s):
    c = s["case"]
    idx = s["idx"].long()
    if c["path"] == "kmajor":
        x = s["Xt"].gather(1, idx[:, :, None].expand(-1, -1, c["M"])).float().transpose(1, 2)
    else:
        x = s["X"].gather(2, idx[:, None, :].expand(-1, c["M"], -1)).float()
    y = torch.matmul(x, s["W"][idx].float())
    if c["bias"]:
        y = y + s["bias"].float()
    y = _act(y, c["act"])
    if c["residual"]:
        y = y + c["scale"] * s["R"].float()
    return {"Y": y.to(s["Y"].dtype)}


def _inv_rms(x):
    """1 / sqrt(mean square + eps) of rows, the sum in float64 and rounded once."""
    return (1 / (x.double().square().sum(-1, keepdim=True) / x.shape[-1] + _EPS32).sqrt()).float()


def _plain_join(s):
    c = s["case"]
    y = s["Y"].float()
    if c["post"]:
        y = y * _inv_rms(y) * s["post"].float()
    if c["gate"] != "none":
        y = y * s["gate"].float()
    h = (s["R"].float() * c["scale"] + y).to(s["R"].dtype)
    x = h.float()
    x = (x * _inv_rms(x) * s["pre"].float()).to(s["Y"].dtype)
    if c["out"] == "rows":
        return {"H": h, "X": x}
    return {"H": h, "Xt": x.transpose(1, 2).contiguous(), "e": x.double().square().sum(1).flatten()}


def _plain_logprobs(s):
    c, z = s["case"], s["z"]
    x = z.float() * c["scale"]
    m = x.amax(1, keepdim=True)
    e = (x - m).exp()
    total = e.double().sum(1, keepdim=True)
    lse = m.double() + total.log()
    out = {}
    if c["given"]:
        t = s["tokens"].long()
        lp = x.gather(1, t.clamp_min(0)).double() - lse
        out["logp"] = torch.where(t < 0, torch.zeros_like(lp), lp).float()
    if c["entropy"]:
        d = torch.where(e > 0, (x - m) * e, torch.zeros_like(e))
        out["entropy"] = (total.log() - d.double().sum(1, keepdim=True) / total).flatten().float()
    if c["top"]:
        # whole numbers in the order of the logits, the lower index first among equal ones
        b = (z.float() + 0.0).view(torch.int32)
        key = torch.where(b < 0, b ^ 0x7FFFFFFF, b).long() * 2 ** 32 + (2 ** 31 - torch.arange(c["V"], device=DEV))
        at = key.topk(c["top"], dim=1).indices
        out["top_idx"] = at.int()
        out["top_logp"] = (x.gather(1, at).double() - lse).float()
    return out


# ------------------------------------------------------------------ run

def run(s):
    c = s["case"]
    if not own:
        return {"product": _plain_product, "join": _plain_join, "logprobs": _plain_logprobs}[c["kind"]](s)
    import paper_2608_13426_amd as rmm
    if c["kind"] == "product":
        ep = dict(bias=s["bias"], act=c["act"], residual=s["R"], residual_scale=c["scale"])
        if c["path"] == "kmajor":
            rmm.rmm_reduced_gemm_kmajor_epilogue(s["Xt"], s["W"], s["idx"], s["Y"], **ep)
        elif c["path"] == "few":
            rmm.rmm_reduced_gemv_epilogue(s["X"], s["W"], s["idx"], s["Y"], workspace=s["ws"], **ep)
        else:
            rmm.rmm_reduced_gemm_epilogue(s["X"], s["W"], s["idx"], s["Y"], **ep)
        return {"Y": s["Y"]}
    if c["kind"] == "join":
        ends = dict(Xt=s["Xt"], energy=s["e"]) if c["out"] == "kmajor" else dict(X=s["X"])
        rmm.rmm_block_join(s["Y"], s["R"], s["H"], post_norm=c["post"], post_gamma=s["post"], gate=s["gate"],
                           residual_scale=c["scale"], pre_gamma=s["pre"], eps=_EPS, workspace=s["ws"], **ends)
        return {"H": s["H"], **({"Xt": s["Xt"], "e": s["e"]} if c["out"] == "kmajor" else {"X": s["X"]})}
    rmm.rmm_token_logprobs(s["z"], tokens=s["tokens"] if c["given"] else None, logp=s["logp"], entropy=s["entropy"],
                           top_idx=s["top_idx"], top_logp=s["top_logp"], scale=c["scale"], workspace=s["ws"])
    return {n: s[n] for n in ("logp", "entropy", "top_idx", "top_logp") if s[n] is not None}


# ----------------------------------------------------------------- exact

def _act64(x, name):
    if name == "relu":
        return x.clamp_min(0)
    if name == "silu":
        return x * torch.sigmoid(x)
    if name in ("gelu", "gelu_tanh"):
        return torch.nn.functional.gelu(x, approximate="tanh" if name == "gelu_tanh" else "none")
    return x


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "product":
        Y = []
        for b in range(c["B"]):
            i = s["idx"][b].long()
            x = s["Xt"][b, i].double().t() if c["path"] == "kmajor" else s["X"][b][:, i].double()
            y = x @ s["W"][i].double()
            if c["bias"]:
                y += s["bias"].double()
            y = _act64(y, c["act"])
            Y.append(y + c["scale"] * s["R"][b].double() if c["residual"] else y)
        return {"Y": torch.stack(Y)}
    if c["kind"] == "join":
        y = s["Y"].double()
        if c["post"]:
            y = y * torch.rsqrt(y.pow(2).mean(-1, keepdim=True) + _EPS32) * s["post"].double()
        h = c["scale"] * s["R"].double() + (y if c["gate"] == "none" else y * s["gate"].double())
        x = h if c["stream"] == "f32" else h.to(s["R"].dtype).double()      # the norm is of the stored stream
        x = x * torch.rsqrt(x.pow(2).mean(-1, keepdim=True) + _EPS32) * s["pre"].double()
        return {"H": h, "X": x} if c["out"] == "rows" else {"H": h, "Xt": x.transpose(1, 2), "e": None}   # of rounded values
    out = {n: [] for n in ("logp", "entropy", "top_idx", "top_logp") if s[n] is not None}
    for t0 in range(0, c["T"], 256):
        z = s["z"][t0:t0 + 256].double()
        lp = torch.log_softmax(z * c["scale"], 1)
        if c["given"]:
            t = s["tokens"][t0:t0 + 256].long()
            out["logp"].append(lp.gather(1, t % c["V"]).masked_fill(t < 0, 0.0))
        if c["entropy"]:
            out["entropy"].append(torch.special.entr(lp.exp()).sum(1))
        if c["top"]:
            at = z.sort(dim=1, descending=True, stable=True).indices[:, :c["top"]]
            out["top_idx"].append(at.int())
            out["top_logp"].append(lp.gather(1, at))
    return {n: torch.cat(v) for n, v in out.items()}


# ------------------------------------------------------------------ work

def work(case):
    c = case
    if c["kind"] == "product":
        size, out = (2 if c["dtype"] == "bf16" else 4), c["B"] * c["M"] * c["N"]
        k = max(1, math.ceil(c["r"] * c["K"] - 1e-9 * c["K"]))
        # at least one set's rows of W: the sets of several units may coincide
        return {"bytes": size * (c["B"] * c["M"] * k + k * c["N"] + out * (2 if c["residual"] else 1)) + 4 * c["B"] * k,
                "flops": 2 * out * k}
    if c["kind"] == "join":
        n = c["B"] * c["M"] * c["K"]
        size, stream = (2 if c["dtype"] == "bf16" else 4), (2 if c["stream"] == "bf16" else 4)
        gate = {"none": 0, "channel": c["K"], "unit": c["B"] * c["K"], "token": n}[c["gate"]]
        return {"bytes": n * (2 * size + 2 * stream) + gate * size + (8 * c["B"] * c["K"] if c["out"] == "kmajor" else 0),
                "flops": n * (6 + (4 if c["post"] else 0) + (2 if c["out"] == "kmajor" else 0))}
    n = c["T"] * c["V"]
    return {"bytes": n * (2 if c["dtype"] == "bf16" else 4) + c["T"] * (8 * c["given"] + 4 * c["entropy"] + 8 * c["top"]),
            "flops": n * (4 + (2 if c["entropy"] else 0))}
