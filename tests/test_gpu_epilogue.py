"""Products with bias, activation and residual in their epilogue against float64."""
import math

import pytest
import torch

import paper_2608_13426_amd as rmm
from tests import block_ref as ref
from tests.gpu_util import gpu, require_gpu

pytestmark = gpu
BF, F32 = torch.bfloat16, torch.float32


def make(dev, dt, B, M, N, K, k, seed=0, bias=True, residual=True, pad=0):
    g = torch.Generator(device=dev).manual_seed(seed)
    X = torch.randn(B, M, K, device=dev, generator=g)
    X[..., torch.randperm(K, device=dev, generator=g)[:max(1, K // 100)]] *= 20
    W = torch.zeros(K, (N + 7) // 8 * 8 + 8 * pad, dtype=dt, device=dev)[:, :N]
    W.copy_(0.1 * torch.randn(K, N, device=dev, generator=g))
    idx = torch.rand(B, K, device=dev, generator=g).topk(k, dim=1).indices.sort(dim=1).values.int().contiguous()
    b = torch.randn(N, device=dev, generator=g).to(dt) if bias else None
    R = (2 * torch.randn(B, M, N, device=dev, generator=g)).to(dt) if residual else None
    return X.to(dt), W, idx, b, R


def call(form, X, W, idx, Y, **kw):
    if form == "kmajor":
        B, M, K = X.shape
        Xt = torch.zeros(B, K, (M + 7) // 8 * 8, dtype=X.dtype, device=X.device)[:, :, :M]
        Xt.copy_(X.transpose(1, 2))
        return rmm.rmm_reduced_gemm_kmajor_epilogue(Xt, W, idx, Y, **kw)
    return (rmm.rmm_reduced_gemv_epilogue if form == "few" else rmm.rmm_reduced_gemm_epilogue)(X, W, idx, Y, **kw)


def check(Y, want):
    y, tol = want
    err = (Y.double() - y).abs()
    assert bool((err <= tol).all()), f"worst {float((err / tol).max())} of the bound"


# tiles of 64, 128, 256, 256 x 128; rows and columns that end inside a tile; one of each
KMAJOR = [(1, 9, 64, 40, 7), (2, 65, 100, 72, 72), (1, 1, 1, 8, 1), (3, 130, 257, 64, 33), (1, 700, 1000, 128, 90),
          (1, 1025, 2051, 96, 61), (1, 2048, 4096, 64, 33), (2, 1500, 2500, 32, 32), (40, 4200, 120, 40, 20)]


@pytest.mark.parametrize("B,M,N,K,k", KMAJOR)
@pytest.mark.parametrize("act", [None, "gelu"])
def test_kmajor(B, M, N, K, k, act):
    dev = require_gpu()
    X, W, idx, b, R = make(dev, BF, B, M, N, K, k)
    Y = torch.empty(B, M, N, dtype=BF, device=dev)
    call("kmajor", X, W, idx, Y, bias=b, act=act, residual=R, residual_scale=0.5)
    check(Y, ref.product(X, W, idx, b, act, R, 0.5, BF))


@pytest.mark.parametrize("B,M,N,K,k", [(1, 1, 4096, 512, 256), (2, 3, 1000, 700, 351), (5, 8, 77, 64, 64), (1, 5, 1, 9, 4),
                                       (16, 1, 640, 2048, 1024), (1, 2, 513, 40, 13),
                                       (3, 5, 6144, 600, 301), (1, 6, 520, 3000, 2999), (2, 7, 1032, 33, 33)])
@pytest.mark.parametrize("act", [None, "silu"])
def test_few_rows(B, M, N, K, k, act):
    dev = require_gpu()
    X, W, idx, b, R = make(dev, BF, B, M, N, K, k, seed=1)
    Y = torch.empty(B, M, N, dtype=BF, device=dev)
    call("few", X, W, idx, Y, bias=b, act=act, residual=R, residual_scale=-1.5)
    check(Y, ref.product(X, W, idx, b, act, R, -1.5, BF))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("B,M,N,K,k", [(1, 37, 131, 100, 51), (2, 300, 513, 64, 64), (3, 1, 5, 7, 3), (1, 600, 2100, 200, 17),
                                       (1, 4000, 4000, 64, 40), (2, 3000, 2100, 96, 70)])
def test_row_major(dt, B, M, N, K, k):
    dev = require_gpu()
    X, W, idx, b, R = make(dev, dt, B, M, N, K, k, seed=2)
    Y = torch.empty(B, M, N, dtype=dt, device=dev)
    call("rows", X, W, idx, Y, bias=b, act="gelu_tanh", residual=R)
    check(Y, ref.product(X, W, idx, b, "gelu_tanh", R, 1.0, dt))


SHAPES = {"kmajor": (BF, 2, 130, 256, 64, 40), "few": (BF, 2, 4, 256, 64, 40), "rows": (F32, 2, 40, 64, 48, 20)}


@pytest.mark.parametrize("form", list(SHAPES))
@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("bias,residual", [(True, True), (True, False), (False, True), (False, False)])
def test_parts(form, act, bias, residual):
    dev = require_gpu()
    dt, B, M, N, K, k = SHAPES[form]
    X, W, idx, b, R = make(dev, dt, B, M, N, K, k, seed=3, bias=bias, residual=residual)
    Y = torch.empty(B, M, N, dtype=dt, device=dev)
    call(form, X, W, idx, Y, bias=b, act=act, residual=R, residual_scale=2.0)
    check(Y, ref.product(X, W, idx, b, act, R, 2.0, dt))


@pytest.mark.parametrize("form,M,N", [("kmajor", 300, 520), ("kmajor", 2100, 4096), ("kmajor", 90, 61), ("few", 5, 520),
                                      ("rows", 50, 77)])
def test_residual_in_place(form, M, N):
    """Y is the residual stream itself; its neighbours' rows stay as they were."""
    dev = require_gpu()
    B, K, k = 2, 64, 30
    X, W, idx, b, R = make(dev, BF, B, M, N, K, k, seed=4)
    held = torch.full((B, M, N + 8), 7.0, dtype=BF, device=dev)
    Y = held[:, :, :N]
    Y.copy_(R)
    call(form, X, W, idx, Y, bias=b, residual=Y, residual_scale=1.0)
    check(Y, ref.product(X, W, idx, b, None, R, 1.0, BF))
    assert bool((held[:, :, N:] == 7.0).all())


@pytest.mark.parametrize("form", ["kmajor", "few", "rows"])
def test_alignments(form):
    """Bias, residual and output at every offset of two bytes, odd strides."""
    dev = require_gpu()
    B, M, N, K, k = 1, (8 if form == "few" else 200), 200, 40, 21
    X, W, idx, b, R = make(dev, BF, B, M, N, K, k, seed=5)
    want = ref.product(X, W, idx, b, "relu", R, 1.0, BF)
    for off, ld in ((1, 201), (2, 202), (3, 205), (4, 204), (0, 208)):
        mem = torch.zeros(3, M * ld + 16, dtype=BF, device=dev)
        Y, Ro = (m[off:off + M * ld].view(M, ld)[:, :N] for m in mem[:2])
        bo = mem[2, off:off + N]
        Ro.copy_(R[0])
        bo.copy_(b)
        call(form, X, W, idx, Y, bias=bo, act="relu", residual=Ro)
        check(Y[None], want)


@pytest.mark.parametrize("form", list(SHAPES))
def test_nothing_asked_for_is_the_plain_product(form):
    dev = require_gpu()
    dt, B, M, N, K, k = SHAPES[form]
    X, W, idx, _, _ = make(dev, dt, B, M, N, K, k, seed=6)
    Y, Z = (torch.empty(B, M, N, dtype=dt, device=dev) for _ in range(2))
    call(form, X, W, idx, Y)
    if form == "kmajor":
        rmm.rmm_reduced_gemm_kmajor(X.transpose(1, 2).contiguous()[:, :, :M] if M % 8 == 0 else
                                    torch.nn.functional.pad(X.transpose(1, 2), (0, -M % 8))[:, :, :M], W, idx, Z)
    else:
        (rmm.rmm_reduced_gemv if form == "few" else rmm.rmm_reduced_gemm)(X, W, idx, Z)
    if form == "few":                        # another order of the sums
        check(Y, ref.product(X, W, idx, None, None, None, 1.0, dt))
    else:
        assert torch.equal(Y, Z)


@pytest.mark.parametrize("form", list(SHAPES))
def test_nonfinite(form):
    """An infinite or NaN bias or residual reaches its own outputs alone."""
    dev = require_gpu()
    dt, B, M, N, K, k = SHAPES[form]
    X, W, idx, b, R = make(dev, dt, B, M, N, K, k, seed=7)
    b[3], b[5], R[1, 2, 9], R[0, 0, 0] = math.inf, math.nan, math.nan, -math.inf
    Y = torch.empty(B, M, N, dtype=dt, device=dev)
    call(form, X, W, idx, Y, bias=b, act="gelu", residual=R)
    bad = torch.zeros(B, M, N, dtype=torch.bool, device=dev)
    bad[:, :, 3], bad[:, :, 5], bad[1, 2, 9], bad[0, 0, 0] = True, True, True, True
    assert torch.equal(~Y.isfinite(), bad)
    assert bool((Y[:, :, 3] == math.inf).all()) and bool(Y[:, :, 5].isnan().all()) and float(Y[0, 0, 0]) == -math.inf


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh", "relu"])
@pytest.mark.parametrize("form", ["kmajor", "few", "rows"])
def test_activation_over_its_range(form, act):
    """Arguments from far negative to far positive, as biases of an empty product."""
    dev = require_gpu()
    dt = F32 if form == "rows" else BF
    b = torch.cat([torch.linspace(-20, 20, 4000), torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1e4, -1e4, 3e37, -3e37]),
                   torch.logspace(-8, 2, 92)]).to(dev).to(dt)
    X, W = torch.zeros(1, 8, 8, dtype=dt, device=dev), torch.zeros(8, b.numel() + 4, dtype=dt, device=dev)[:, :b.numel()]
    idx = torch.arange(8, dtype=torch.int32, device=dev)
    Y = torch.empty(1, 8, b.numel(), dtype=dt, device=dev)
    call(form, X, W, idx, Y, bias=b, act=act)
    y, tol = ref.product(X, W, idx, b, act, None, 1.0, dt)
    assert bool(Y.isfinite().all())
    check(Y, (y, tol))


@pytest.mark.parametrize("form", ["kmajor", "rows"])
def test_past_32_bit_offsets(form):
    """The last rows of an output and a residual of more than 2^31 elements."""
    dev = require_gpu()
    M, N, K, k = 40000, 56000, 16, 8
    X, W, idx, b, _ = make(dev, BF, 1, M, N, K, k, seed=9, residual=False)
    Y = torch.empty(1, M, N, dtype=BF, device=dev)
    R = torch.ones(1, M, N, dtype=BF, device=dev)
    R[:, -300:].normal_()
    call(form, X, W, idx, Y, bias=b, act="relu", residual=R)
    for rows in (slice(0, 200), slice(M - 300, M)):
        check(Y[:, rows], ref.product(X[:, rows], W, idx, b, "relu", R[:, rows], 1.0, BF))


@pytest.mark.parametrize("form,dt,B,M,N,k", [("kmajor", BF, 1, 700, 1000, 50), ("kmajor", BF, 2, 90, 61, 30), ("kmajor", BF, 40, 4200, 120, 40),
                                             ("kmajor", BF, 1, 2100, 4096, 50), ("rows", BF, 1, 2048, 4096, 50), ("rows", BF, 2, 130, 77, 50),
                                             ("rows", F32, 2, 130, 256, 50), ("rows", F32, 1, 130, 77, 50), ("rows", F32, 1, 1100, 1028, 50),
                                             ("few", BF, 2, 1, 1024, 50), ("few", BF, 2, 1, 1001, 900), ("few", BF, 2, 5, 1024, 50),
                                             ("few", BF, 1, 8, 1001, 900), ("few", BF, 1, 3, 1024, 900)])
@pytest.mark.parametrize("act", [None, "silu"])
def test_in_place_is_the_same_bits(form, dt, B, M, N, k, act):
    """A residual that is Y gives what it gives elsewhere, in every kernel."""
    dev = require_gpu()
    X, W, idx, b, R = make(dev, dt, B, M, N, 1000, k, seed=10)
    Y = torch.empty(B, M, N, dtype=dt, device=dev)
    kw = dict(bias=b, act=act, residual_scale=0.75)
    call(form, X, W, idx, Y, residual=R, **kw)
    Z = R.clone()
    call(form, X, W, idx, Z, residual=Z, **kw)
    assert torch.equal(Y, Z)


def tail_bound(x, act, out):
    """(y, bound) of an activation alone, relative to its value: on the far negative side
    that is what keeps a wrong or missing tail from passing.

    silu: rounding the exponent's argument moves e^-x by 2 u32 |x| (argument and
    constant), exponential, sum, reciprocal and product add 8 u32.  gelu_tanh: its
    argument w of 2^w is off by up to 4 roundings, 3 u32 |w| of the value.  bf16 gelu:
    a Phi(-a) from the polynomial, off by 1.9e-5 as given and by up to 1e-5 through its
    rounding to fp32 (largest last steps: 2^-18 + 10 * 2^-22 + 100 * 2^-25 of a log2), 5e-5
    in all; past |x| = 10 it stays below 1e-22.  Where 2^126 is passed a reciprocal is 0: |y| < 2e-36."""
    x = x.double()
    if act == "silu":
        y = x * torch.sigmoid(x)
        e = (2 * x.abs() + 8) * ref.U32 * y.abs()
    elif act == "gelu_tanh":
        u = math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3)
        y = x * torch.sigmoid(2 * u)
        e = (3 * 2 * u.abs() / math.log(2) + 8) * ref.U32 * y.abs()
    else:
        y = 0.5 * x * torch.erfc(-x * math.sqrt(0.5))
        e = 5e-5 * 0.5 * x.abs() * torch.erfc(x.abs() * math.sqrt(0.5)) + 2 * ref.U32 * y.clamp_min(0) + 1e-22 * (x.abs() > 10)
    return y, e + ref.U[out] * (y.abs() + e) + 2e-36


# fp32 gelu, 1 + erf, is exact to the argument's size only (test_activation_over_its_range)
TAILS = [(*f, act) for f in (("kmajor", BF, 8, 8), ("rows", BF, 8, 8), ("few", BF, 1, 8), ("few", BF, 1, 2048), ("few", BF, 5, 8),
                             ("few", BF, 5, 2048), ("rows", F32, 8, 8)) for act in ("silu", "gelu", "gelu_tanh") if (f[1], act) != (F32, "gelu")]


@pytest.mark.parametrize("form,dt,M,K,act", TAILS)
def test_activation_tails(form, dt, M, K, act):
    """Far negative arguments, as biases of an empty product: each output is as exact as its own size."""
    dev = require_gpu()
    b = torch.cat([torch.linspace(-20, 20, 4000), torch.linspace(-7, 0, 3000), torch.tensor([-30.0, -50.0, -80.0, -1e3, 1e3])]).to(dev).to(dt)
    N = b.numel()
    X, W = torch.zeros(1, M, K, dtype=dt, device=dev), torch.zeros(K, (N + 7) // 8 * 8, dtype=dt, device=dev)[:, :N]
    idx = torch.arange(K, dtype=torch.int32, device=dev)
    Y = torch.empty(1, M, N, dtype=dt, device=dev)
    call(form, X, W, idx, Y, bias=b, act=act)
    y, tol = tail_bound(b, act, dt)
    err = (Y.double() - y).abs() / tol
    assert float(err.max()) <= 1, (float(err.max()), float(b[int(err.amax((0, 1)).argmax())]))


@pytest.mark.parametrize("B,M,N,K,k", [(2, 1001, 4097, 1000, 610), (1, 3000, 3000, 600, 300), (40, 4200, 120, 200, 100), (1, 100, 100, 4096, 2048),
                                       (1, 2048, 4096, 600, 50)])
@pytest.mark.parametrize("form,dt", [("kmajor", BF), ("rows", BF), ("rows", F32)])
def test_without_an_epilogue_the_plain_bits_whatever_the_tiles(form, dt, B, M, N, K, k):
    """The tile rules differ (prompts of an odd width); the order of a sum does not."""
    dev = require_gpu()
    X, W, idx, _, _ = make(dev, dt, B, M, N, K, k, seed=12, bias=False, residual=False)
    Y, Z = (torch.empty(B, M, N, dtype=dt, device=dev) for _ in range(2))
    call(form, X, W, idx, Y)
    if form == "kmajor":
        Xt = torch.zeros(B, K, (M + 7) // 8 * 8, dtype=dt, device=dev)[:, :, :M]
        rmm.rmm_reduced_gemm_kmajor(Xt.copy_(X.transpose(1, 2)), W, idx, Z)
    else:
        rmm.rmm_reduced_gemm(X, W, idx, Z)
    assert torch.equal(Y, Z)
