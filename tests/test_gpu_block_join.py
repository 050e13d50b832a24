"""The join of a block's output with the residual stream against float64."""
import math

import numpy as np
import pytest
import torch

import paper_2608_13426_amd as rmm
from tests import block_ref as ref
from tests.gpu_util import check_energies, gpu, require_gpu

pytestmark = gpu
BF, F32 = torch.bfloat16, torch.float32
EPS = 1e-6


def make(dev, dt, sd, B, M, K, gate="none", seed=0):
    g = torch.Generator(device=dev).manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, device=dev, generator=g)  # noqa: E731
    Y, R = rnd(B, M, K).to(dt), (3 * rnd(B, M, K)).to(sd)
    gp, gq = ((1 + 0.1 * rnd(K)).to(dt) for _ in range(2))
    shape = {"channel": (K,), "unit": (B, 1, K), "row": (1, M, K), "token": (B, M, K)}.get(gate)
    return Y, R, gp, gq, None if shape is None else rnd(*shape).to(dt)


def kmajor(dev, B, M, K, fill=0.0):
    held = torch.full((B, K, (M + 7) // 8 * 8), fill, dtype=BF, device=dev)
    return held, held[:, :, :M], torch.full((B * K,), math.nan, dtype=torch.float64, device=dev)


def check_h(H, Y, R, post, gpost, gate, rs, sd):
    h, tol = ref.join(Y, R, post, gpost, gate, rs, EPS, sd)
    err = (H.double() - h).abs()
    assert bool((err <= tol).all()), f"H: {float((err / tol).max())} of the bound"


def check_x(X, H, gpre, dt):
    x, tol = ref.normed(H, gpre, EPS, dt)
    err = (X.double() - x).abs()
    assert bool((err <= tol).all()), f"X: {float((err / tol).max())} of the bound"


TYPES = [(BF, BF), (BF, F32), (F32, F32)]


@pytest.mark.parametrize("dt,sd", TYPES)
@pytest.mark.parametrize("B,M,K", [(1, 1, 1), (1, 3, 7), (2, 5, 64), (1, 4, 2048), (1, 3, 2056), (1, 2, 2049), (3, 1, 4096),
                                   (1, 2, 5000), (1, 2, 8192), (1, 2, 8193), (1, 1, 16384), (1, 1, 16392), (1, 1, 65536),
                                   (2, 300, 200), (1, 1000, 4096)])
@pytest.mark.parametrize("post", [False, True])
def test_rows(dt, sd, B, M, K, post):
    dev = require_gpu()
    Y, R, gp, gq, _ = make(dev, dt, sd, B, M, K)
    H, X = torch.empty_like(R), torch.empty_like(Y)
    rmm.rmm_block_join(Y, R, H, X=X, post_norm=post, post_gamma=gp, pre_gamma=gq, residual_scale=0.7, eps=EPS)
    check_h(H, Y, R, post, gp, None, 0.7, sd)
    check_x(X, H, gq, dt)


@pytest.mark.parametrize("sd", [BF, F32])
@pytest.mark.parametrize("B,M,K", [(1, 1, 8), (1, 7, 64), (2, 64, 72), (3, 65, 264), (1, 129, 4096), (2, 1001, 1024), (1, 33, 4104),
                                   (1, 9, 8192), (1, 31, 16384), (1, 3000, 512), (5, 513, 128), (1, 2, 65536),
                                   (1, 4100, 1024), (2, 2100, 2056), (1, 4096, 4096), (3, 1500, 520)])
@pytest.mark.parametrize("gate", ["none", "unit"])
def test_kmajor(sd, B, M, K, gate):
    """The K-major outputs are the row-major ones, bit for bit, and their energies."""
    dev = require_gpu()
    Y, R, gp, gq, gt = make(dev, BF, sd, B, M, K, gate, seed=1)
    H, X, Hx = torch.empty_like(R), torch.empty_like(Y), torch.empty_like(R)
    held, Xt, e = kmajor(dev, B, M, K, 5.0)
    kw = dict(post_norm=True, post_gamma=gp, gate=gt, pre_gamma=gq, residual_scale=1.0, eps=EPS)
    rmm.rmm_block_join(Y, R, H, Xt=Xt, energy=e, **kw)
    rmm.rmm_block_join(Y, R, Hx, X=X, **kw)
    check_h(H, Y, R, True, gp, gt, 1.0, sd)
    check_x(Xt.transpose(1, 2), H, gq, BF)
    assert torch.equal(H, Hx) and torch.equal(Xt.transpose(1, 2), X)
    assert bool((held[:, :, M:] == 5.0).all())
    check_energies(e.cpu().numpy(), X.double().square().sum(1).flatten().cpu().numpy(), M + 1)


@pytest.mark.parametrize("gate", ["channel", "unit", "row", "token"])
@pytest.mark.parametrize("dt,sd", TYPES)
@pytest.mark.parametrize("K", [96, 101])
def test_gates(gate, dt, sd, K):
    dev = require_gpu()
    Y, R, gp, gq, gt = make(dev, dt, sd, 3, 5, K, gate, seed=2)
    H, X = torch.empty_like(R), torch.empty_like(Y)
    rmm.rmm_block_join(Y, R, H, X=X, gate=gt, pre_gamma=gq, eps=EPS)
    check_h(H, Y, R, False, None, gt, 1.0, sd)
    check_x(X, H, gq, dt)
    if gate == "token":                                  # a broadcast view, and strided rows
        rmm.rmm_block_join(Y, R, H, X=X, gate=gt[:, :1].expand(3, 5, K), pre_gamma=gq, eps=EPS)
        check_h(H, Y, R, False, None, gt[:, :1], 1.0, sd)


@pytest.mark.parametrize("K", [64, 2049])
def test_parts(K):
    """Each input and output left out in turn; gains of one."""
    dev = require_gpu()
    Y, R, gp, gq, _ = make(dev, BF, BF, 2, 9, K, seed=3)
    H, X = torch.empty_like(R), torch.empty_like(Y)
    rmm.rmm_block_join(None, R, X=X, pre_gamma=gq, eps=EPS)                    # a plain norm of the stream
    check_x(X, R, gq, BF)
    rmm.rmm_block_join(Y, None, H, post_norm=True, post_gamma=gp, eps=EPS)      # a plain norm of the block
    check_h(H, Y, None, True, gp, None, 1.0, BF)
    rmm.rmm_block_join(Y, R, H)
    check_h(H, Y, R, False, None, None, 1.0, BF)
    rmm.rmm_block_join(Y, R, H, X=X, post_norm=True, eps=EPS)
    check_h(H, Y, R, True, None, None, 1.0, BF)
    check_x(X, H, None, BF)
    X2 = torch.empty_like(X)
    rmm.rmm_block_join(Y, R, X=X2, post_norm=True, eps=EPS)                     # the norm is of the stored stream
    assert torch.equal(X, X2)
    if K % 8 == 0:
        _, Xt, e = kmajor(dev, 2, 9, K)
        rmm.rmm_block_join(Y, R, H, Xt=Xt, energy=e, post_norm=True, eps=EPS)
        assert torch.equal(Xt.transpose(1, 2), X)


@pytest.mark.parametrize("parts", ["all", "no Y", "no R", "no gains", "in place", "strided", "channel gate", "eps 0"])
def test_many_rows(parts):
    """Inputs left out in turn at many rows, against the row-major outputs."""
    dev = require_gpu()
    B, M, K = 2, 2100, 1032
    Y, R, gp, gq, gt = make(dev, BF, BF, B, M, K, "channel", seed=8)
    if parts == "strided":
        Y, R = (torch.cat([t, t[..., :16]], -1)[..., :K] for t in (Y, R))
    Y[1, 7] = 0
    kw = dict(post_norm=True, post_gamma=gp, pre_gamma=gq, residual_scale=0.5, eps=EPS)
    if parts == "no Y":
        kw.update(post_norm=False, post_gamma=None)
        Y = None
    if parts == "no R":
        R = None
    if parts == "no gains":
        kw.update(post_gamma=None, pre_gamma=None)
    if parts == "channel gate":
        kw.update(gate=gt)
    if parts == "eps 0":
        kw.update(post_norm=False, post_gamma=None, eps=0.0)
    H, X = (torch.empty(B, M, K, dtype=BF, device=dev) for _ in range(2))
    rmm.rmm_block_join(Y, R, H, X=X, **kw)
    held, Xt, e = kmajor(dev, B, M, K, 5.0)
    H2 = R if parts == "in place" else torch.empty_like(H)
    rmm.rmm_block_join(Y, R, H2, Xt=Xt, energy=e, **kw)
    assert torch.equal(H, H2) and torch.equal(Xt.transpose(1, 2), X)
    assert bool((held[:, :, M:] == 5.0).all())
    check_energies(e.cpu().numpy(), X.double().square().sum(1).flatten().cpu().numpy(), M + 1)


def test_kmajor_matches_selection_input():
    """The energies are those of rmm_score on the row-major rows."""
    dev = require_gpu()
    Y, R, gp, gq, _ = make(dev, BF, BF, 1, 500, 1024, seed=4)
    H, X = torch.empty_like(R), torch.empty_like(Y)
    _, Xt, e = kmajor(dev, 1, 500, 1024)
    rmm.rmm_block_join(Y, R, H, Xt=Xt, energy=e, pre_gamma=gq)
    rmm.rmm_block_join(Y, R, H, X=X, pre_gamma=gq)
    e2 = torch.empty(1024, dtype=torch.float64, device=dev)
    ws = torch.empty(max(1, rmm.rmm_workspace_size(rmm.RMM_OP_SCORE, 1, 500, 1024)), dtype=torch.uint8, device=dev)
    rmm.rmm_score(X, e2, ws)
    check_energies(e.cpu().numpy(), e2.cpu().numpy(), 501)


@pytest.mark.parametrize("K", [128, 131])
@pytest.mark.parametrize("dt,sd", TYPES)
def test_in_place_and_strides(K, dt, sd):
    """H over R and X over Y, in rows of a longer stride, at an offset."""
    dev = require_gpu()
    B, M = 2, 6
    Y, R, gp, gq, _ = make(dev, dt, sd, B, M, K, seed=5)
    H, X = torch.empty_like(R), torch.empty_like(Y)
    kw = dict(post_norm=True, post_gamma=gp, pre_gamma=gq, residual_scale=0.5)
    rmm.rmm_block_join(Y, R, H, X=X, **kw)
    for off, ld in ((0, K), (3, K + 5), (8, K + 8), (1, K + 1)):
        a = torch.full((B * M * ld + 16,), 3.0, dtype=dt, device=dev)
        b = torch.full((B * M * ld + 16,), 3.0, dtype=sd, device=dev)
        Yv, Rv = (t[off:off + B * M * ld].view(B, M, ld)[:, :, :K] for t in (a, b))
        Yv.copy_(Y)
        Rv.copy_(R)
        rmm.rmm_block_join(Yv, Rv, Rv, X=Yv, **kw)
        assert torch.equal(Rv, H) and torch.equal(Yv, X)
        for t in (a, b):
            assert bool((t[off:off + B * M * ld].view(B, M, ld)[:, :, K:] == 3.0).all())
            assert bool((t[:off] == 3.0).all()) and bool((t[off + B * M * ld:] == 3.0).all())


def test_rows_of_zeros_and_extremes():
    dev = require_gpu()
    Y = torch.zeros(1, 4, 64, dtype=BF, device=dev)
    R = torch.zeros(1, 4, 64, dtype=F32, device=dev)
    R[0, 1] = 1e19                       # squares past fp32's range
    R[0, 2] = 1e-25
    H, X = torch.empty_like(R), torch.empty_like(Y)
    rmm.rmm_block_join(Y, R, H, X=X, post_norm=True, eps=0.0)
    # eps = 0: 0 * r(0) = 0 * infinity in both norms
    assert bool(X[0, 0].isnan().all())
    Y.fill_(1e-20)
    rmm.rmm_block_join(Y, R, H, X=X, eps=0.0)
    assert bool((X[0, 1] == 1).all()) and bool((X[0, 0] == 1).all()) and bool((X[0, 2] == 1).all())
    rmm.rmm_block_join(Y, R, H, X=X, eps=1.0)
    assert bool((H[0, 0] == Y[0, 0].float()).all()) and bool(X.isfinite().all())


@pytest.mark.parametrize("out", ["rows", "kmajor"])
def test_nonfinite_rows_stay_alone(out):
    dev = require_gpu()
    Y, R, gp, gq, _ = make(dev, BF, BF, 1, 70, 64, seed=6)
    Y[0, 3, 5], R[0, 66, 1] = math.nan, math.inf
    H, X = torch.empty_like(R), torch.empty_like(Y)
    _, Xt, e = kmajor(dev, 1, 70, 64)
    if out == "rows":
        rmm.rmm_block_join(Y, R, H, X=X, post_norm=True, post_gamma=gp, pre_gamma=gq)
    else:
        rmm.rmm_block_join(Y, R, H, Xt=Xt, energy=e, post_norm=True, post_gamma=gp, pre_gamma=gq)
        X = Xt.transpose(1, 2)
        assert bool(e.isnan().all())
    fine = torch.ones(70, dtype=torch.bool, device=dev)
    fine[3] = fine[66] = False
    assert bool(X[0, fine].isfinite().all()) and bool(X[0, 3].isnan().all()) and bool(X[0, 66, 1].isnan())


def test_repeats_are_bit_identical_on_streams_with_own_workspaces():
    dev = require_gpu()
    Y, R, gp, gq, _ = make(dev, BF, BF, 1, 2000, 1024, seed=7)
    outs = []
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for s in streams * 2:
        H = torch.empty_like(R)
        _, Xt, e = kmajor(dev, 1, 2000, 1024)
        torch.cuda.synchronize()
        rmm.rmm_block_join(Y, R, H, Xt=Xt, energy=e, post_norm=True, post_gamma=gp, pre_gamma=gq, stream=s)
        outs.append((H, Xt, e))
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))
    assert np.isfinite(outs[0][2].cpu().numpy()).all()


def test_past_32_bit_offsets():
    """The first and last rows and columns of tensors of more than 2^31 elements."""
    dev = require_gpu()
    M, K = 66000, 32768
    Y, R = (torch.ones(1, M, K, dtype=BF, device=dev) for _ in range(2))
    for t in (Y, R):
        t[0, -70:].normal_()
    g = (1 + 0.1 * torch.randn(K, device=dev)).to(BF)
    H, X = torch.empty_like(R), torch.empty_like(Y)
    Xt, e = torch.empty(1, K, M, dtype=BF, device=dev), torch.empty(K, dtype=torch.float64, device=dev)
    kw = dict(post_norm=True, post_gamma=g, pre_gamma=g, eps=EPS)
    for out in (dict(Xt=Xt, energy=e), dict(X=X)):
        H.zero_()
        rmm.rmm_block_join(Y, R, H, **out, **kw)
        for rows in (slice(0, 70), slice(M - 70, M)):
            check_h(H[:, rows], Y[:, rows], R[:, rows], True, g, None, 1.0, BF)
            check_x(X[:, rows] if "X" in out else Xt[:, :, rows].transpose(1, 2), H[:, rows], g, BF)
    squares = torch.zeros(K, dtype=torch.float64, device=dev)
    for r in range(0, M, 3000):
        assert torch.equal(Xt[0, :, r:r + 3000].T, X[0, r:r + 3000])
        squares += X[0, r:r + 3000].double().square().sum(0)
    check_energies(e.cpu().numpy(), squares.cpu().numpy(), M + 1)


@pytest.mark.parametrize("sd", [BF, F32])
@pytest.mark.parametrize("M,K", [(1, 64), (77, 1024), (300, 4096)])
def test_the_stream_itself_as_h(M, K, sd):
    """A norm of the stream alone, K-major, with the stream as H: it keeps its bits, and Xt and the energies are as with a copy."""
    dev = require_gpu()
    _, R, _, gq, _ = make(dev, BF, sd, 2, M, K, seed=11)
    R0, H = R.clone(), torch.empty_like(R)
    (_, xa, ea), (_, xb, eb) = (kmajor(dev, 2, M, K) for _ in range(2))
    rmm.rmm_block_join(None, R, H, Xt=xa, energy=ea, pre_gamma=gq, eps=EPS)
    rmm.rmm_block_join(None, R, R, Xt=xb, energy=eb, pre_gamma=gq, eps=EPS)
    assert torch.equal(R, R0) and torch.equal(H, R0) and torch.equal(xa, xb) and torch.equal(ea, eb)
