"""Log probabilities, entropy and most likely tokens against float64."""
import math

import pytest
import torch

import paper_2608_13426_amd as rmm
from tests import block_ref as ref
from tests.gpu_util import gpu, require_gpu

pytestmark = gpu
BF, F32 = torch.bfloat16, torch.float32


def run(z, tokens=None, top=0, entropy=True, scale=1.0, stream=None):
    T, dev = z.shape[0], z.device
    lp = None if tokens is None else torch.full(tokens.shape, 77.0, device=dev)
    en = torch.full((T,), 77.0, device=dev) if entropy else None
    ti = torch.full((T, top), -5, dtype=torch.int32, device=dev) if top else None
    tl = torch.full((T, top), 77.0, device=dev) if top else None
    rmm.rmm_token_logprobs(z, tokens=tokens, logp=lp, entropy=en, top_idx=ti, top_logp=tl, scale=scale, stream=stream)
    return lp, en, ti, tl


def check(z, tokens, top, scale, got):
    lp, en, ti, tl = got
    want, ent, tol, etol = ref.logprobs(z, scale)

    def near(a, at, what):
        w, t = want.gather(1, at), tol.gather(1, at)
        fine = w.isfinite()
        assert torch.equal(a[~fine].double(), w[~fine]), what
        err = (a.double() - w).abs()[fine] / t[fine]
        assert err.numel() == 0 or float(err.max()) <= 1, (what, float(err.max()))

    if lp is not None:
        near(lp.reshape(z.shape[0], -1), tokens.reshape(z.shape[0], -1).long(), "logp")
    if en is not None:
        err = (en.double() - ent).abs() / etol
        assert float(err.max()) <= 1, ("entropy", float(err.max()))
    if ti is not None:
        at = ref.top_tokens(z, top)
        assert torch.equal(ti.long(), at)
        near(tl, at, "top")


def logits(dev, T, V, dt, seed=0, spread=3.0, pad=None):
    g = torch.Generator(device=dev).manual_seed(seed)
    ld = V if pad is None else pad
    z = torch.full((T, ld), 50.0, dtype=dt, device=dev)[:, :V]       # what stands behind a row is large
    z.copy_(spread * torch.randn(T, V, device=dev, generator=g))
    return z, torch.randint(0, V, (T, 3), device=dev, generator=g, dtype=torch.int32)


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 63, 64, 65, 511, 512, 513, 2047, 2048, 2049, 8191, 20000, 131072, 200003])
@pytest.mark.parametrize("T", [1, 5])
def test_sizes(dt, V, T):
    dev = require_gpu()
    z, tok = logits(dev, T, V, dt, pad=(V + 7) // 8 * 8 + 8)
    top = min(V, 20)
    check(z, tok, top, 1.0, run(z, tok, top))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("top", [1, 2, 5, 33, 63, 64])
@pytest.mark.parametrize("T,V", [(1, 60000), (3, 64), (200, 3001), (1300, 777)])
def test_top(dt, top, T, V):
    dev = require_gpu()
    z, tok = logits(dev, T, V, dt, seed=1)
    check(z, tok, top, 0.7, run(z, tok, top, scale=0.7))


@pytest.mark.parametrize("dt", [BF, F32])
def test_parts_and_odd_rows(dt):
    """Each output alone; rows at every offset of one element."""
    dev = require_gpu()
    z0, tok = logits(dev, 6, 1501, dt, seed=2)
    check(z0, tok, 0, 1.0, run(z0, tok, 0, entropy=False))
    check(z0, tok[:, 0], 0, 1.0, run(z0, tok[:, 0].contiguous(), 0, entropy=False))
    check(z0, None, 0, 2.5, run(z0, None, 0, scale=2.5))
    check(z0, None, 9, 1.0, run(z0, None, 9, entropy=False))
    for off, ld in ((1, 1501), (2, 1503), (4, 1504), (7, 1520)):
        mem = torch.full((6 * ld + 8,), 60.0, dtype=dt, device=dev)
        z = mem[off:off + 6 * ld].view(6, ld)[:, :1501]
        z.copy_(z0)
        check(z, tok, 7, 1.0, run(z, tok, 7))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [100, 5000, 70000])
def test_ties_go_to_the_lower_token(dt, V):
    dev = require_gpu()
    z = torch.zeros(4, V, dtype=dt, device=dev)
    z[1] = -0.0
    z[1, ::2] = 0.0
    z[2] = torch.arange(V, device=dev) % 3
    z[3, V // 2:] = 1
    tok = torch.tensor([[0, V - 1, V // 2]] * 4, dtype=torch.int32, device=dev)
    check(z, tok, 64, 1.0, run(z, tok, 64))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [300, 9000, 150000])
def test_order_of_the_row(dt, V):
    """Rising, falling and far-spread logits: the base moves often, or never."""
    dev = require_gpu()
    up = torch.linspace(-3000, 3000, V, device=dev)
    z = torch.stack([up, -up, up.roll(V // 3), 0.01 * up, up.abs()]).to(dt)
    tok = torch.randint(0, V, (5, 3), device=dev, dtype=torch.int32)
    check(z, tok, 64, 1.0, run(z, tok, 64))
    check(z, tok, 5, 0.01, run(z, tok, 5, scale=0.01))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [90, 4000, 100000])
def test_masks(dt, V):
    """-infinity or the type's lowest value in most places, in all but one, in all."""
    dev = require_gpu()
    for low in (-math.inf, torch.finfo(dt).min):
        z, tok = logits(dev, 5, V, dt, seed=3)
        z[0, torch.rand(V, device=dev) < 0.97] = low
        z[0, 11] = 0.5
        z[1, : V // 2] = low
        z[2] = low
        z[2, V - 1] = -3.0
        z[3, V // 3:] = low
        n = min(V, 64)
        check(z, tok, n, 1.0, run(z, tok, n))
        z[4] = low
        lp, en, ti, tl = run(z, tok, n)
        assert torch.equal(ti[4].cpu(), torch.arange(n, dtype=torch.int32))
        if low == -math.inf:
            assert float(en[4]) == 0 and bool((lp[4] == -math.inf).all()) and bool((tl[4] == -math.inf).all())
        else:
            want = -math.log(V)
            assert abs(float(en[4]) + want) < 1e-5 * -want and bool(((lp[4] - want).abs() < 1e-5 * -want).all())


def test_given_tokens_outside_the_row():
    dev = require_gpu()
    z, _ = logits(dev, 3, 1000, BF, seed=4)
    tok = torch.tensor([[-1, 5, 1000], [999, -2, 0], [2 ** 31 - 1, -2 ** 31, 7]], dtype=torch.int32, device=dev)
    lp, _, _, _ = run(z, tok)
    want = ref.logprobs(z, 1.0)[0]
    assert float(lp[0, 0]) == 0
    for i, j in ((0, 2), (1, 1), (2, 0), (2, 1)):
        assert math.isnan(float(lp[i, j]))
    for i, j in ((0, 1), (1, 0), (1, 2), (2, 2)):
        assert abs(float(lp[i, j]) - float(want[i, tok[i, j]])) < 1e-4


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("V", [200, 6000, 90000])
def test_nonfinite_rows_stay_alone(dt, V):
    dev = require_gpu()
    z, tok = logits(dev, 4, V, dt, seed=5)
    z[1, V // 2] = math.nan
    z[1, V - 1] = math.nan
    z[1, 3] = math.inf
    z[2, V - 2] = math.inf
    lp, en, ti, tl = run(z, tok, 8)
    assert torch.equal(ti.long(), ref.top_tokens(z, 8))
    for r in (1, 2):
        assert bool(lp[r].isnan().all()) and math.isnan(float(en[r])) and bool(tl[r].isnan().all())
    keep = torch.tensor([0, 3], device=dev)
    check(z[keep], tok[keep], 8, 1.0, (lp[keep], en[keep], ti[keep], tl[keep]))


def test_peaked_rows():
    """One token takes nearly all: its log probability is as small as the rest weighs."""
    dev = require_gpu()
    z = torch.zeros(3, 50000, dtype=F32, device=dev)
    z[0, 40000], z[1, 5], z[2, 49999] = 30.0, 60.0, 25.0
    tok = torch.tensor([[40000], [5], [49999]], dtype=torch.int32, device=dev)
    lp, en, _, _ = run(z, tok)
    want, ent, _, _ = ref.logprobs(z, 1.0)
    w = want.gather(1, tok.long())
    # in the lane that holds the peak the small weights of its own are lost: at most 2^-24
    assert bool(((lp.double() - w).abs() <= 2.0 ** -24 + 1e-5 * w.abs()).all())
    assert bool(((en.double() - ent).abs() <= 30 * 2.0 ** -23 + 1e-4 * ent).all())


def test_many_rows_match_few():
    """A row's results do not depend on how many rows the call has, up to the order of its sums."""
    dev = require_gpu()
    z, tok = logits(dev, 1500, 6001, BF, seed=6)
    many = run(z, tok, 10)
    check(z, tok, 10, 1.0, many)
    one = run(z[700:701], tok[700:701], 10)
    assert torch.equal(one[2], many[2][700:701])
    assert float((one[0] - many[0][700:701]).abs().max()) < 1e-5


def test_long_rows_past_32_bit_offsets():
    """The last rows of a tensor of more than 2^32 elements."""
    dev = require_gpu()
    T, V = 33000, 131072
    z = torch.empty(T, V, dtype=BF, device=dev)
    z.fill_(-1.0)
    z[-1].copy_(torch.randn(V, device=dev))
    z[-2, 5] = 4.0
    idx = torch.full((T, 3), -5, dtype=torch.int32, device=dev)
    lp = torch.empty(T, 3, device=dev)
    en = torch.empty(T, device=dev)
    rmm.rmm_token_logprobs(z, entropy=en, top_idx=idx, top_logp=lp)
    check(z[-2:], None, 3, 1.0, (None, en[-2:], idx[-2:], lp[-2:]))
    assert bool((idx[:-2].cpu() == torch.arange(3, dtype=torch.int32)).all())


@pytest.mark.parametrize("given", [0, 65, 300, 1000])
@pytest.mark.parametrize("V", [700, 40000])
def test_many_given_tokens(given, V):
    """More given tokens than a workgroup has threads; none beside the largest."""
    dev = require_gpu()
    z, _ = logits(dev, 3, V, BF, seed=7)
    tok = torch.randint(0, V, (3, given), device=dev, dtype=torch.int32)
    check(z, tok if given else None, 4, 1.0, run(z, tok, 4) if given else (None, *run(z, tok, 4)[1:]))


def nan_rows(z, tok, top, entropy=True):
    """Every result of z's rows, each of which holds a NaN, but the ranking is NaN."""
    lp, en, ti, tl = run(z, tok, top, entropy=entropy)
    assert bool(lp.isnan().all()), "logp"
    assert en is None or bool(en.isnan().all()), "entropy"
    if top:
        assert torch.equal(ti.long(), ref.top_tokens(z, top)) and bool(tl.isnan().all()), "top"


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("T,V", [(1, 513), (1, 9000), (1, 150000), (5, 20000), (1300, 1500), (1300, 9000)])
@pytest.mark.parametrize("rest", ["lowest", "-inf", "low"])
def test_a_nan_among_masked_logits(dt, T, V, rest):
    """One NaN where every other logit is masked or far below: its wave's base weighs
    nothing beside the row's."""
    dev = require_gpu()
    low = {"lowest": torch.finfo(dt).min, "-inf": -math.inf, "low": -300.0}[rest]
    for at in (V - 1, 512, V // 2):
        z, tok = logits(dev, T, V, dt, seed=8)
        z[:, 300:] = low
        z[:, at] = math.nan
        nan_rows(z, tok % 300, 6)
        nan_rows(z, tok % 300, 0, entropy=False)
        z[:, at] = low                       # without it the row is an ordinary one
        check(z, tok % 300, 6, 1.0, run(z, tok % 300, 6))


@pytest.mark.parametrize("dt", [BF, F32])
@pytest.mark.parametrize("T,V", [(1, 513), (1, 9000), (1, 150000), (5, 20000), (1300, 1500), (1300, 9000)])
@pytest.mark.parametrize("level", [100.0, 300.0, -300.0])
def test_a_run_of_nan(dt, T, V, level):
    """Waves and pieces of nothing but NaN beside logits far from 0."""
    dev = require_gpu()
    z, tok = logits(dev, T, V, dt, seed=9)
    z += level
    z[:, min(512, V - 1):] = math.nan
    nan_rows(z, tok % 512, 6)
    nan_rows(z, tok % 512, 0, entropy=False)
