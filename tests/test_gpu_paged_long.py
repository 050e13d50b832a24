"""Attention over a paged cache at the lengths and batch sizes where its work is cut in
every way there is (tests/paged_cases.py), within limits that a lost or doubled run of
keys would pass; and the short shapes within the same limits."""
import numpy as np
import pytest
import torch

import paper_2608_13426_amd as rmm
from tests import paged_cases as pc
from tests import paged_ref as pr
from tests import test_gpu_paged_attention as short
from tests.gpu_util import gpu, require_gpu

pytestmark = gpu


def _compare(O, Q, hist, seqs, lens, starts, news, Hkv, scale, causal, unrounded, what, keep=None):
    """The given sequences' rows, which read one history (K, V [L, Hkv, D])."""
    grp, D = Q.shape[1] // Hkv, Q.shape[2]
    tok = torch.cat([torch.arange(starts[b], starts[b] + news[b]) for b in seqs]).to(Q.device)
    see = torch.cat([torch.arange(lens[b] - news[b], lens[b]) + 1 if causal else torch.full((news[b],), lens[b])
                     for b in seqs]).clamp_min(0).to(Q.device)
    see = see[:, None].expand(-1, grp).reshape(-1)
    K, V = hist
    step = max(1, 2 ** 26 // max(len(K), 1))
    for g in range(Hkv):
        q, o = (x[tok, g * grp:(g + 1) * grp].reshape(-1, D).double() for x in (Q, O))
        kp = None if keep is None else keep[tok, g * grp:(g + 1) * grp].reshape(-1, D)
        k, v = K[:, g].double(), V[:, g].double()
        for r in range(0, len(q), step):
            ref = pr.attend(q[r:r + step], k, v, see[r:r + step], scale, unrounded, None if kp is None else kp[r:r + step])
            pr.check(o[r:r + step], *ref, what=f"{what}, kv head {g}, rows from {r}")


def _long(dev, mx, case):
    _, D, H, Hkv, causal, page, lens, news, _ = case
    g = torch.Generator(device=dev).manual_seed(len(lens) + D + page)
    B, per = len(lens), -(-max(lens) // page)
    cache = rmm.kv_cache(2 * per + 1, Hkv, page, D, mx=mx, device=dev)
    rows = torch.randperm(2 * per + 1, device=dev, generator=g)[:2 * per].int().view(2, per)
    spread = torch.randn(Hkv, D, device=dev, generator=g).abs() + 0.1
    hist = []
    for h in range(2):
        L = max(lens[h::2], default=1)
        t = torch.arange(L, device=dev)
        slots = (rows[h, t // page] * page + t % page).int()
        rmm.rmm_kv_append((torch.randn(L, Hkv, D, device=dev, generator=g) * spread).bfloat16(),
                          torch.randn(L, Hkv, D, device=dev, generator=g).bfloat16(), slots, cache)
        kv = [torch.empty(L, Hkv, D, dtype=torch.bfloat16, device=dev) for _ in range(2)]
        hist.append(rmm.rmm_kv_gather(cache, slots, *kv))
    table = rows[torch.arange(B, device=dev) % 2].contiguous()
    n = [1] * B if news is None else news
    starts = np.cumsum([0] + n)
    q_start = None if news is None else torch.tensor(starts, dtype=torch.int32, device=dev)
    Q = torch.randn(int(starts[-1]), H, D, device=dev, generator=g).bfloat16()
    return cache, table, q_start, Q, torch.tensor(lens, dtype=torch.int32, device=dev), hist, n, starts


LONG = [(n, t) for n, c in pc.CASES.items() for t in c[0]]


@pytest.mark.parametrize("name,kind", LONG)
def test_long(name, kind):
    dev = require_gpu()
    case = pc.CASES[name]
    _, D, H, Hkv, causal, page, lens, _, _ = case
    cache, table, q_start, Q, length, hist, news, starts = _long(dev, kind == "mx", case)
    O = torch.empty_like(Q)
    rmm.rmm_paged_attention(Q, cache, table, length, O, q_start=q_start, causal=causal)
    for h in range(2):
        if len(lens) > h:
            _compare(O, Q, hist[h], range(h, len(lens), 2), lens, starts, news, Hkv, D ** -0.5, causal,
                     D == 128, f"{name}, history {h}")
    O2 = torch.empty_like(Q)
    rmm.rmm_paged_attention(Q, cache, table, length, O2, q_start=q_start, causal=causal)
    assert torch.equal(O, O2)


@pytest.mark.parametrize("name,kind", [c for c in LONG if "long" in c[0]])
def test_bad_page_late(name, kind):
    """A page number outside the cache that is read long after a piece's first ones."""
    dev = require_gpu()
    case = pc.CASES[name]
    causal, page, lens = case[4], case[5], case[6]
    cache, table, q_start, Q, length, _, news, starts = _long(dev, kind == "mx", case)
    O, O2 = torch.empty_like(Q), torch.empty_like(Q)
    rmm.rmm_paged_attention(Q, cache, table, length, O, q_start=q_start, causal=causal)
    b = 1
    for at in (lens[b] // page // 2, (lens[b] - news[b]) // page - 1):
        t2 = table.clone()
        t2[b, at] = cache.n_pages
        rmm.rmm_paged_attention(Q, cache, t2, length, O2, q_start=q_start, causal=causal)
        rows = slice(int(starts[b]), int(starts[b + 1]))
        assert O2[rows].isnan().all()
        O2[rows] = O[rows]
        assert torch.equal(O, O2)


_ARGS, _SHAPES = next(m.args for m in short.test_attention.pytestmark if m.args[0].startswith("lens"))


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize(_ARGS, _SHAPES)
def test_short(lens, news, H, Hkv, D, page, causal, r, scale, mx):
    """The shapes of the other file's test, element by element and row by row."""
    dev = require_gpu()
    cache, table, q_start, Q, idx = short._setup(dev, lens, news, H, Hkv, D, page, mx, len(lens) * 1000 + D, r)
    O = torch.empty_like(Q)
    length = torch.tensor(lens, dtype=torch.int32, device=dev)
    rmm.rmm_paged_attention(Q, cache, table, length, O, q_start=q_start, idx=idx, causal=causal, scale=scale)
    keep = None
    if idx is not None:
        keep = torch.zeros(*Q.shape, dtype=torch.bool, device=dev).scatter_(2, idx.long(), True)
    unrounded = D == 128 and sum(news) * (H // Hkv) > 32 * len(lens)
    starts = np.cumsum([0] + list(news))
    for b, L in enumerate(lens):
        if news[b] and L > 0:
            t = torch.arange(L, device=dev)
            slots = (table[b, t // page] * page + t % page).int()
            kv = [torch.empty(L, Hkv, D, dtype=torch.bfloat16, device=dev) for _ in range(2)]
            _compare(O, Q, rmm.rmm_kv_gather(cache, slots, *kv), [b], lens, starts, news, Hkv,
                     D ** -0.5 if scale is None else float(np.float32(scale)), causal, unrounded, f"sequence {b}", keep)


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("n,H,Hkv,D", [(1, 8, 2, 128), (7, 8, 2, 64), (12, 8, 2, 64), (40, 4, 2, 128), (90, 8, 2, 64),
                                       (300, 4, 2, 128)])
def test_rising_maximum(n, H, Hkv, D, mx):
    """Two keys have all the weight, the heavier one later and in the same stream of keys: each is
    the largest when it comes, so neither weight is rounded and what is left are the scores' errors
    and the output's rounding.  Their values almost cancel, which makes a rounded weight show."""
    dev = require_gpu()
    L, page, at = 1000, 16, 130
    g = torch.Generator(device=dev).manual_seed(n)
    cache = rmm.kv_cache(-(-L // page), Hkv, page, D, mx=mx, device=dev)
    K, V = torch.zeros(L, Hkv, D, device=dev), torch.zeros(L, Hkv, D, device=dev)
    K[:, :, 5], K[0, :, 5], K[at, :, 5] = -96, 0, 2
    V[0], V[at] = 6, torch.tensor([-1.0, -0.5, -0.25, -0.125], device=dev).repeat(D // 4)
    slots = torch.arange(L, dtype=torch.int32, device=dev)
    rmm.rmm_kv_append(K.bfloat16(), V.bfloat16(), slots, cache)
    Q = torch.zeros(n, H, D, dtype=torch.bfloat16, device=dev)
    Q[:, :, 5] = (8 + 16 * torch.rand(n, H, device=dev, generator=g)) * (D / 128) ** 0.5     # scores of 1.4 to 4.2
    O = torch.empty_like(Q)
    rmm.rmm_paged_attention(Q, cache, slots.view(1, -1)[:, :-(-L // page)].contiguous(),
                            torch.tensor([L], dtype=torch.int32, device=dev), O,
                            q_start=torch.tensor([0, n], dtype=torch.int32, device=dev))
    k, v = (torch.empty(L, Hkv, D, dtype=torch.bfloat16, device=dev) for _ in range(2))
    rmm.rmm_kv_gather(cache, slots, k, v)
    q = Q.double().view(n * H, D)
    assert torch.equal(k, K.bfloat16()) and torch.equal(v, V.bfloat16())
    want, _, _ = pr.attend(q, k[:, 0].double(), v[:, 0].double(), torch.full((n * H,), L, device=dev), D ** -0.5, False)
    eps = (8 * 6 + 64) * 4 * 2.0 ** -24              # relative, of a weight: scores of up to 6, the exponential
    limit = 1.01 * 2.0 ** -8 * want.abs() + 8 * eps
    assert bool(((O.double().view(n * H, D) - want).abs() <= limit).all())
