"""Attention over a paged cache where scores, keys or values are infinite, NaN or at the
type's ends: units kept whole and cut ones, few query rows and many."""
import numpy as np
import pytest
import torch

import paper_2608_13426_amd as rmm
from tests import paged_ref as pr
from tests.gpu_util import gpu, require_gpu

pytestmark = gpu
INF, NAN = float("inf"), float("nan")

# (L, n, H, Hkv, D): one sequence of L keys, n new tokens
FORMS = {
    "few": (40, 1, 8, 2, 128),
    "few_cut": (5000, 1, 8, 2, 64),
    "few_32": (50, 7, 8, 2, 128),
    "few_32_cut": (5000, 7, 8, 2, 128),
    "64": (90, 12, 8, 2, 64),               # 64-row units over a 4-bit cache, 256-row ones over bf16
    "64_cut": (5000, 12, 8, 2, 64),
    "rows": (200, 90, 8, 2, 64),
    "rows_cut": (6000, 90, 8, 2, 64),
    "rows_128": (700, 500, 2, 2, 128),
    "rows_128_cut": (9000, 300, 2, 2, 128),
}
PAGE = 16
both = pytest.mark.parametrize("mx", [False, True])
forms = pytest.mark.parametrize("form", FORMS)


def _make(form, mx, K, V, Q, causal=True, scale=None, idx=None, length=None):
    """(O, K, V as cached [L, Hkv, D] float64) of one call."""
    dev = Q.device
    L, Hkv, D = K.shape
    cache = rmm.kv_cache(-(-L // PAGE) + 1, Hkv, PAGE, D, mx=mx, device=dev)
    slots = torch.arange(PAGE, PAGE + L, dtype=torch.int32, device=dev)
    rmm.rmm_kv_append(K, V, slots, cache)
    kv = [torch.empty(L, Hkv, D, dtype=torch.bfloat16, device=dev) for _ in range(2)]
    rmm.rmm_kv_gather(cache, slots, *kv)
    table = torch.arange(1, 1 + -(-L // PAGE), dtype=torch.int32, device=dev)[None]
    start = torch.tensor([0, Q.shape[0]], dtype=torch.int32, device=dev)
    O = torch.full_like(Q, 3.0)
    rmm.rmm_paged_attention(Q, cache, table, torch.tensor([L if length is None else length], dtype=torch.int32, device=dev),
                            O, q_start=start, causal=causal, scale=scale, idx=idx)
    return O, kv[0].double(), kv[1].double()


def _inputs(form, seed):
    dev = require_gpu()
    L, n, H, Hkv, D = FORMS[form]
    g = torch.Generator(device=dev).manual_seed(seed)
    K, V = (torch.randn(L, Hkv, D, device=dev, generator=g).bfloat16() for _ in range(2))
    return L, n, H, Hkv, D, K, V, torch.randn(n, H, D, device=dev, generator=g).bfloat16()


def _check(O, K, V, Q, see, tokens, unrounded=True):
    """The given tokens against float64, token j over its first see[j] keys."""
    H, Hkv = Q.shape[1], K.shape[1]
    grp, D = H // Hkv, Q.shape[2]
    t = torch.as_tensor(tokens, device=Q.device)
    if not len(t):
        return
    rows = torch.as_tensor(see, device=Q.device)[t][:, None].expand(-1, grp).reshape(-1)
    for h in range(Hkv):
        q, o = (x[t, h * grp:(h + 1) * grp].reshape(-1, D).double() for x in (Q, O))
        pr.check(o, *pr.attend(q, K[:, h], V[:, h], rows, D ** -0.5, unrounded), what=f"kv head {h}")


@both
@forms
def test_every_score_minus_infinity(form, mx):
    """A softmax of nothing but -inf is NaN; only a token that sees no key gives 0.  The scores are
    -3e38 * 2e38 * scale, past fp32; the other heads' tokens are ordinary."""
    L, n, H, Hkv, D, K, V, Q = _inputs(form, 1)
    K[:, 0, 5] = -2e38
    Q[:, :, 5] = 0
    Q[::2, 0, 5] = 3e38                     # every second token of the first query head
    length = L if n == 1 else n - 1         # the first token sees no key
    O, Kc, Vc = _make(form, mx, K, V, Q, length=length)
    for j in range(n):
        if length - n + j + 1 <= 0:
            assert bool((O[j] == 0).all())
        elif j % 2 == 0:
            assert O[j, 0].isnan().all(), j
    assert O[:, H // Hkv:].isfinite().all()
    O, Kc, Vc = _make(form, mx, K, V, Q)
    assert O[::2, 0].isnan().all() and O[1::2].isfinite().all()
    Qz = Q.clone()
    Qz[::2, 0] = 0
    O[::2, 0] = _make(form, mx, K, V, Qz)[0][::2, 0]
    _check(O, Kc, Vc, Qz, [L - n + j + 1 for j in range(n)], range(n))


@both
@forms
def test_some_scores_minus_infinity(form, mx):
    """A key whose score is -inf has no weight, wherever the others lie (in other pieces too)."""
    L, n, H, Hkv, D, K, V, Q = _inputs(form, 2)
    Q[:, :, 5] = 3e38
    for lo, hi in ((0, L // 2), (L // 4, L - n), (L // 2, L - n)):
        Kb = K.clone()
        Kb[:, :, 5] = 0
        Kb[lo:hi, :, 5] = -2e38
        O, Kc, Vc = _make(form, mx, Kb, V, Q)
        left = torch.ones(L, dtype=torch.bool, device=Q.device)
        left[lo:hi] = False
        Qz = Q.clone()
        Qz[:, :, 5] = 0
        see = [int(left[:L - n + j + 1].sum()) for j in range(n)]
        if mx:                              # a group of 32 dims has one scale: the other keys' are as they were
            Kc = Kc.nan_to_num()
        _check(O, Kc[left], Vc[left], Qz, see, [j for j in range(n) if see[j]])


@both
@forms
def test_infinite_value_without_weight(form, mx):
    """0 * infinity is NaN: an infinite value whose weight is zero or too small for fp32 is not
    lost on the way through pieces; the other dims are as they would be."""
    L, n, H, Hkv, D, K, V, Q = _inputs(form, 3)
    K[:, :, 5] = 0
    K[:L // 2, :, 5] = -50
    Q[:, :, 5] = 400                        # scores 1768 to 2500 below the others', e^-1768 = 0 in fp32
    Vb = V.clone()
    Vb[3, :, 70 % D] = INF
    O, Kc, Vc = _make(form, mx, K, Vb, Q)
    see = [max(L - n + j + 1, 0) for j in range(n)]
    rows = [j for j in range(n) if see[j] > L // 2]
    lost = torch.zeros(D, dtype=torch.bool, device=Q.device)
    lost[slice(32 * (70 % D // 32), 32 * (70 % D // 32) + 32) if mx else 70 % D] = True
    assert not O[rows][..., lost].isfinite().any()
    assert O[rows][..., ~lost].isfinite().all()
    O[..., lost] = 0
    Vc[..., lost] = 0
    _check(O, Kc, Vc, Q, see, rows)


@both
@forms
def test_values_at_the_types_end(form, mx):
    """A weighted mean of finite values is finite, however large they are."""
    L, n, H, Hkv, D, K, V, Q = _inputs(form, 4)
    V = (V.sign() * 2.5e38).bfloat16()
    V[..., 0] = 2.5e38
    O, Kc, Vc = _make(form, mx, K, V, Q)
    assert Vc.isfinite().all()
    _check(O * 2.0 ** -100, Kc, Vc * 2.0 ** -100, Q, [L - n + j + 1 for j in range(n)], range(n))


@both
@forms
def test_visible_nonfinite_values(form, mx):
    """Infinite values that every token sees: their dims are infinite or NaN, the other dims and a
    query of NaN leave the rest alone; with one more NaN that only the last token sees."""
    L, n, H, Hkv, D, K, V, Q = _inputs(form, 5)
    Vb, Qb = V.clone(), Q.clone()
    Vb[L // 3 if n < L // 2 else 0, :, 40] = INF
    lost = torch.zeros(D, dtype=torch.bool, device=Q.device)
    lost[slice(32, 64) if mx else 40] = True
    Qb[n // 2, H - 1, 7] = NAN
    see = [L - n + j + 1 for j in range(n)]
    for hidden in (False, True):
        if hidden:
            if n == 1:
                break
            Vb[L - 1] = NAN
        O, Kc, Vc = _make(form, mx, K, Vb, Qb)
        assert O[n // 2, H - 1].isnan().all()
        assert not O[..., lost].isfinite().any()
        O[..., lost] = 0
        Vc[..., lost] = 0
        if hidden:
            assert O[n - 1][..., ~lost].isnan().all()
            Vc[L - 1] = 0
        rows = [j for j in range(n) if j != n // 2 and not (hidden and j == n - 1)]
        _check(O, Kc, Vc, Q, see, rows)
        if H > Hkv:                          # the NaN query's neighbours of the same token
            assert O[n // 2, :H - 1].isfinite().all() or (hidden and n // 2 == n - 1)


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("n,D", [(1, 128), (12, 64), (200, 128)])
def test_a_poisoned_key_costs_little(n, D, mx):
    """A NaN key and value that every token sees: the answer is NaN and takes no longer than 20
    passes without it (a second way through the keys, one row at a time, would)."""
    dev = require_gpu()
    L, H, Hkv = 40000, 8, 2
    g = torch.Generator(device=dev).manual_seed(6)
    K, V = (torch.randn(L, Hkv, D, device=dev, generator=g).bfloat16() for _ in range(2))
    Q = torch.randn(n, H, D, device=dev, generator=g).bfloat16()
    cache = rmm.kv_cache(L // PAGE, Hkv, PAGE, D, mx=mx, device=dev)
    rmm.rmm_kv_append(K, V, torch.arange(L, dtype=torch.int32, device=dev), cache)
    table = torch.arange(L // PAGE, dtype=torch.int32, device=dev)[None]
    length, start = (torch.tensor(x, dtype=torch.int32, device=dev) for x in ([L], [0, n]))
    O = torch.empty_like(Q)

    def passes():
        ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        best = 1e9
        for _ in range(5):
            ev[0].record()
            rmm.rmm_paged_attention(Q, cache, table, length, O, q_start=start)
            ev[1].record()
            torch.cuda.synchronize()
            best = min(best, ev[0].elapsed_time(ev[1]))
        return best
    clean = passes()
    assert O.isfinite().all()
    bad = torch.full((1, Hkv, D), NAN, dtype=torch.bfloat16, device=dev)
    for k, v in ((bad, bad), (K[L // 2:L // 2 + 1], bad)):
        rmm.rmm_kv_append(k, v, torch.tensor([L // 2], dtype=torch.int32, device=dev), cache)
        slow = passes()
        assert O.isnan().all()
        assert slow <= 20 * clean, (clean, slow)


@both
@pytest.mark.parametrize("n", [1, 8, 40])
def test_overlapping_sequences(n, mx):
    """A q_start whose sequences have more tokens than there are: NaN, whatever else it says."""
    dev = require_gpu()
    B, H, Hkv, D, L = 70, 4, 2, 128, 100
    g = torch.Generator(device=dev).manual_seed(7)
    cache = rmm.kv_cache(8, Hkv, PAGE, D, mx=mx, device=dev)
    table = (torch.arange(7, device=dev).expand(B, 7) + 1).int().contiguous()
    length = torch.full((B,), L, dtype=torch.int32, device=dev)
    Q = torch.randn(n * B, H, D, device=dev, generator=g).bfloat16()
    rows = torch.full((n * B, H + 1, D), 3.0, dtype=torch.bfloat16, device=dev)
    start = n * torch.arange(B + 1, dtype=torch.int32, device=dev)
    rmm.rmm_paged_attention(Q, cache, table, length, rows[:, :H], q_start=start)
    assert bool((rows[:, :H] == 0).all()) and bool((rows[:, H] == 3).all())      # a cache of zeros
    start[65] = 0                            # rows 0 .. 66 n once more
    rmm.rmm_paged_attention(Q, cache, table, length, rows[:, :H], q_start=start)
    assert rows[:, :H].isnan().all() and bool((rows[:, H] == 3).all())


@both
@forms
def test_scale_of_zero(form, mx):
    """The mean of the visible values; NaN where a score is infinite, whichever sign it has."""
    L, n, H, Hkv, D, K, V, Q = _inputs(form, 8)
    K[:, :, 5] = 0
    K[L - n, :, 5] = -2e38
    Q[:, :, 5] = 0
    O, Kc, Vc = _make(form, mx, K, V, Q, scale=0.0)
    see = [L - n + j + 1 for j in range(n)]
    _check(O, 0 * Kc, Vc, Q, see, range(n))
    for sign in (1, -1):
        Qb = Q.clone()
        Qb[0, 0, 5] = sign * 3e38
        Ob = _make(form, mx, K, V, Qb, scale=0.0)[0]
        assert Ob[0, 0].isnan().all()
        Ob[0, 0] = O[0, 0]
        assert torch.equal(O, Ob)
