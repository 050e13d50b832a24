"""Rotation and per-head norms of queries and keys, and the paged cache's append
and read-back, against float64 definitions."""
import numpy as np
import pytest
import torch

import paper_2608_13426_amd as rmm
from tests import cache_ref as cr
from tests.gpu_util import U16, U32, check_energies, gpu, require_gpu

pytestmark = gpu


def _gen(dev, seed):
    return torch.Generator(device=dev).manual_seed(seed)


def _randn(g, dev, *shape):
    x = torch.randn(*shape, device=dev, generator=g)
    x[..., ::37] *= 20
    return x


def _check(got, want, err, dtype):
    u = U16 if dtype == torch.bfloat16 else U32
    assert np.all(np.abs(got - want) <= (u * np.abs(want) + err) * (1 + u))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("batch,L,H,Hkv,D,rot,inter,norm", [
    (1, 1, 1, 1, 64, 64, False, "qk"),          # one token, one head
    (3, 1, 32, 8, 128, 128, False, ""),         # a decode step
    (1, 5, 3, 1, 128, 128, True, "q"),          # odd head count; a norm on one side only
    (2, 67, 5, 5, 128, 80, False, "qk"),        # rotation pieces that do not fill the lanes
    (1, 130, 9, 3, 64, 16, False, "k"),
    (2, 33, 4, 2, 64, 48, True, "qk"),
    (1, 300, 16, 2, 128, 0, False, "qk"),       # no rotation
    (1, 1100, 24, 8, 128, 128, False, ""),      # several tokens per wave
])
def test_rotate(batch, L, H, Hkv, D, rot, inter, norm, dtype):
    dev = require_gpu()
    g = _gen(dev, L * 31 + D)
    rows = _randn(g, dev, batch, L, H + 2 * Hkv, D).to(dtype)      # a projection's rows: strided heads
    Q, K = rows[:, :, :H], rows[:, :, H:H + Hkv]
    cos, sin = rmm.rope_tables(4096, max(rot, 16), 500000.0, dev)
    rope = rmm.Rope(cos, sin, inter) if rot else None
    pos = torch.randint(0, 4096, (batch * L,), device=dev, generator=g, dtype=torch.int32)
    gq = (1 + 0.1 * _randn(g, dev, D)).to(dtype) if "q" in norm else None
    gk = (1 + 0.1 * _randn(g, dev, D)).to(dtype) if "k" in norm else None
    Qo = torch.empty(batch, H, L, D, dtype=dtype, device=dev)
    Ko = torch.empty(batch, Hkv, L, D, dtype=dtype, device=dev)
    e = torch.empty(batch * H * D, dtype=torch.float64, device=dev)
    rmm.rmm_qk_norm_rope(Q, Qo, pos if rot else None, rope, K=K, Ko=Ko, gamma_q=gq, gamma_k=gk, eps=cr.EPS, energy=e)
    tab = (cr.np64(cos), cr.np64(sin)) if rot else (None, None)
    for x, o, gm in ((Q, Qo, gq), (K, Ko, gk)):
        want, err = cr.rotate(cr.np64(x).reshape(batch * L, -1, D), None if gm is None else cr.np64(gm),
                              pos.cpu().numpy(), *tab, inter)
        _check(cr.np64(o).transpose(0, 2, 1, 3).reshape(want.shape), want, err, dtype)
    check_energies(e.cpu().numpy(), (cr.np64(Qo) ** 2).sum(2).reshape(-1), L)
    # the same values without energies, in place, and for the queries alone
    P = rows.clone()
    rmm.rmm_qk_norm_rope(P[:, :, :H], P[:, :, :H].transpose(1, 2), pos if rot else None, rope, gamma_q=gq, eps=cr.EPS)
    assert torch.equal(P[:, :, :H].transpose(1, 2), Qo) and torch.equal(P[:, :, H:], rows[:, :, H:])
    # energies as the scoring pass forms them from the rotated heads
    e2 = torch.empty_like(e)
    ws = torch.empty(max(1, rmm.rmm_workspace_size(rmm.RMM_OP_SCORE, batch * H, L, D)), dtype=torch.uint8, device=dev)
    rmm.rmm_score(Qo.view(batch * H, L, D), e2, ws)
    assert torch.allclose(e, e2, rtol=2 * (L + 1) * 2.0 ** -53, atol=0)


def test_energies_of_many_sequences():
    """More sequences than a grid's second axis holds, each over two workgroups' tokens."""
    dev = require_gpu()
    batch, L, D = 65537, 65, 64
    Q = _randn(_gen(dev, 9), dev, batch, L, 1, D).bfloat16()
    Qo = torch.empty(batch, 1, L, D, dtype=Q.dtype, device=dev)
    cos, sin = rmm.rope_tables(128, D, device=dev)
    pos = torch.arange(L, dtype=torch.int32, device=dev).repeat(batch)
    e = torch.empty(batch * D, dtype=torch.float64, device=dev)
    rmm.rmm_qk_norm_rope(Q, Qo, pos, rmm.Rope(cos, sin), energy=e)
    want, err = cr.rotate(cr.np64(Q[-2:]).reshape(2 * L, 1, D), None, pos[:2 * L].cpu().numpy(), cr.np64(cos), cr.np64(sin), False)
    _check(cr.np64(Qo[-2:]).reshape(want.shape), want, err, Q.dtype)
    check_energies(e.cpu().numpy(), (Qo.double() ** 2).sum(2).reshape(-1).cpu().numpy(), L)


def test_rotate_positions_and_nonfinite():
    """Positions outside the tables give NaN heads; a NaN or infinite value stays in its pair (or, normed, head)."""
    dev = require_gpu()
    D, T = 128, 6
    x = torch.ones(1, T, 2, D, dtype=torch.bfloat16, device=dev)
    x[0, 3, 1, 5], x[0, 4, 0, 70] = float("nan"), float("inf")
    cos, sin = rmm.rope_tables(100, D, device=dev)
    pos = torch.tensor([0, -1, 100, 99, 1, 2 ** 31 - 1], dtype=torch.int32, device=dev)
    o = torch.empty(1, 2, T, D, dtype=torch.bfloat16, device=dev)
    rmm.rmm_qk_norm_rope(x, o, pos, rmm.Rope(cos, sin))
    o = o[0].transpose(0, 1).float()
    for t in (1, 2, 5):
        assert o[t].isnan().all()
    assert torch.equal(o[0], torch.ones_like(o[0]))
    bad = ~o[3].isfinite()
    assert bad.sum() == 2 and bad[1, 5] and bad[1, 69]
    bad = ~o[4].isfinite()
    assert bad.sum() == 2 and bad[0, 70] and bad[0, 6]


def _cache(dev, n_pages, Hkv, page, D, mx, strided):
    """A cache filled with a known pattern; strided: pages interleaved with those of another layer."""
    m = 2 if strided else 1
    if not mx:
        ts = [torch.full((n_pages, m, Hkv, page, D), 7.0, dtype=torch.bfloat16, device=dev) for _ in range(2)]
    else:
        ts = [torch.full((n_pages, m, Hkv, page, w), 0x5A, dtype=torch.uint8, device=dev)
              for w in (D // 2, D // 2, D // 32, D // 32)]
    return ts, rmm.KvCache(*(t[:, m - 1] for t in ts))


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("T,H,Hkv,D,page,rot,inter,norm,strided", [
    (1, 0, 1, 64, 16, 64, False, False, False),
    (7, 4, 2, 128, 16, 128, False, True, True),
    (33, 8, 8, 128, 64, 80, False, False, False),
    (50, 3, 1, 64, 32, 32, True, True, True),
    (520, 0, 3, 128, 128, 0, False, True, False),
    (1300, 6, 2, 128, 1024, 128, True, False, True),
])
def test_append_and_gather(T, H, Hkv, D, page, rot, inter, norm, strided, mx):
    dev = require_gpu()
    g = _gen(dev, T + page)
    n_pages = -(-T // page) + 3
    raw, cache = _cache(dev, n_pages, Hkv, page, D, mx, strided)
    before = [t.clone() for t in raw]
    rows = _randn(g, dev, T, H + 2 * Hkv, D).bfloat16()
    K, V = rows[:, H:H + Hkv], rows[:, H + Hkv:]
    slots = torch.randperm(n_pages * page, device=dev, generator=g)[:T].int()
    out = torch.zeros(T, dtype=torch.bool, device=dev)
    if T > 2:                                   # tokens that are not appended
        slots[1], slots[T // 2], slots[2] = -1, n_pages * page, -(2 ** 31)
        out[1] = out[T // 2] = out[2] = True
    cos, sin = rmm.rope_tables(2000, max(rot, 16), device=dev)
    pos = torch.randint(0, 2000, (T,), device=dev, generator=g, dtype=torch.int32)
    gm = [(1 + 0.1 * _randn(g, dev, D)).bfloat16() if norm else None for _ in range(2)]
    rope = rmm.Rope(cos, sin, inter) if rot else None
    q = {}
    if H:
        q = dict(Q=rows[:, :H], Qo=torch.empty(T, H, D, dtype=torch.bfloat16, device=dev), gamma_q=gm[1])
    rmm.rmm_kv_append(K, V, slots, cache, positions=pos if rot else None, rope=rope, gamma_k=gm[0], eps=cr.EPS, **q)
    tab = (cr.np64(cos), cr.np64(sin)) if rot else (None, None)
    p = pos.cpu().numpy()

    def turned(x, gamma):
        return cr.rotate_f32(cr.np64(x), None if gamma is None else cr.np64(gamma), p, *tab, inter)
    if H:
        assert np.array_equal(cr.np64(q["Qo"]), cr.bf16(turned(rows[:, :H], gm[1])))
    kept = (~out).cpu().numpy()
    Kr = torch.full((Hkv, T, D), 3.0, dtype=torch.bfloat16, device=dev)       # heads-major: strided rows
    Vr = torch.full((T, Hkv, D), 3.0, dtype=torch.bfloat16, device=dev)
    rmm.rmm_kv_gather(cache, slots, Kr.transpose(0, 1), Vr)
    for got, x, gamma in ((Kr.transpose(0, 1), K, gm[0]), (Vr, V, None)):
        want = turned(x, gamma) if x is K else cr.np64(x)
        want = cr.mx_round(want) if mx else cr.bf16(want)
        want[~kept] = 0
        assert np.array_equal(cr.np64(got), want)
    # nothing else in the cache has changed
    touched = torch.zeros(n_pages, page, dtype=torch.bool, device=dev)
    s = slots[~out].long()
    touched[s // page, s % page] = True
    m = raw[0].shape[1]
    for a, b in zip(raw, before):
        same = (a == b).all(-1)                 # [pages, layers, heads, page]
        assert same[:, :m - 1].all() and same[:, m - 1].transpose(1, 2)[~touched].all()


def test_mx_special_values():
    """Groups of zeros, of the type's extremes, ties, NaN and infinities."""
    dev = require_gpu()
    D = 128
    v = torch.zeros(8, 1, D)
    v[0, 0, :34] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 4 + [-0.25, -5.0])
    v[1] = 2.0 ** -130
    v[2, 0, ::3] = torch.finfo(torch.bfloat16).max
    v[3, 0, 1] = 6.96875                        # rounds to 6 at the scale of 1
    v[4, 0, 1] = 7.0                            # rounds to 8: the next scale
    v[5, 0, 40] = float("nan")
    v[6, 0, 100] = float("-inf")
    v[7, 0, 5], v[7, 0, 6] = 1.0, 2.0 ** -9
    v = v.bfloat16().to(dev)
    cache = rmm.kv_cache(1, 1, 16, D, mx=True, device=dev)
    slots = torch.arange(8, dtype=torch.int32, device=dev)
    rmm.rmm_kv_append(v, v, slots, cache)
    K, V = torch.empty_like(v), torch.empty_like(v)
    rmm.rmm_kv_gather(cache, slots, K, V)
    want = cr.mx_round(cr.np64(v))
    assert np.array_equal(cr.np64(K), want, equal_nan=True) and np.array_equal(cr.np64(V), want, equal_nan=True)
    assert np.isnan(want[5, 0, 32:64]).all() and np.isfinite(want[5, 0, :32]).all()
    assert np.array_equal(cr.mx_values(cache.k[0, :, :8].cpu().numpy(), cache.k_scale[0, :, :8].cpu().numpy())[0],
                          want[:, 0], equal_nan=True)


def test_gather_reads_every_scale():
    """Bytes that the append never writes read as what they stand for."""
    dev = require_gpu()
    D, n = 64, 256
    cache = rmm.kv_cache(n // 16, 1, 16, D, mx=True, device=dev)
    cache.k.copy_(torch.randint(0, 256, cache.k.shape, dtype=torch.uint8, device=dev))
    cache.k_scale.copy_(torch.arange(256, device=dev).view(16, 1, 16, 1).expand(16, 1, 16, 2).to(torch.uint8))
    K, V = (torch.empty(n, 1, D, dtype=torch.bfloat16, device=dev) for _ in range(2))
    rmm.rmm_kv_gather(cache, torch.arange(n, dtype=torch.int32, device=dev), K, V)
    want = cr.mx_values(cache.k.cpu().numpy(), cache.k_scale.cpu().numpy()).reshape(n, 1, D)
    want[np.abs(want) >= 2.0 ** 128] = np.sign(want[np.abs(want) >= 2.0 ** 128]) * np.inf
    assert np.array_equal(cr.np64(K), want, equal_nan=True)
    assert np.array_equal(cr.np64(V), np.zeros_like(want))


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("T,Hkv,D", [(4101, 8, 128), (8203, 8, 64), (13120, 5, 128)])
def test_gather_many(T, Hkv, D, mx):
    """Several rows per thread: what reading the same slots in short runs gives, nothing past the end."""
    dev = require_gpu()
    g = _gen(dev, T)
    raw, cache = _cache(dev, 40, Hkv, 32, D, mx, True)
    for t in raw[:2]:
        t.copy_(torch.randint(0, 256, t.shape, device=dev, generator=g).to(t.dtype))
    for t in raw[2:]:
        t.copy_(torch.randint(100, 140, t.shape, device=dev, generator=g).to(t.dtype))
    slots = torch.randint(-20, 40 * 32 + 20, (T,), device=dev, generator=g, dtype=torch.int32)
    K = torch.full((Hkv, T + 1, D), 3.0, dtype=torch.bfloat16, device=dev)
    V = torch.full((T + 1, Hkv, D), 3.0, dtype=torch.bfloat16, device=dev)
    rmm.rmm_kv_gather(cache, slots, K[:, :T].transpose(0, 1), V[:T])
    k, v = (torch.empty(1000, Hkv, D, dtype=torch.bfloat16, device=dev) for _ in range(2))
    for t in range(0, T, 1000):
        n = min(1000, T - t)
        rmm.rmm_kv_gather(cache, slots[t:t + n], k[:n], v[:n])
        assert torch.equal(K[:, t:t + n].transpose(0, 1), k[:n]) and torch.equal(V[t:t + n], v[:n])
    assert bool((K[:, T] == 3.0).all()) and bool((V[T] == 3.0).all())
    out = (slots < 0) | (slots >= 40 * 32)
    assert bool((V[:T][out] == 0).all()) and bool((V[:T][~out] != 0).any())


@pytest.mark.parametrize("mx", [False, True])
def test_same_slot_twice(mx):
    """Each 8-element piece of a slot named twice is one of its tokens'."""
    dev = require_gpu()
    g = _gen(dev, 5)
    cache = rmm.kv_cache(2, 2, 16, 128, mx=mx, device=dev)
    x = torch.randn(4, 2, 128, device=dev, generator=g).sign().bfloat16()       # one scale for all
    slots = torch.tensor([3, 9, 3, 3], dtype=torch.int32, device=dev)
    rmm.rmm_kv_append(x, x, slots, cache)
    K, V = torch.empty_like(x), torch.empty_like(x)
    rmm.rmm_kv_gather(cache, slots, K, V)
    assert torch.equal(K[1], x[1]) and torch.equal(K[0], K[2])
    pieces = (K[0].view(1, 2, 16, 8) == x[[0, 2, 3]].view(3, 2, 16, 8)).all(-1)
    assert pieces.any(0).all()


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("T", [1, 37, 700])
def test_append_queries_in_place(T, mx):
    """Queries rotated where they lie, in the same rows as the keys and values that are appended."""
    dev = require_gpu()
    H, Hkv, D = 6, 2, 128
    rows = _randn(_gen(dev, T), dev, T, H + 2 * Hkv, D).bfloat16()
    slots = torch.arange(T, dtype=torch.int32, device=dev)
    rope = rmm.Rope(*rmm.rope_tables(1000, D, device=dev))
    got = []
    for place in (False, True):
        x = rows.clone()
        q = x[:, :H] if place else torch.empty(T, H, D, dtype=x.dtype, device=dev)
        cache = rmm.kv_cache(-(-T // 16), Hkv, 16, D, mx=mx, device=dev)
        rmm.rmm_kv_append(x[:, H:H + Hkv], x[:, H + Hkv:], slots, cache, positions=slots, rope=rope, Q=x[:, :H], Qo=q)
        assert torch.equal(x[:, H:], rows[:, H:])
        got.append((q.clone(), cache.k, cache.v))
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_large_cache_offsets():
    """A cache past 4 GiB: the last page is written, read and attended."""
    dev = require_gpu()
    n_pages, Hkv, page, D = 150000, 8, 16, 128
    k = torch.empty(n_pages, Hkv, page, D, dtype=torch.bfloat16, device=dev)
    cache = rmm.KvCache(k, torch.empty_like(k))
    g = _gen(dev, 2)
    x, y = (torch.randn(page, Hkv, D, device=dev, generator=g).bfloat16() for _ in range(2))
    slots = (n_pages - 1) * page + torch.arange(page, dtype=torch.int32, device=dev)
    rmm.rmm_kv_append(x, y, slots, cache)
    assert torch.equal(k[-1].transpose(0, 1), x) and torch.equal(cache.v[-1].transpose(0, 1), y)
    K, V = torch.empty_like(x), torch.empty_like(y)
    rmm.rmm_kv_gather(cache, slots, K, V)
    assert torch.equal(K, x) and torch.equal(V, y)
    Q = torch.randn(1, 16, D, device=dev, generator=g).bfloat16()
    O = torch.empty_like(Q)
    table = torch.tensor([[n_pages - 1]], dtype=torch.int32, device=dev)
    rmm.rmm_paged_attention(Q, cache, table, torch.tensor([13], dtype=torch.int32, device=dev), O)
    want, bound = cr.attend(cr.np64(Q), *cr.history(cache, table, 0, 13), 1, D ** -0.5, True)
    assert np.all(np.abs(cr.np64(O) - want) <= bound)
