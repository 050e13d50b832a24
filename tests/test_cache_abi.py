"""Host-side checks of the rotation, cache and cache-attention entry points: only
calls that are refused before any HIP call are made here."""
import ctypes

import pytest
import torch

import paper_2608_13426_amd as rmm

INVALID, UNSUPPORTED, WS_SMALL = 1, 2, 3
A = 0x100000                           # an aligned address that is never dereferenced
P = ctypes.c_void_p(A)


def heads(n=4, data=A, sb=0, st=2048, sh=128):
    return rmm._Heads(data, n, sb, st, sh)


def rope(**kw):
    d = dict(cos=A, sin=A, n_pos=100, rot=128, interleaved=0)
    d.update(kw)
    return rmm._RopeTables(*d.values())


def cache(mx=False, **kw):
    row = 64 if mx else 256
    d = dict(type=int(mx), k=A, v=A, k_scale=A if mx else None, v_scale=A if mx else None, n_pages=10, page_size=16,
             Hkv=4, D=128, k_stride=64 * row, v_stride=64 * row, k_scale_stride=64 * 4, v_scale_stride=64 * 4)
    d.update(kw)
    return rmm._KvCacheC(*d.values())


BAD_HEADS = [(dict(data=None), INVALID), (dict(n=0), INVALID), (dict(st=-8), INVALID), (dict(sh=-8), INVALID),
             (dict(data=A + 8), UNSUPPORTED), (dict(st=2049), UNSUPPORTED), (dict(sh=4), UNSUPPORTED),
             (dict(n=70000), UNSUPPORTED)]
BAD_ROPE = [(dict(cos=None), INVALID), (dict(sin=None), INVALID), (dict(n_pos=0), INVALID), (dict(rot=144), INVALID),
            (dict(rot=-16), INVALID), (dict(rot=72), UNSUPPORTED), (dict(cos=A + 4), UNSUPPORTED),
            (dict(n_pos=2 ** 31), UNSUPPORTED)]
BAD_CACHE = [(dict(type=2), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(n_pages=0), INVALID),
             (dict(Hkv=0), INVALID), (dict(page_size=0), INVALID), (dict(k_stride=64 * 32), INVALID), (dict(v_stride=0), INVALID),
             (dict(page_size=24), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED), (dict(page_size=2048), UNSUPPORTED),
             (dict(D=96), UNSUPPORTED), (dict(k=A + 8), UNSUPPORTED), (dict(n_pages=2 ** 28), UNSUPPORTED)]


def test_rotate_refusals():
    f = rmm.lib.rmm_qk_norm_rope

    def call(dtype=1, batch=2, L=4, D=128, q=heads(sb=8192), qo=heads(sb=8192), k=None, ko=None, gq=None, gk=None,
             eps=1e-6, r=rope(), pos=P, energy=None, ws=None, n=0):
        b = [None if x is None else ctypes.byref(x) for x in (q, qo, k, ko, r)]
        return f(dtype, batch, L, D, *b[:4], gq, gk, eps, b[4], pos, energy, ws, n, None)

    for kw, want in BAD_HEADS:
        assert call(q=heads(**kw)) == want and call(qo=heads(**kw)) == want
        assert call(k=heads(**kw), ko=heads()) == want and call(k=heads(), ko=heads(**kw)) == want
    for kw, want in BAD_ROPE:
        assert call(r=rope(**kw)) == want
    assert call(q=heads(sb=4)) == UNSUPPORTED
    assert call(dtype=0, q=heads(sb=8194)) == UNSUPPORTED
    assert call(dtype=5) == INVALID and call(batch=0) == INVALID and call(L=0) == INVALID and call(D=0) == INVALID
    assert call(q=None) == INVALID and call(qo=None) == INVALID and call(k=heads()) == INVALID
    assert call(q=None, qo=None) == INVALID and call(q=None, qo=None, k=heads(), ko=heads(), energy=P) == INVALID
    assert call(qo=heads(n=3)) == INVALID and call(pos=None) == INVALID
    for eps in (-1.0, float("nan"), float("inf")):
        assert call(eps=eps) == INVALID
    assert call(D=96) == UNSUPPORTED and call(batch=2 ** 20, L=2 ** 20) == UNSUPPORTED
    assert call(gq=ctypes.c_void_p(A + 2)) == UNSUPPORTED and call(energy=ctypes.c_void_p(A + 4)) == UNSUPPORTED
    need = rmm.rmm_qk_norm_rope_workspace_size(2, 4, 4000, 128)
    assert need > 0 and rmm.rmm_qk_norm_rope_workspace_size(2, 4, 1, 128) == 0
    assert call(L=4000, energy=P) == WS_SMALL and call(L=4000, energy=P, ws=P, n=need - 1) == WS_SMALL
    assert call(L=4000, energy=P, ws=ctypes.c_void_p(A + 4), n=need) == INVALID
    for bad in ((0, 4, 4, 128), (1, 0, 4, 128), (1, 4, 0, 128), (1, 4, 4, 96), (2 ** 20, 4, 2 ** 20, 128)):
        assert rmm.rmm_qk_norm_rope_workspace_size(*bad) == 0


def test_append_and_gather_refusals():
    f, g = rmm.lib.rmm_kv_append, rmm.lib.rmm_kv_gather

    def call(T=3, k=heads(), v=heads(), slots=P, c=cache(), gk=None, q=None, qo=None, gq=None, eps=1e-6, r=rope(), pos=P):
        b = [None if x is None else ctypes.byref(x) for x in (k, v, c, q, qo, r)]
        return f(T, b[0], b[1], slots, b[2], gk, b[3], b[4], gq, eps, b[5], pos, None)

    def back(c=cache(), slots=P, T=3, k=heads(), v=heads()):
        b = [None if x is None else ctypes.byref(x) for x in (c, k, v)]
        return g(b[0], slots, T, b[1], b[2], None)

    for kw, want in BAD_HEADS:
        assert call(k=heads(**kw)) == want and call(v=heads(**kw)) == want
        assert call(q=heads(**kw), qo=heads()) == want and call(q=heads(), qo=heads(**kw)) == want
        assert back(k=heads(**kw)) == want and back(v=heads(**kw)) == want
    for kw, want in BAD_ROPE:
        assert call(r=rope(**kw)) == want
    for kw, want in BAD_CACHE:
        assert call(c=cache(**kw)) == want and back(c=cache(**kw)) == want
    for kw, want in ((dict(k_scale=None), INVALID), (dict(v_scale=None), INVALID), (dict(k_scale_stride=64), INVALID),
                     (dict(v_scale=A + 4), UNSUPPORTED), (dict(v_scale_stride=64 * 4 + 8), UNSUPPORTED)):
        assert call(c=cache(mx=True, **kw)) == want and back(c=cache(mx=True, **kw)) == want
    assert call(T=0) == INVALID and call(k=None) == INVALID and call(v=None) == INVALID and call(slots=None) == INVALID
    assert call(c=None) == INVALID and call(q=heads()) == INVALID and call(qo=heads()) == INVALID
    assert call(k=heads(n=3)) == INVALID and call(v=heads(n=5)) == INVALID and call(q=heads(), qo=heads(n=5)) == INVALID
    assert call(eps=float("nan")) == INVALID and call(pos=None) == INVALID
    assert call(T=2 ** 31) == UNSUPPORTED and call(gk=ctypes.c_void_p(A + 8)) == UNSUPPORTED
    assert back(T=0) == INVALID and back(slots=None) == INVALID and back(c=None) == INVALID and back(k=heads(n=3)) == INVALID
    assert back(T=2 ** 30) == UNSUPPORTED


def test_attention_refusals():
    f = rmm.lib.rmm_paged_attention
    need = rmm.rmm_paged_attention_workspace_size(3, 3, 8, 4, 128)
    assert need > 0

    def call(T=3, q=heads(8), c=cache(), table=P, ld=5, width=5, lens=P, B=3, qs=None, idx=None, k=0, o=heads(8),
             ws=P, n=need):
        b = [None if x is None else ctypes.byref(x) for x in (q, c, o)]
        return f(T, b[0], b[1], table, ld, width, lens, B, qs, idx, k, 0.1, 1, b[2], ws, n, None)

    for kw, want in BAD_HEADS:
        kw = dict(dict(n=8), **kw)
        assert call(q=heads(**kw)) == want and call(o=heads(**kw)) == want
    for kw, want in BAD_CACHE:
        assert call(c=cache(**kw)) == want
    assert call(q=None) == INVALID and call(o=None) == INVALID and call(c=None) == INVALID
    assert call(table=None) == INVALID and call(lens=None) == INVALID
    assert call(T=0) == INVALID and call(B=0) == INVALID and call(width=0) == INVALID and call(ld=4) == INVALID
    assert call(T=4) == INVALID                       # no q_start: one token each
    assert call(q=heads(6), o=heads(6)) == INVALID and call(o=heads(4)) == INVALID
    assert call(idx=P, k=0) == INVALID and call(idx=P, k=129) == INVALID
    assert call(width=2 ** 27, ld=2 ** 27) == UNSUPPORTED and call(T=2 ** 29, qs=P) == UNSUPPORTED
    # 2^15 sequences of one token, 8 heads on 4 kv heads: 2^17 units of up to 2^13 blocks
    assert call(T=2 ** 15, B=2 ** 15, width=2 ** 14, ld=2 ** 14) == UNSUPPORTED
    assert call(T=2 ** 15, B=2 ** 15, width=2 ** 12, ld=2 ** 12, ws=None) == WS_SMALL
    assert call(table=ctypes.c_void_p(A + 2)) == UNSUPPORTED
    assert call(ws=None) == WS_SMALL and call(n=need - 1) == WS_SMALL
    assert call(ws=ctypes.c_void_p(A + 16)) == INVALID
    for bad in ((0, 1, 8, 4, 128), (1, 0, 8, 4, 128), (1, 1, 0, 4, 128), (1, 1, 8, 3, 128), (1, 1, 8, 4, 96),
                (2 ** 30, 1, 8, 4, 128)):
        assert rmm.rmm_paged_attention_workspace_size(*bad) == 0


def test_binding_refusals():
    """What the Python layer refuses before it calls the library (CPU tensors reach none of it)."""
    bf = torch.bfloat16
    with pytest.raises(ValueError, match="GPU"):
        rmm.kv_cache(2, 1, 16, 64, device="cpu")
    with pytest.raises(ValueError, match="GPU"):
        rmm.Rope(torch.zeros(4, 8), torch.zeros(4, 8))
    with pytest.raises(ValueError):
        rmm.Rope(torch.zeros(4, 8), torch.zeros(4, 4))
    with pytest.raises(TypeError):
        rmm.Rope(torch.zeros(4, 8, dtype=bf), torch.zeros(4, 8, dtype=bf))
    with pytest.raises(ValueError):
        rmm.rope_tables(4, 7, device="cpu")
    x = torch.zeros(2, 1, 16, 64, dtype=bf)
    u = torch.zeros(2, 1, 16, 32, dtype=torch.uint8)
    with pytest.raises(TypeError):
        rmm.KvCache(x, u)
    with pytest.raises(TypeError):
        rmm.KvCache(x.float(), x.float())
    with pytest.raises(ValueError):
        rmm.KvCache(x, x, u, u)
    with pytest.raises(ValueError):
        rmm.KvCache(u, u)
    with pytest.raises(ValueError):
        rmm.KvCache(u, u, u[..., :1], u[..., :2])
    with pytest.raises(ValueError, match="contiguous"):
        rmm.KvCache(x.transpose(2, 3).contiguous().transpose(2, 3), x)
    Q = torch.zeros(1, 3, 4, 64, dtype=bf)
    with pytest.raises(ValueError, match="GPU"):
        rmm.rmm_qk_norm_rope(Q, Q.transpose(1, 2))
    with pytest.raises(ValueError, match="positions"):
        rmm._positions(object(), None, 3)
    with pytest.raises(ValueError):
        rmm.rmm_qk_norm_rope(Q, Q)
    with pytest.raises(ValueError):
        rmm.rmm_qk_norm_rope(Q, Q.transpose(1, 2), K=Q)
    with pytest.raises(TypeError):
        rmm.rmm_qk_norm_rope(Q, Q.transpose(1, 2).float())


def test_rope_tables_in_float64():
    cos, sin = rmm.rope_tables(100001, 64, 500000.0, device="cpu")
    a = torch.arange(100001, dtype=torch.float64)[:, None] * 500000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)
    assert cos.dtype == torch.float32 and torch.equal(cos, a.cos().float()) and torch.equal(sin, a.sin().float())
