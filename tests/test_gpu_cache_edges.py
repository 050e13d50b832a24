"""Rotation, appending and reading back at the edges of what the cache entry points take."""
import pytest
import torch

import paper_2608_13426_amd as rmm
from tests.gpu_util import gpu, require_gpu

pytestmark = gpu


def test_rotate_more_entries_than_a_grid():
    """2^24 + 5 sequences of one token with energies, a workgroup each (2^32 threads and more): as
    the same tokens in short calls."""
    dev = require_gpu()
    batch, D = 2 ** 24 + 5, 64
    Q = torch.empty(batch, 1, 1, D, dtype=torch.bfloat16, device=dev)
    Q.view(torch.int16).random_(-30000, 30000)
    Q[~Q.isfinite()] = 1.0
    pos = torch.arange(batch, device=dev).remainder(100).int()
    rope = rmm.Rope(*rmm.rope_tables(100, D, device=dev))
    Qo = torch.zeros_like(Q)
    e = torch.zeros(batch, D, dtype=torch.float64, device=dev)
    rmm.rmm_qk_norm_rope(Q, Qo, pos, rope, energy=e)
    for at in (0, 2 ** 22 - 500, 2 ** 23 - 500, 2 ** 24 - 500, batch - 1000):
        s = slice(at, at + 1000)
        o, f = torch.empty_like(Q[s]), torch.empty_like(e[s])
        rmm.rmm_qk_norm_rope(Q[s], o, pos[s].contiguous(), rope, energy=f.view(-1))
        assert torch.equal(Qo[s], o) and torch.equal(e[s], f)
        assert torch.equal(f, o.view(-1, D).double().square())


def test_same_slot_twice_with_other_scales():
    """In a 4-bit cache every 8 codes and every scale byte of a slot named twice are one of its
    tokens'; other slots are as they should be."""
    dev = require_gpu()
    Hkv, D, T = 2, 128, 6
    g = torch.Generator(device=dev).manual_seed(5)
    x = torch.randn(T, Hkv, D, device=dev, generator=g)
    x = (x * 2.0 ** (3 * torch.arange(T, device=dev))[:, None, None]).bfloat16()
    alone = rmm.kv_cache(1, Hkv, 16, D, mx=True, device=dev)
    rmm.rmm_kv_append(x, x, torch.arange(T, dtype=torch.int32, device=dev), alone)
    assert alone.k_scale[0, :, :T].unique().numel() >= T
    cache = rmm.kv_cache(1, Hkv, 16, D, mx=True, device=dev)
    rmm.rmm_kv_append(x, x, torch.tensor([3, 9, 3, 3, 11, 3], dtype=torch.int32, device=dev), cache)
    for t, s in ((cache.k, alone.k), (cache.v, alone.v), (cache.k_scale, alone.k_scale), (cache.v_scale, alone.v_scale)):
        n = 4 if t.shape[-1] == D // 2 else 1              # bytes of a piece
        assert torch.equal(t[0, :, 9], s[0, :, 1]) and torch.equal(t[0, :, 11], s[0, :, 4])
        got, of = t[0, :, 3].view(Hkv, 1, -1, n), s[0][:, [0, 2, 3, 5]].view(Hkv, 4, -1, n)
        assert (got == of).all(-1).any(1).all()
        rest = torch.ones(16, dtype=torch.bool, device=dev)
        rest[[3, 9, 11]] = False
        assert bool((t[0][:, rest] == 0).all())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rotate_keys_alone(dtype):
    """Keys without queries: as beside them, in place too."""
    dev = require_gpu()
    g = torch.Generator(device=dev).manual_seed(4)
    Q, K = (torch.randn(2, 37, n, 128, device=dev, generator=g).to(dtype) for n in (6, 3))
    rope = rmm.Rope(*rmm.rope_tables(100, 128, device=dev))
    pos = torch.arange(74, dtype=torch.int32, device=dev)
    gk = torch.randn(128, device=dev, generator=g).to(dtype)
    Qo, Ko, Ka = (torch.empty(2, n, 37, 128, dtype=dtype, device=dev) for n in (6, 3, 3))
    rmm.rmm_qk_norm_rope(Q, Qo, pos, rope, K=K, Ko=Ko, gamma_k=gk)
    assert rmm.rmm_qk_norm_rope(None, None, pos, rope, K=K, Ko=Ka, gamma_k=gk) is Ka
    assert torch.equal(Ka, Ko)
    rmm.rmm_qk_norm_rope(None, None, pos, rope, K=K, Ko=K.transpose(1, 2), gamma_k=gk)
    assert torch.equal(K.transpose(1, 2), Ko)


@pytest.mark.parametrize("mx", [False, True])
def test_calls_on_two_streams_at_once(mx):
    """Calls that allocate their own workspaces, in turn on the current stream and on another one,
    with nothing between them to wait for: cut units, whose pieces pass through the workspace."""
    dev = require_gpu()
    lens, H, Hkv, D, page = [9000, 300, 4000], 8, 2, 128, 16
    g = torch.Generator(device=dev).manual_seed(6)
    per = -(-max(lens) // page)
    cache = rmm.kv_cache(3 * per, Hkv, page, D, mx=mx, device=dev)
    table = torch.arange(3 * per, dtype=torch.int32, device=dev).view(3, per)
    for b, L in enumerate(lens):
        kv = [torch.randn(L, Hkv, D, device=dev, generator=g).bfloat16() for _ in range(2)]
        rmm.rmm_kv_append(*kv, torch.arange(L, dtype=torch.int32, device=dev) + b * per * page, cache)
    length = torch.tensor(lens, dtype=torch.int32, device=dev)
    Qs = torch.randn(8, 3, H, D, device=dev, generator=g).bfloat16()
    want = torch.stack([rmm.rmm_paged_attention(q, cache, table, length, torch.empty_like(q)) for q in Qs])
    L = 2000
    X = torch.randn(8, 1, L, H, D, device=dev, generator=g).bfloat16()
    e = torch.zeros(8, H * D, dtype=torch.float64, device=dev)
    for x, f in zip(X, e):
        rmm.rmm_qk_norm_rope(x, torch.empty(1, H, L, D, dtype=x.dtype, device=dev), energy=f)
    s = torch.cuda.Stream(dev)
    for _ in range(3):
        O, E = torch.zeros_like(want), torch.zeros_like(e)
        Xo = torch.empty(8, 1, H, L, D, dtype=X.dtype, device=dev)
        torch.cuda.synchronize()
        for i in range(8):
            st = s if i % 2 else None
            rmm.rmm_qk_norm_rope(X[i], Xo[i], energy=E[i], stream=st)
            rmm.rmm_paged_attention(Qs[i], cache, table, length, O[i], stream=st)
        torch.cuda.synchronize()
        assert torch.equal(O, want) and torch.equal(E, e)
