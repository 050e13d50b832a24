"""Attention over a paged cache (bf16 and 4-bit) against a float64 definition."""
import math

import numpy as np
import pytest
import torch

import paper_2608_13426_amd as rmm
from tests import cache_ref as cr
from tests.gpu_util import gpu, require_gpu

pytestmark = gpu


def _setup(dev, lens, news, H, Hkv, D, page, mx, seed, r=None, extra=0):
    """Cache (unused rows NaN), table, q_start, Q with `extra` rows behind the last sequence, idx."""
    g = torch.Generator(device=dev).manual_seed(seed)
    per = [-(-max(x, 0) // page) for x in lens]
    n_pages, width = sum(per) + 2, max(max(per), 1)
    order = torch.randperm(n_pages, device=dev, generator=g).int()
    table = torch.full((len(lens), width), -7, dtype=torch.int32, device=dev)     # unused entries are no pages
    at = 0
    for b, m in enumerate(per):
        table[b, :m] = order[at:at + m]
        at += m
    cache = rmm.kv_cache(n_pages, Hkv, page, D, mx=mx, device=dev)
    if mx:
        cache.k_scale.fill_(255)
        cache.v_scale.fill_(255)
    else:
        cache.k.fill_(float("nan"))
        cache.v.fill_(float("inf"))
    spread = torch.randn(Hkv, D, device=dev, generator=g).abs() + 0.1
    for b, L in enumerate(lens):
        if L <= 0:
            continue
        t = torch.arange(L, device=dev)
        slots = (table[b, t // page] * page + t % page).int()
        rmm.rmm_kv_append((torch.randn(L, Hkv, D, device=dev, generator=g) * spread).bfloat16(),
                          torch.randn(L, Hkv, D, device=dev, generator=g).bfloat16(), slots, cache)
    T = sum(news) + extra
    Q = torch.randn(T, H, D, device=dev, generator=g).bfloat16()
    q_start = torch.tensor(np.cumsum([0] + list(news)), dtype=torch.int32, device=dev)
    idx = None
    if r is not None:
        k = max(1, math.ceil(r * D))
        idx = torch.empty(T * H * k, dtype=torch.int32, device=dev)
        rmm.rmm_select_tokens(Q.view(T * H, D), k, idx)
        idx = idx.view(T, H, k)
    return cache, table, q_start, Q, idx


def _check(O, cache, table, lens, news, Q, scale, causal, idx):
    at = 0
    for b, (L, n) in enumerate(zip(lens, news)):
        if n:
            K, V = cr.history(cache, table, b, max(L, 0))
            want, bound = cr.attend(cr.np64(Q[at:at + n]), K, V, n, scale, causal,
                                    None if idx is None else idx[at:at + n].cpu().numpy())
            got = cr.np64(O[at:at + n])
            assert np.isfinite(got).all(), f"sequence {b}"
            assert np.all(np.abs(got - want) <= bound), f"sequence {b}: {np.max(np.abs(got - want) - bound)}"
        at += n


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("lens,news,H,Hkv,D,page,causal,r,scale", [
    ([1], [1], 1, 1, 64, 16, True, None, None),
    ([0, 1, 2, 15, 16, 17, 31, 32, 33, 64, 65], [1] * 11, 8, 2, 128, 16, True, None, None),   # ends inside pages and tiles
    ([129, 4, 300], [1] * 3, 6, 2, 64, 32, True, None, None),          # three heads per kv head
    ([1000], [1], 16, 1, 128, 64, True, None, None),                   # 16 heads per kv head, several workgroups
    ([500, 77], [1, 1], 24, 1, 128, 1024, True, None, None),           # 24: two row tiles
    ([700, 33], [1, 1], 40, 1, 64, 128, True, 0.5, None),              # 40: four
    ([5, 40, 3, 0, 90], [5, 2, 7, 3, 0], 8, 4, 128, 16, True, None, None),    # more new tokens than keys, none at all
    ([260, 31], [9, 30], 4, 2, 64, 32, True, 0.25, None),
    ([200, 50, 64], [3, 40, 1], 8, 8, 128, 32, False, None, None),     # not causal: lengths of their own
    ([150], [33], 10, 2, 128, 64, False, 0.5, -0.05),                  # negative scale
    ([90, 10], [4, 1], 4, 4, 128, 16, True, 1.0, 0.0),
    ([400], [2], 8, 2, 128, 32, True, None, 3.0),                      # peaked: the maximum rises several times
    ([20000], [1], 4, 1, 64, 64, True, None, None),                    # one unit over many workgroups
    ([130] * 70, [1] * 70, 4, 2, 64, 16, True, None, None),            # more sequences than lanes
    ([1 + 7 * (i % 29) for i in range(200)], [i % 3 for i in range(200)], 2, 1, 64, 16, True, None, None),
    ([600, 300], [200, 129], 4, 1, 64, 64, True, None, None),          # prompt chunks: 256-row tiles
    ([2500], [2500], 2, 1, 64, 32, True, None, None),                  # a whole prompt: 20 tiles in pairs, cut
    ([1300, 40], [1300, 1], 2, 1, 128, 16, True, None, None),          # 11 tiles: one without a partner
    ([700, 20], [33, 90], 4, 2, 128, 16, True, 0.5, None),             # more new tokens than keys, full and partial row tiles
    ([1500, 2100, 64], [70, 60, 1], 4, 4, 64, 64, False, None, None),
    ([300, 5], [80, 70], 6, 1, 128, 128, True, 0.25, -0.2),            # 256-row tiles with lists
    ([2200], [40], 1, 1, 128, 256, True, None, None),                  # 40 rows over many workgroups
])
def test_attention(lens, news, H, Hkv, D, page, causal, r, scale, mx):
    dev = require_gpu()
    cache, table, q_start, Q, idx = _setup(dev, lens, news, H, Hkv, D, page, mx, len(lens) * 1000 + D + page, r, extra=2)
    O = torch.full_like(Q, 3.0)
    length = torch.tensor(lens, dtype=torch.int32, device=dev)
    rmm.rmm_paged_attention(Q, cache, table, length, O, q_start=q_start, idx=idx, causal=causal, scale=scale)
    _check(O, cache, table, lens, news, Q, D ** -0.5 if scale is None else float(np.float32(scale)), causal, idx)
    assert bool((O[sum(news):] == 3.0).all())              # rows behind the last sequence
    O2 = torch.zeros_like(Q)
    rmm.rmm_paged_attention(Q, cache, table, length, O2, q_start=q_start, idx=idx, causal=causal, scale=scale)
    assert torch.equal(O2[:sum(news)], O[:sum(news)])
    if all(n == 1 for n in news):                          # one token each: no q_start needed
        T = len(news)
        rmm.rmm_paged_attention(Q[:T], cache, table, length, O2[:T], idx=None if idx is None else idx[:T].contiguous(),
                                causal=causal, scale=scale)
        # another T can mean other row tiles, so another order of the sums
        _check(O2, cache, table, lens, news, Q, D ** -0.5 if scale is None else float(np.float32(scale)), causal, idx)


@pytest.mark.parametrize("mx", [False, True])
def test_strided(mx):
    """Queries as a slice of projection rows, outputs of another layout, pages interleaved with
    another layer's, a table wider than used."""
    dev = require_gpu()
    lens, H, Hkv, D, page = [70, 133], 8, 2, 128, 16
    cache, table, _, Q, _ = _setup(dev, lens, [1, 1], H, Hkv, D, page, mx, 9)
    ts = [t for t in (cache.k, cache.v, cache.k_scale, cache.v_scale) if t is not None]
    wide = [torch.stack([torch.zeros_like(t), t], 1) for t in ts]
    rows = torch.randn(2, H + 2 * Hkv, D, device=dev).bfloat16()
    rows[:, :H] = Q
    O = torch.full((H, 2, D), 3.0, dtype=torch.bfloat16, device=dev)
    tab = torch.full((2, 40), 10 ** 6, dtype=torch.int32, device=dev)
    tab[:, :table.shape[1]] = table
    length = torch.tensor(lens, dtype=torch.int32, device=dev)
    rmm.rmm_paged_attention(rows[:, :H], rmm.KvCache(*(w[:, 1] for w in wide)), tab, length, O.transpose(0, 1))
    _check(O.transpose(0, 1), cache, table, lens, [1, 1], Q, D ** -0.5, True, None)
    R = rows.clone()                                       # in place
    rmm.rmm_paged_attention(R[:, :H], cache, table, length, R[:, :H])
    assert torch.equal(R[:, :H], O.transpose(0, 1)) and torch.equal(R[:, H:], rows[:, H:])


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("news,r", [([1, 1, 1], None), ([6, 9, 1], 0.5), ([45, 60, 20], None), ([700, 300, 1], 0.5)])
def test_in_place(news, r, mx):
    """o may be q: units kept whole, units cut over workgroups, and ones that are redone."""
    dev = require_gpu()
    lens, H, Hkv, D, page = [max(n, 40 + 700 * i) for i, n in enumerate(news)], 8, 2, 128, 32
    cache, table, q_start, Q, idx = _setup(dev, lens, news, H, Hkv, D, page, mx, 11, r=r)
    length = torch.tensor(lens, dtype=torch.int32, device=dev)
    last = (table[0, (lens[0] - 1) // page] * page + (lens[0] - 1) % page).view(1)
    bad = torch.full((1, Hkv, D), float("nan"), dtype=torch.bfloat16, device=dev)
    for redo in (False, True):
        if redo:
            rmm.rmm_kv_append(bad, bad, last, cache)
        O = torch.empty_like(Q)
        rmm.rmm_paged_attention(Q, cache, table, length, O, q_start=q_start, idx=idx)
        R = Q.clone()
        rmm.rmm_paged_attention(R, cache, table, length, R, q_start=q_start, idx=idx)
        assert torch.equal(R.view(torch.int16), O.view(torch.int16))
        assert redo == bool(O.isnan().any())


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("n", [2, 21, 40, 75])
def test_masked_nonfinite_keys_and_values(mx, n):
    """What a token does not see has no effect on it, infinite or NaN (but on the order of its sums)."""
    dev = require_gpu()
    L, H, Hkv, D, page = 75, 4, 2, 128, 16
    cache, table, q_start, Q, _ = _setup(dev, [L], [n], H, Hkv, D, page, mx, 3)
    bad = torch.full((1, Hkv, D), float("inf"), dtype=torch.bfloat16, device=dev)
    slot = (table[0, (L - 1) // page] * page + (L - 1) % page).view(1)
    rmm.rmm_kv_append(-bad, bad, slot, cache)              # the last token's key and value
    O2 = torch.empty_like(Q)
    rmm.rmm_paged_attention(Q, cache, table, torch.tensor([L], dtype=torch.int32, device=dev), O2, q_start=q_start)
    _check(O2[:n - 1], cache, table, [L - 1], [n - 1], Q[:n - 1], D ** -0.5, True, None)
    assert not O2[n - 1].isfinite().any()


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("news", [[3, 1], [20, 9], [45, 60]])
def test_lists_ignore_dropped_dims(news, mx):
    """Infinite and NaN key or query values in dims outside a list, and list entries that are no dims."""
    dev = require_gpu()
    lens, H, Hkv, D, page = [45, 200], 8, 2, 128, 32
    cache, table, q_start, Q, idx = _setup(dev, lens, news, H, Hkv, D, page, mx, 4, r=0.25)
    # lists without dims 64 .. 95, and those dims of some keys and queries infinite or NaN
    idx = (idx % 64).sort(-1).values.int().contiguous()
    Qd = Q.clone()
    Qd[:, ::2, 70] = float("nan")
    Qd[:, 1::2, 90] = float("inf")
    if mx:
        cache.k_scale[table[0, 0].long(), :, 3, 2] = 255
        cache.k_scale[table[1, 1].long(), :, 5:9, 2] = 255
    else:
        cache.k[table[0, 0].long(), :, 3, 70] = float("nan")
        cache.k[table[1, 1].long(), :, 5:9, 80] = float("-inf")
    O = torch.empty_like(Q)
    length = torch.tensor(lens, dtype=torch.int32, device=dev)
    rmm.rmm_paged_attention(Qd, cache, table, length, O, q_start=q_start, idx=idx)
    uniq = [[sorted(set(map(int, idx[t, h]))) for h in range(H)] for t in range(sum(news))]
    at = 0
    for b, (L, n) in enumerate(zip(lens, news)):
        K, V = cr.history(cache, table, b, L)
        for j in range(n):
            for h in range(H):
                I = uniq[at + j][h]
                g = h // (H // Hkv)
                want, bound = cr.attend(cr.np64(Q[at + j:at + j + 1, h:h + 1]), K[g:g + 1, :L - n + j + 1],
                                        V[g:g + 1, :L - n + j + 1], 1, D ** -0.5, True, np.array([[I]]))
                assert np.all(np.abs(cr.np64(O[at + j, h]) - want[0, 0]) <= bound[0, 0])
        at += n
    more = torch.cat([idx, torch.full_like(idx[..., :2], -1)], -1)
    more[..., -1] = D
    O2 = torch.empty_like(O)
    rmm.rmm_paged_attention(Qd, cache, table, length, O2, q_start=q_start, idx=more.contiguous())
    assert torch.equal(O, O2)


@pytest.mark.parametrize("mx", [False, True])
def test_bad_pages_and_lengths(mx):
    """A page number outside the cache, or a length past the table, makes that sequence NaN and no other."""
    dev = require_gpu()
    lens, H, Hkv, D, page = [70, 3000, 70, 70, 20], 4, 2, 64, 16
    cache, table, _, Q, _ = _setup(dev, lens, [1] * 5, H, Hkv, D, page, mx, 6)
    table = table[:, :190].contiguous()
    O = torch.empty_like(Q)
    length = torch.tensor(lens, dtype=torch.int32, device=dev)
    rmm.rmm_paged_attention(Q, cache, table, length, O)
    t2, l2 = table.clone(), length.clone()
    t2[0, 4], t2[1, 100], l2[2], l2[4] = cache.n_pages, -1, 190 * page + 1, -5
    t2[2] = t2[3, 0]
    O2 = torch.empty_like(Q)
    rmm.rmm_paged_attention(Q, cache, t2, l2, O2)
    assert O2[:3].isnan().all()
    assert torch.equal(O2[3], O[3]) and bool((O2[4] == 0).all())


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("n,D", [(30, 128), (70, 64), (300, 128)])
def test_bad_pages_of_prompts(n, D, mx):
    """The same with many new tokens: the tokens that see the page are NaN, other sequences as they were."""
    dev = require_gpu()
    lens, H, Hkv, page = [n, 3000, n, n, 20], 8, 4, 16
    cache, table, q_start, Q, _ = _setup(dev, lens, [n] * 5, H, Hkv, D, page, mx, 6)
    table = table[:, :190].contiguous()
    O = torch.empty_like(Q)
    t2, l2 = table.clone(), torch.tensor(lens, dtype=torch.int32, device=dev)
    t2[0, 1], t2[1, 100], l2[2], l2[4] = cache.n_pages, -1, 190 * page + 1, -5
    # (the same lengths: the order of the sums follows them)
    rmm.rmm_paged_attention(Q, cache, table, l2, O, q_start=q_start)
    O2 = torch.empty_like(Q)
    rmm.rmm_paged_attention(Q, cache, t2, l2, O2, q_start=q_start)
    o, o2 = O.split(n), O2.split(n)
    assert o2[0][page:].isnan().all() and o2[1].isnan().all() and o2[2].isnan().all()
    assert torch.equal(o2[3], o[3]) and bool((o2[4] == 0).all())


def test_q_start_past_the_tokens():
    """What q_start says past T is cut off; a descending step is an empty sequence."""
    dev = require_gpu()
    lens, H, Hkv, D, page = [40, 50, 60], 4, 2, 64, 16
    cache, table, _, Q, _ = _setup(dev, lens, [2, 2, 2], H, Hkv, D, page, False, 8)
    length = torch.tensor(lens, dtype=torch.int32, device=dev)
    O = torch.full_like(Q, 3.0)
    rmm.rmm_paged_attention(Q, cache, table, length, O, q_start=torch.tensor([0, 2, 1, 4], dtype=torch.int32, device=dev),
                            causal=False)
    # sequence 1 is empty; sequence 2 has rows 1 .. 3, row 1 also being sequence 0's
    assert bool((O[4:] == 3.0).all()) and O[:4].isfinite().all()
    O2 = torch.full_like(Q, 3.0)
    rmm.rmm_paged_attention(Q, cache, table, length, O2, q_start=torch.tensor([0, 2, 4, 100], dtype=torch.int32, device=dev),
                            causal=False)
    _check(O2, cache, table, lens, [2, 2, 2], Q, D ** -0.5, False, None)


def test_streams_and_graph_replay():
    """A side stream, two captured graphs that share a workspace, replays with other lengths."""
    dev = require_gpu()
    lens, H, Hkv, D, page = [700, 90, 1500], 8, 2, 128, 16
    cache, table, _, Q, _ = _setup(dev, lens, [1] * 3, H, Hkv, D, page, True, 12)
    length = torch.tensor(lens, dtype=torch.int32, device=dev)
    ws = torch.empty(rmm.rmm_paged_attention_workspace_size(3, 3, H, Hkv, D), dtype=torch.uint8, device=dev)
    want = [rmm.rmm_paged_attention(q, cache, table, length, torch.empty_like(Q)).clone() for q in (Q, Q.flip(0))]
    Qs = [Q.clone(), Q.flip(0).contiguous()]
    outs = [torch.zeros_like(Q) for _ in Qs]
    s = torch.cuda.Stream(dev)
    s.wait_stream(torch.cuda.current_stream(dev))
    rmm.rmm_paged_attention(Qs[0], cache, table, length, outs[0], workspace=ws, stream=s)
    s.synchronize()
    assert torch.equal(outs[0], want[0])
    graphs = []
    for q, o in zip(Qs, outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            rmm.rmm_paged_attention(q, cache, table, length, o, workspace=ws)
        graphs.append(graph)
    for rep in range(3):
        for o in outs:
            o.zero_()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])
    length.copy_(torch.tensor([31, 90, 2], dtype=torch.int32))
    graphs[0].replay()
    eager = rmm.rmm_paged_attention(Qs[0], cache, table, length, torch.empty_like(Q))
    torch.cuda.synchronize()
    assert torch.equal(outs[0], eager) and not torch.equal(outs[0], want[0])
