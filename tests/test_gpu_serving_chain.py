"""The cache operators together with the reduced products, as a serving program
runs them: a prompt into the cache, then decode steps, eager and captured."""
import numpy as np
import pytest
import torch

import paper_2608_13426_amd as rmm
from oracle import rmm_oracle as ro
from tests import cache_ref as cr
from tests.gpu_util import attention_bound, gpu, require_gpu

pytestmark = gpu

H, HKV, D, HIDDEN, PAGE = 8, 2, 128, 512, 16
ROW = (H + 2 * HKV) * D


def _weights(dev):
    g = torch.Generator(device=dev).manual_seed(3)
    W = (0.05 * torch.randn(HIDDEN, ROW, device=dev, generator=g)).bfloat16()
    Wo = (0.05 * torch.randn(H * D, HIDDEN, device=dev, generator=g)).bfloat16()
    gammas = [(1 + 0.1 * torch.randn(D, device=dev, generator=g)).bfloat16() for _ in range(2)]
    return W, Wo, gammas, rmm.Rope(*rmm.rope_tables(512, D, device=dev)), g


@pytest.mark.parametrize("L", [67, 300])
def test_prompt(L):
    """Projection, norm and rotation with energies, selection, reduced attention; the same prompt
    through the cache gives the same attention within the bounds of both."""
    dev = require_gpu()
    W, _, (gq, gk), rope, g = _weights(dev)
    X = torch.randn(1, L, HIDDEN, device=dev, generator=g).bfloat16()
    rows = torch.empty(1, L, ROW, dtype=torch.bfloat16, device=dev)
    rmm.rmm_linear(X, W, 0.5, rows)
    heads = rows.view(1, L, H + 2 * HKV, D)
    Q = torch.empty(1, H, L, D, dtype=torch.bfloat16, device=dev)
    K = torch.empty(1, HKV, L, D, dtype=torch.bfloat16, device=dev)
    e = torch.empty(H * D, dtype=torch.float64, device=dev)
    pos = torch.arange(L, dtype=torch.int32, device=dev)
    rmm.rmm_qk_norm_rope(heads[:, :, :H], Q, pos, rope, K=heads[:, :, H:H + HKV], Ko=K, gamma_q=gq, gamma_k=gk, energy=e)
    k = rmm.rmm_retained_count(0.5, D)
    idx = torch.empty(1, H, k, dtype=torch.int32, device=dev)
    rmm.rmm_select(e, k, idx)
    e2 = torch.empty_like(e)
    rmm.rmm_score(Q[0], e2, torch.empty(max(1, rmm.rmm_workspace_size(rmm.RMM_OP_SCORE, H, L, D)), dtype=torch.uint8,
                                        device=dev))
    assert torch.equal(rmm.rmm_select(e2, k, torch.empty_like(idx)), idx)
    V = heads[:, :, H + HKV:].transpose(1, 2).contiguous()
    O = torch.empty_like(Q)
    rmm.rmm_reduced_attention(Q, K, V, idx, O)
    # into a cache of scattered pages: raw keys rotated on the way are the rotated ones
    n_pages = -(-L // PAGE) + 5
    table = torch.randperm(n_pages, device=dev, generator=g)[:-(-L // PAGE)].int().view(1, -1)
    slots = (table[0, pos.long() // PAGE] * PAGE + pos % PAGE).int()
    cache = rmm.kv_cache(n_pages, HKV, PAGE, D, device=dev)
    rmm.rmm_kv_append(heads[0, :, H:H + HKV], heads[0, :, H + HKV:], slots, cache, positions=pos, rope=rope, gamma_k=gk)
    Kr, Vr = torch.empty_like(K), torch.empty_like(V)
    rmm.rmm_kv_gather(cache, slots, Kr[0].transpose(0, 1), Vr[0].transpose(0, 1))
    assert torch.equal(Kr, K) and torch.equal(Vr, V)
    Oc = torch.empty(L, H, D, dtype=torch.bfloat16, device=dev)
    lists = idx.expand(L, H, k).contiguous()
    rmm.rmm_paged_attention(Q[0].transpose(0, 1), cache, table, torch.tensor([L], dtype=torch.int32, device=dev), Oc,
                            q_start=torch.tensor([0, L], dtype=torch.int32, device=dev), idx=lists)
    q, kk, v, I = cr.np64(Q[0]), cr.np64(K[0]), cr.np64(V[0]), idx[0].cpu().numpy()
    ref = ro.reduced_attention(q, kk, v, I, True)
    bound = attention_bound(q, kk, v, I, True, D ** -0.5)[:, :, None] + 2.0 ** -8 * np.abs(ref)
    assert np.all(np.abs(cr.np64(O[0]) - ref) <= bound)
    assert np.all(np.abs(cr.np64(Oc).transpose(1, 0, 2) - ref) <= bound)


@pytest.mark.parametrize("mx", [False, True])
def test_decode_steps(mx):
    """Steps of a batch in which a sequence is idle: projections of the tokens' own sets, append with
    the rotation, selection on the rotated queries, attention over the cache, output projection."""
    dev = require_gpu()
    W, Wo, (gq, gk), rope, g = _weights(dev)
    B, k = 5, rmm.rmm_retained_count(0.5, HIDDEN)
    ko, kq = rmm.rmm_retained_count(0.5, H * D), rmm.rmm_retained_count(0.75, D)
    start = [0, 15, 33, 100, 0]                        # keys before the first step; the last sequence is idle
    width = 9
    table = torch.randperm(B * width, device=dev, generator=g).int().view(B, width)

    def fill(cache):
        gg = torch.Generator(device=dev).manual_seed(8)
        for b, L in enumerate(start):
            if L:
                t = torch.arange(L, device=dev)
                kv = torch.randn(2, L, HKV, D, device=dev, generator=gg).bfloat16()
                rmm.rmm_kv_append(kv[0], kv[1], (table[b, t // PAGE] * PAGE + t % PAGE).int(), cache)

    def program(cache):
        """(inputs, outputs, the step on them)"""
        bf = dict(dtype=torch.bfloat16, device=dev)
        i32 = dict(dtype=torch.int32, device=dev)
        s = dict(X=torch.zeros(B, HIDDEN, **bf), rows=torch.zeros(B, ROW, **bf), Q=torch.zeros(B, H, D, **bf),
                 O=torch.zeros(B, H, D, **bf), Y=torch.zeros(B, HIDDEN, **bf), pos=torch.zeros(B, **i32),
                 slots=torch.zeros(B, **i32), lens=torch.zeros(B, **i32), i1=torch.zeros(B * k, **i32),
                 iq=torch.zeros(B, H, kq, **i32), io=torch.zeros(B * ko, **i32))
        g1, g2 = [(s["X"], W, k, s["i1"], s["rows"])], [(s["O"].view(B, H * D), Wo, ko, s["io"], s["Y"])]
        ws1, ws2 = (torch.empty(rmm.rmm_decode_products_shared_workspace_size(x), dtype=torch.uint8, device=dev)
                    for x in (g1, g2))
        wsa = torch.empty(rmm.rmm_paged_attention_workspace_size(B, B, H, HKV, D), dtype=torch.uint8, device=dev)
        heads = s["rows"].view(B, H + 2 * HKV, D)

        def step():
            rmm.rmm_decode_step_shared(g1, workspace=ws1)
            rmm.rmm_kv_append(heads[:, H:H + HKV], heads[:, H + HKV:], s["slots"], cache, positions=s["pos"], rope=rope,
                              gamma_k=gk, Q=heads[:, :H], Qo=s["Q"], gamma_q=gq)
            rmm.rmm_select_tokens(s["Q"].view(B * H, D), kq, s["iq"])
            rmm.rmm_paged_attention(s["Q"], cache, table, s["lens"], s["O"], idx=s["iq"], workspace=wsa)
            rmm.rmm_decode_step_shared(g2, workspace=ws2)
        return s, step

    def feed(s, n):
        gg = torch.Generator(device=dev).manual_seed(20 + n)
        s["X"].copy_(torch.randn(B, HIDDEN, device=dev, generator=gg))
        at = torch.tensor([x + n for x in start], device=dev)
        s["pos"].copy_(at)
        s["lens"].copy_(at + 1)
        s["slots"].copy_(table[torch.arange(B, device=dev), at // PAGE] * PAGE + at % PAGE)
        s["slots"][B - 1], s["lens"][B - 1], s["pos"][B - 1] = -1, 0, 0

    caches = [rmm.kv_cache(B * width, HKV, PAGE, D, mx=mx, device=dev) for _ in range(2)]
    for c in caches:
        fill(c)
    (s, step), (sg, stepg) = program(caches[0]), program(caches[1])
    feed(sg, 0)
    warm = torch.cuda.Stream(dev)
    warm.wait_stream(torch.cuda.current_stream(dev))
    with torch.cuda.stream(warm):
        stepg()
    torch.cuda.current_stream(dev).wait_stream(warm)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        stepg()
    for n in range(4):
        feed(s, n)
        step()
        feed(sg, n)
        graph.replay()
        torch.cuda.synchronize()
        for name in ("Q", "O", "Y", "iq", "io"):
            assert torch.equal(s[name], sg[name]), (n, name)
        # each stage from the GPU's own inputs of it
        rows = cr.np64(s["rows"]).reshape(B, H + 2 * HKV, D)
        pos = s["pos"].cpu().numpy()
        tab = (cr.np64(rope.cos), cr.np64(rope.sin))
        want = cr.bf16(cr.rotate_f32(rows[:, :H], cr.np64(gq), pos, *tab, False))
        assert np.array_equal(cr.np64(s["Q"]), want)
        newk = cr.rotate_f32(rows[:, H:H + HKV], cr.np64(gk), pos, *tab, False)
        newv = rows[:, H + HKV:]
        Q, O, iq = cr.np64(s["Q"]), cr.np64(s["O"]), s["iq"].cpu().numpy()
        for b in range(B - 1):
            K, V = cr.history(caches[0], table, b, start[b] + n + 1)
            assert np.array_equal(K[:, -1], cr.mx_round(newk[b]) if mx else cr.bf16(newk[b]))
            assert np.array_equal(V[:, -1], cr.mx_round(newv[b]) if mx else newv[b])
            for h in range(H):
                assert np.array_equal(iq[b, h], ro.topk_indices(Q[b, h] ** 2, kq))
            ref, bound = cr.attend(Q[b:b + 1], K, V, 1, D ** -0.5, True, iq[b:b + 1])
            assert np.all(np.abs(O[b:b + 1] - ref) <= bound)
        assert not O[B - 1].any()
        io = s["io"].view(B, ko).cpu().numpy()
        Y, X, Wf = cr.np64(s["Y"]), O.reshape(B, H * D), cr.np64(Wo)
        for b in range(B):
            assert np.array_equal(io[b], ro.topk_indices(X[b] ** 2, ko))
            ref = X[b, io[b]] @ Wf[io[b]]
            tol = 2.0 ** -8 * np.abs(ref) + (ko + 2) * 2.0 ** -24 * (np.abs(X[b, io[b]]) @ np.abs(Wf[io[b]])) * (1 + 2.0 ** -8)
            assert np.all(np.abs(Y[b] - ref) <= tol)
