"""A reduced layer's ends as a program runs them: the join, products with epilogues,
the output projection's log probabilities -- a prompt and decode steps, eager and
as a captured graph, each stage against its float64 form on the stage's own inputs."""
import math

import pytest
import torch

import paper_2608_13426_amd as rmm
from tests import block_ref as ref
from tests.gpu_util import gpu, require_gpu

pytestmark = gpu
BF, I32, F64 = torch.bfloat16, torch.int32, torch.float64
K, F, V = 256, 640, 1003
k1, k2 = rmm.rmm_retained_count(0.5, K), rmm.rmm_retained_count(0.5, F)


def weights(dev):
    g = torch.Generator(device=dev).manual_seed(11)
    rnd = lambda *s: torch.randn(*s, device=dev, generator=g)  # noqa: E731
    head = torch.zeros(K, 1008, dtype=BF, device=dev)[:, :V]
    head.copy_(0.1 * rnd(K, V))
    return dict(up=(0.1 * rnd(K, F)).to(BF), bu=rnd(F).to(BF), down=(0.1 * rnd(F, K)).to(BF), bd=rnd(K).to(BF), head=head,
                g1=(1 + 0.1 * rnd(K)).to(BF), g2=(1 + 0.1 * rnd(K)).to(BF), g3=(1 + 0.1 * rnd(K)).to(BF),
                gate=(0.5 + 0.1 * rnd(K)).to(BF))


def near(got, want):
    y, tol = want
    err = (got.double() - y).abs()
    assert bool((err <= tol).all()), f"worst {float((err / tol).max())} of the bound"


class Prompt:
    """Buffers of one prompt's pass; R is the residual stream, updated in place."""

    def __init__(self, dev, M):
        e = lambda *s, dtype=BF: torch.empty(*s, dtype=dtype, device=dev)  # noqa: E731
        self.M, ld = M, (M + 7) // 8 * 8
        self.R, self.H = e(1, M, K), e(1, M, K)
        self.Xt, self.e1 = torch.zeros(1, K, ld, dtype=BF, device=dev)[:, :, :M], e(K, dtype=F64)
        self.i1, self.U = e(1, k1, dtype=I32), e(1, M, F)
        self.Ut, self.e2 = torch.zeros(1, F, ld, dtype=BF, device=dev)[:, :, :M], e(F, dtype=F64)
        self.i2, self.D = e(1, k2, dtype=I32), e(1, M, K)
        self.X, self.i3, self.Z = e(1, M, K), e(M, k1, dtype=I32), e(M, 1, 1008)
        self.tok = torch.zeros(M, dtype=I32, device=dev)
        self.lp, self.en = e(M, dtype=torch.float32), e(M, dtype=torch.float32)
        self.ti, self.tl = e(M, 5, dtype=I32), e(M, 5, dtype=torch.float32)
        u8 = lambda n: torch.empty(max(n, 1), dtype=torch.uint8, device=dev)  # noqa: E731
        self.wj, self.ws = u8(rmm.rmm_block_join_workspace_size(1, M, K)), u8(rmm.rmm_workspace_size(rmm.RMM_OP_SCORE, 1, M, F))
        self.wl, self.wg = u8(rmm.rmm_token_logprobs_workspace_size(M, V, 5)), u8(rmm.rmm_gemv_workspace_size(M, 1, V, k1))

    def run(self, w):
        rmm.rmm_block_join(None, self.R, self.H, Xt=self.Xt, energy=self.e1, pre_gamma=w["g1"], workspace=self.wj)
        rmm.rmm_select(self.e1, k1, self.i1)
        rmm.rmm_reduced_gemm_kmajor_epilogue(self.Xt, w["up"], self.i1, self.U, bias=w["bu"], act="gelu")
        rmm.rmm_score_kmajor(self.U, self.e2, self.Ut, self.ws)
        rmm.rmm_select(self.e2, k2, self.i2)
        rmm.rmm_reduced_gemm_kmajor_epilogue(self.Ut, w["down"], self.i2, self.D, bias=w["bd"])
        rmm.rmm_block_join(self.D, self.H, self.H, X=self.X, post_norm=True, post_gamma=w["g2"], gate=w["gate"],
                           pre_gamma=w["g3"], workspace=self.wj)
        x = self.X.view(self.M, 1, K)
        rmm.rmm_select_tokens(x, k1, self.i3)
        rmm.rmm_reduced_gemv_epilogue(x, w["head"], self.i3, self.Z[:, :, :V], workspace=self.wg)
        rmm.rmm_token_logprobs(self.Z[:, 0, :V], tokens=self.tok, logp=self.lp, entropy=self.en, top_idx=self.ti,
                               top_logp=self.tl, workspace=self.wl)

    def outputs(self):
        return [t.clone() for t in (self.H, self.X, self.i1, self.i2, self.Z[:, :, :V], self.lp, self.en, self.ti, self.tl)]


@pytest.mark.parametrize("M", [1, 5, 77, 300])
def test_prompt_stage_by_stage(M):
    dev = require_gpu()
    w, p = weights(dev), Prompt(dev, M)
    p.R.normal_()
    p.R[..., :3] *= 20
    p.run(w)
    near(p.Xt.transpose(1, 2), ref.normed(p.R, w["g1"], 1e-6, BF))
    near(p.U, ref.product(p.Xt.transpose(1, 2), w["up"], p.i1, w["bu"], "gelu", None, 1.0, BF))
    assert torch.equal(p.Ut.transpose(1, 2), p.U)
    near(p.D, ref.product(p.U, w["down"], p.i2, w["bd"], None, None, 1.0, BF))
    near(p.H, ref.join(p.D, p.R, True, w["g2"], w["gate"], 1.0, 1e-6, BF))
    near(p.X, ref.normed(p.H, w["g3"], 1e-6, BF))
    near(p.Z[:, :, :V], ref.product(p.X.view(M, 1, K), w["head"], p.i3, None, None, None, 1.0, BF))
    z = p.Z[:, 0, :V]
    lp, ent, tol, etol = ref.logprobs(z, 1.0)
    assert bool(((p.lp.double() - lp[:, 0]).abs() <= tol[:, 0]).all())
    assert bool(((p.en.double() - ent).abs() <= etol).all())
    assert torch.equal(p.ti.long(), ref.top_tokens(z, 5))


class Step:
    """One decode step of B sequences: the few-row forms, the stream in place."""

    def __init__(self, dev, B):
        e = lambda *s, dtype=BF: torch.empty(*s, dtype=dtype, device=dev)  # noqa: E731
        self.B, self.R0, self.R = B, e(B, 1, K), e(B, 1, K)
        self.X, self.U, self.i1, self.i2 = e(B, 1, K), e(B, 1, F), e(B, k1, dtype=I32), e(B, k2, dtype=I32)
        self.Z, self.ti, self.tl = e(B, 1, V), e(B, 3, dtype=I32), e(B, 3, dtype=torch.float32)
        u8 = lambda n: torch.empty(max(n, 1), dtype=torch.uint8, device=dev)  # noqa: E731
        self.wg = u8(max(rmm.rmm_gemv_workspace_size(B, 1, n, k) for n, k in ((F, k1), (K, k2), (V, k1))))
        self.wl = u8(rmm.rmm_token_logprobs_workspace_size(B, V, 3))

    def run(self, w):
        self.R.copy_(self.R0)
        rmm.rmm_block_join(None, self.R, X=self.X, pre_gamma=w["g1"])
        rmm.rmm_select_tokens(self.X, k1, self.i1)
        rmm.rmm_reduced_gemv_epilogue(self.X, w["up"], self.i1, self.U, bias=w["bu"], act="silu", workspace=self.wg)
        rmm.rmm_select_tokens(self.U, k2, self.i2)
        rmm.rmm_reduced_gemv_epilogue(self.U, w["down"], self.i2, self.R, bias=w["bd"], residual=self.R, workspace=self.wg)
        rmm.rmm_block_join(None, self.R, X=self.X, pre_gamma=w["g3"])
        rmm.rmm_select_tokens(self.X, k1, self.i1)
        rmm.rmm_reduced_gemv_epilogue(self.X, w["head"], self.i1, self.Z, workspace=self.wg)
        rmm.rmm_token_logprobs(self.Z[:, 0], top_idx=self.ti, top_logp=self.tl, workspace=self.wl)

    def outputs(self):
        return [t.clone() for t in (self.R, self.X, self.Z, self.ti, self.tl)]


@pytest.mark.parametrize("make", [lambda d: Prompt(d, 200), lambda d: Step(d, 1), lambda d: Step(d, 13)], ids=["prompt", "one", "batch"])
def test_captured_and_replayed(make):
    """Replays on new inputs, between eager work and synchronizations, give the eager results."""
    dev = require_gpu()
    w = weights(dev)
    eager, held = make(dev), make(dev)
    inp = lambda p: p.R0 if isinstance(p, Step) else p.R  # noqa: E731
    s = torch.cuda.Stream()
    inp(held).normal_()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        held.run(w)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held.run(w)
    for i in range(4):
        x = torch.randn(inp(held).shape, device=dev).to(BF)
        inp(held).copy_(x)
        inp(eager).copy_(x)
        graph.replay()
        if i % 2:
            torch.cuda.synchronize()
        eager.run(w)
        torch.cuda.synchronize()
        for a, b in zip(held.outputs(), eager.outputs()):
            assert torch.equal(a, b)


def test_two_calls_at_once_on_streams_of_their_own():
    dev = require_gpu()
    w = weights(dev)
    runs = [Prompt(dev, 300), Prompt(dev, 300), Step(dev, 13), Step(dev, 13)]
    for r in runs:
        (r.R0 if isinstance(r, Step) else r.R).normal_()
    runs[1].R.copy_(runs[0].R)
    runs[3].R0.copy_(runs[2].R0)
    streams = [torch.cuda.Stream() for _ in runs]
    torch.cuda.synchronize()
    for _ in range(3):
        for r, s in zip(runs, streams):
            with torch.cuda.stream(s):
                r.run(w)
    torch.cuda.synchronize()
    for a, b in ((0, 1), (2, 3)):
        for x, y in zip(runs[a].outputs(), runs[b].outputs()):
            assert torch.equal(x, y)


def test_scratch_of_the_binding_on_a_given_stream():
    """Calls that bring no workspace, on a stream other than the current one."""
    dev = require_gpu()
    w, s = weights(dev), torch.cuda.Stream()
    z = torch.randn(2, 40000, device=dev)
    X = torch.randn(2, 3, K, device=dev).to(BF)
    i = torch.arange(k1, dtype=I32, device=dev).repeat(2, 1)
    outs = []
    torch.cuda.synchronize()
    for st in (None, s):
        en, Y = torch.empty(2, device=dev), torch.empty(2, 3, V, dtype=BF, device=dev)
        H, Xt = torch.empty_like(X), torch.zeros(2, K, 8, dtype=BF, device=dev)[:, :, :3]
        e = torch.empty(2 * K, dtype=F64, device=dev)
        torch.cuda.synchronize()
        rmm.rmm_token_logprobs(z, entropy=en, stream=st)
        rmm.rmm_reduced_gemv_epilogue(X, w["head"], i, Y, act="silu", stream=st)
        rmm.rmm_block_join(X, X, H, Xt=Xt, energy=e, stream=st)
        torch.cuda.synchronize()
        outs.append((en, Y, H, Xt, e))
    assert all(torch.equal(a, b) for a, b in zip(*outs)) and math.isfinite(float(outs[0][0][0]))
