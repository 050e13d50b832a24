"""Host-side checks of the products with an epilogue, the join and the token log
probabilities: only calls that are refused before any HIP call are made here."""
import ctypes
import math

import pytest
import torch

import paper_2608_13426_amd as rmm
from paper_2608_13426_amd import _block

INVALID, UNSUPPORTED, WS_SMALL = 1, 2, 3
A = 0x100000                           # an aligned address that is never dereferenced
P = ctypes.c_void_p(A)


def at(off):
    return ctypes.c_void_p(A + off)


def ep(**kw):
    d = dict(bias=A, act=0, residual_scale=1.0, residual=A + 4096, ldr=64)
    d.update(kw)
    return ctypes.byref(_block._EpilogueC(*d.values()))


BAD_EPILOGUES = [(dict(act=5), INVALID), (dict(act=-1), INVALID), (dict(ldr=63), INVALID), (dict(residual_scale=math.nan), INVALID),
                 (dict(residual_scale=math.inf), INVALID), (dict(bias=A + 1), INVALID), (dict(residual=A + 1), INVALID),
                 (dict(residual=A, ldr=72), INVALID)]


def forms():
    """Each product's call with one argument replaced; Y is A."""
    def gemm(e=None, dtype=1, **kw):
        d = dict(X=P, W=P, idx=P, dtype=dtype, B=1, M=64, N=64, K=128, k=32, ldx=128, ldw=64, Y=P, ldy=64)
        d.update(kw)
        return rmm.lib.rmm_reduced_gemm_epilogue(*d.values(), e, None)

    def kmajor(e=None, **kw):
        d = dict(Xt=P, W=P, idx=P, B=1, M=64, N=64, K=128, k=32, ldxt=64, ldw=64, Y=P, ldy=64)
        d.update(kw)
        return rmm.lib.rmm_reduced_gemm_kmajor_epilogue(*d.values(), e, None)

    def gemv(e=None, ws=P, n=1 << 30, **kw):
        d = dict(X=P, W=P, idx=P, B=1, M=4, N=64, K=4096, k=2048, ldx=4096, ldw=64, Y=P, ldy=64)
        d.update(kw)
        return rmm.lib.rmm_reduced_gemv_epilogue(*d.values(), e, ws, n, None)

    return gemm, kmajor, gemv


def test_product_refusals():
    gemm, kmajor, gemv = forms()
    for f in (gemm, kmajor, gemv):
        for kw in (dict(W=None), dict(idx=None), dict(Y=None), dict(B=0), dict(M=0), dict(N=0), dict(K=0), dict(k=0),
                   dict(k=10 ** 6), dict(ldw=63), dict(ldy=63), dict(N=2 ** 31, ldw=2 ** 31, ldy=2 ** 31)):
            assert f(ep(), **kw) == INVALID, (f, kw)
        for kw, want in BAD_EPILOGUES:
            assert f(ep(**kw)) == want, (f, kw)
        assert f(ep(), B=65536) == UNSUPPORTED
    assert gemm(ep(), X=None) == INVALID and gemm(ep(), ldx=127) == INVALID and gemm(ep(), dtype=2) == INVALID
    assert gemm(ep(bias=A + 2), dtype=0) == INVALID and gemm(ep(), M=65535 * 32 + 1) == UNSUPPORTED
    assert kmajor(ep(), Xt=None) == INVALID and kmajor(ep(), ldxt=63) == INVALID
    for kw in (dict(Xt=at(8)), dict(W=at(8)), dict(ldxt=68), dict(ldw=68), dict(K=2 ** 24, ldw=64)):
        assert kmajor(ep(), **kw) == UNSUPPORTED, kw
    assert gemv(ep(), X=None) == INVALID and gemv(ep(), ldx=4095) == INVALID and gemv(ep(), M=9) == UNSUPPORTED
    assert gemv(ep(), K=2 ** 25, ldx=2 ** 25) == UNSUPPORTED
    need = rmm.rmm_gemv_workspace_size(1, 4, 64, 2048)
    assert need > 256
    assert gemv(ep(), ws=None) == WS_SMALL and gemv(ep(), n=need - 512) == WS_SMALL and gemv(ep(), ws=at(8)) == INVALID


def join(ws=P, n=1 << 40, **kw):
    d = dict(dtype=1, stream_dtype=1, B=2, M=40, K=64, Y=A, ldy=64, R=A + 2 ** 20, ldr=64, residual_scale=1.0, post_norm=0,
             post_gamma=None, gate=None, gate_unit_stride=0, gate_row_stride=0, pre_gamma=A, eps=1e-6, H=A + 2 ** 21, ldh=64,
             X=None, ldx=0, Xt=A, ldxt=40, energy=A)
    d.update(kw)
    return rmm.lib.rmm_block_join(ctypes.byref(_block._JoinC(*d.values())), ws, n, None)


def test_join_refusals():
    assert rmm.lib.rmm_block_join(None, P, 1 << 40, None) == INVALID
    for kw in (dict(dtype=2), dict(stream_dtype=-1), dict(B=0), dict(M=0), dict(K=0), dict(Y=None, R=None),
               dict(H=None, Xt=None, energy=None), dict(energy=None), dict(Xt=None), dict(H=None), dict(ldy=63), dict(ldr=63),
               dict(ldh=63), dict(ldxt=39), dict(X=A, ldx=63, Xt=None, energy=None), dict(Y=None, post_norm=1),
               dict(Y=None, gate=A), dict(gate=A, gate_unit_stride=-8), dict(gate=A, gate_row_stride=-8), dict(eps=-1e-9),
               dict(eps=math.nan), dict(eps=math.inf), dict(residual_scale=math.nan), dict(residual_scale=math.inf),
               dict(H=A + 2 ** 20, ldh=72), dict(X=A, ldx=72, Xt=None, energy=None), dict(Y=A + 1), dict(R=A + 1),
               dict(H=A + 1), dict(gate=A + 1), dict(pre_gamma=A + 1), dict(post_gamma=A + 1), dict(energy=A + 4),
               dict(stream_dtype=0, R=A + 2)):
        assert join(**kw) == INVALID, kw
    for kw in (dict(X=A + 64, ldx=64), dict(dtype=0), dict(K=65544, ldy=65544, ldr=65544, ldh=65544), dict(B=70000, M=1),
               dict(B=2, M=2 ** 21, ldxt=2 ** 21), dict(K=60), dict(ldxt=44), dict(Xt=A + 8), dict(H=A + 2), dict(ldh=68),
               dict(pre_gamma=A + 8), dict(dtype=0, stream_dtype=0)):
        assert join(**kw) == UNSUPPORTED, kw
    need = rmm.rmm_block_join_workspace_size(2, 40, 64)
    assert need > 0
    assert join(ws=None) == WS_SMALL and join(n=need - 1) == WS_SMALL and join(ws=at(128)) == INVALID
    for bad in ((0, 1, 8), (1, 0, 8), (1, 1, 0), (1, 1, 65537), (65536, 1, 8), (1, 2 ** 22, 8)):
        assert rmm.rmm_block_join_workspace_size(*bad) == 0


def test_logprob_refusals():
    def call(ws=P, n=1 << 40, **kw):
        d = dict(z=P, dtype=1, T=3, V=1000, ldl=1000, scale=1.0, tokens=P, given=2, logp=P, entropy=P, top=5, top_idx=P,
                 top_logp=P)
        d.update(kw)
        return rmm.lib.rmm_token_logprobs(*d.values(), ws, n, None)

    for kw in (dict(z=None), dict(dtype=3), dict(T=0), dict(V=0), dict(ldl=999), dict(V=2 ** 31, ldl=2 ** 31), dict(scale=0.0),
               dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(scale=3e38), dict(given=-1), dict(top=-1),
               dict(V=4, top=5), dict(given=0, top=0, entropy=None), dict(tokens=None), dict(logp=None), dict(top_idx=None),
               dict(top_logp=None), dict(z=at(1)), dict(dtype=0, z=at(2)), dict(tokens=at(2)), dict(logp=at(2)),
               dict(entropy=at(2)), dict(top_idx=at(2)), dict(top_logp=at(2))):
        assert call(**kw) == INVALID, kw
    assert call(top=65) == UNSUPPORTED and call(T=2 ** 22) == UNSUPPORTED and call(given=2 ** 31) == UNSUPPORTED
    assert call(V=2 ** 30, ldl=2 ** 30) == UNSUPPORTED
    need = rmm.rmm_token_logprobs_workspace_size(1, 100000, 5)
    assert need > 0
    big = dict(T=1, V=100000, ldl=100000)
    assert call(ws=None, **big) == WS_SMALL and call(n=need - 512, **big) == WS_SMALL and call(ws=at(4), **big) == INVALID
    for bad in ((0, 10, 1), (1, 0, 1), (1, 10, -1), (1, 10, 65), (2 ** 22, 10, 1), (1, 2 ** 30, 1)):
        assert rmm.rmm_token_logprobs_workspace_size(*bad) == 0


def test_binding_refusals():
    """What the Python layer refuses before it calls the library (CPU tensors reach none of it)."""
    bf = torch.bfloat16
    X, W, Y = torch.zeros(2, 3, 16, dtype=bf), torch.zeros(16, 24, dtype=bf), torch.zeros(2, 3, 24, dtype=bf)
    idx = torch.zeros(2, 4, dtype=torch.int32)
    f = rmm.rmm_reduced_gemm_epilogue
    with pytest.raises(ValueError, match="GPU"):
        f(X, W, idx, Y)
    with pytest.raises(ValueError):
        f(X, W[:8], idx, Y)
    with pytest.raises(TypeError):
        f(X, W.float(), idx, Y)
    with pytest.raises(ValueError):
        f(X, W, idx, Y[:, :2])
    with pytest.raises(TypeError):
        f(X, W, idx, Y.float())
    Xt, h = torch.zeros(2, 16, 8, dtype=bf)[:, :, :3], torch.zeros(2, 3, 24)
    with pytest.raises(TypeError):
        rmm.rmm_reduced_gemm_kmajor_epilogue(Xt, W, idx, h)
    with pytest.raises(ValueError):
        _block._epilogue(Y, (2, 3, 24), None, "tanh", None, 1.0)
    with pytest.raises(ValueError):
        _block._epilogue(Y, (2, 3, 24), torch.zeros(23, dtype=bf), None, None, 1.0)
    with pytest.raises(ValueError):
        _block._epilogue(Y, (2, 3, 24), torch.zeros(24), None, None, 1.0)
    with pytest.raises(ValueError):
        _block._epilogue(Y, (2, 3, 24), None, None, Y[:1], 1.0)
    with pytest.raises(ValueError, match="packed"):
        _block._epilogue(Y, (2, 3, 24), None, None, torch.zeros(2, 4, 24, dtype=bf)[:, :3], 1.0)
    j = rmm.rmm_block_join
    with pytest.raises(ValueError):
        j(None, None, H=X)
    with pytest.raises(ValueError):
        j(X, X[:1])
    with pytest.raises(TypeError):
        j(X.half(), X.half(), H=X)
    with pytest.raises(TypeError):
        j(X, X, H=X.float())
    for g in (torch.zeros(15, dtype=bf), torch.zeros(3, 16, dtype=bf), torch.zeros(2, 2, 16, dtype=bf)):
        with pytest.raises(ValueError):
            j(X, X, H=X, gate=g)
    with pytest.raises(TypeError):
        j(X, X, H=X, gate=torch.zeros(16))
    with pytest.raises(ValueError, match="GPU"):
        j(X, X, H=X)
    p = rmm.rmm_token_logprobs
    z, t = torch.zeros(4, 10), torch.zeros(4, 2, dtype=torch.int32)
    for kw in (dict(tokens=t), dict(logp=t), dict(top_idx=t), dict(tokens=t[:3], logp=t[:3]), dict(tokens=t, logp=t[:, 0]),
               dict(top_idx=t[:3], top_logp=t[:3])):
        with pytest.raises(ValueError):
            p(z, **kw)
    with pytest.raises(ValueError, match="contiguous"):
        p(z.t().contiguous().t(), entropy=torch.zeros(4))
    with pytest.raises(ValueError, match="GPU"):
        p(z, entropy=torch.zeros(4))


def test_given_tokens_end_below_the_index_range():
    """A row's loop over its given tokens goes by threads: near 2^31 its index would wrap to negative ones."""
    def call(given):
        return rmm.lib.rmm_token_logprobs(P, 1, 1, 1000, 1000, 1.0, P, given, P, None, 0, None, None, P, 1 << 40, None)

    for given in (2 ** 30, 2 ** 31 - 256, 2 ** 31 - 1):
        assert call(given) == UNSUPPORTED, given


@pytest.mark.parametrize("dtype", [0, 1])
def test_products_end_below_the_index_range(dtype):
    """The row-major products step k and N by whole tiles in 32 bits, past the last column and index."""
    gemm = forms()[0]
    for n in (2 ** 31 - 1023, 2 ** 31 - 1):
        assert gemm(ep(ldr=n), dtype=dtype, N=n, ldw=n, ldy=n) == UNSUPPORTED
        assert gemm(ep(), dtype=dtype, M=1, K=n, k=n, ldx=n) == UNSUPPORTED
        assert rmm.lib.rmm_reduced_gemm(P, P, P, dtype, 1, 4, n, 128, 32, 128, n, P, n, None) == UNSUPPORTED
        assert rmm.lib.rmm_reduced_gemm(P, P, P, dtype, 1, 1, 64, n, n, n, 64, P, 64, None) == UNSUPPORTED
