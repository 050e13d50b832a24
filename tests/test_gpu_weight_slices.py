"""Products whose weights (or K-major activations) are the last columns of a wider matrix,
which ends where its storage does: the same bits as with a matrix of their own."""
import pytest
import torch

import paper_2608_13426_amd as rmm
from tests.gpu_util import gpu, require_gpu

pytestmark = gpu
BF = torch.bfloat16


def make(dev, B, M, K, N, k, first, wide=None, seed=0):
    """X, the last N columns of a [K, first + N] matrix, lists that end with the last row."""
    g = torch.Generator(device=dev).manual_seed(seed)
    X = torch.randn(B, M, K, device=dev, generator=g).to(BF)
    W = (0.1 * torch.randn(K, first + N, device=dev, generator=g)).to(BF)
    idx = torch.rand(B, K - 1, device=dev, generator=g).topk(k - 1, dim=1).indices.sort(dim=1).values
    idx = torch.cat([idx, torch.full((B, 1), K - 1, device=dev)], 1).int().contiguous()
    return X, W[:, first:], idx


def own(W):
    """The same values in rows of their own, 16-byte aligned, with columns behind them."""
    K, N = W.shape
    return torch.zeros(K, (N + 7) // 8 * 8 + 512, dtype=W.dtype, device=W.device)[:, :N].copy_(W)


# (first, N): first + N a multiple of 8 keeps 16-byte loads
@pytest.mark.parametrize("first,N", [(8, 1000), (520, 200), (1024, 40), (8, 8), (24, 4096 + 8), (7, 65), (3, 1001)])
@pytest.mark.parametrize("M", [1, 2, 5, 8])
@pytest.mark.parametrize("k", [12, 700])
def test_few_rows(first, N, M, k):
    dev = require_gpu()
    X, W, idx = make(dev, 2, M, 1000, N, k, first)
    V = own(W) if (first + N) % 8 == 0 and first % 8 == 0 else W.contiguous()
    for f in (rmm.rmm_reduced_gemv, rmm.rmm_reduced_gemv_epilogue):
        Y, Z = (torch.empty(2, M, N, dtype=BF, device=dev) for _ in range(2))
        f(X, W, idx, Y)
        f(X, V, idx, Z)
        if V.stride(0) % 8 == 0 and W.stride(0) % 8 == 0 and first % 8 == 0:
            assert torch.equal(Y, Z), f.__name__
        else:                                    # another kernel's order of the sums
            assert float((Y.double() - Z.double()).abs().max()) <= 2.0 ** -7 * float(Z.double().abs().max()), f.__name__


@pytest.mark.parametrize("B,M,first,N", [(1, 40, 8, 56), (1, 500, 520, 1000), (1, 1025, 8, 2048 + 40), (1, 2048, 64, 4096 + 8), (40, 4200, 16, 120)])
def test_kmajor(B, M, first, N):
    dev = require_gpu()
    X, W, idx = make(dev, B, M, 96, N, 50, first)
    V, ld = own(W), (M + 7) // 8 * 8
    Xw = torch.zeros(B, 96, 16 + ld, dtype=BF, device=dev)[:, :, 16:16 + M]      # the last tokens of a longer copy
    Xw.copy_(X.transpose(1, 2))
    Xt = torch.zeros(B, 96, ld + 256, dtype=BF, device=dev)[:, :, :M]
    Xt.copy_(X.transpose(1, 2))
    for f in (rmm.rmm_reduced_gemm_kmajor, rmm.rmm_reduced_gemm_kmajor_epilogue):
        Y, Z = (torch.empty(B, M, N, dtype=BF, device=dev) for _ in range(2))
        f(Xw, W, idx, Y)
        f(Xt, V, idx, Z)
        assert torch.equal(Y, Z), f.__name__


@pytest.mark.parametrize("M,first,N", [(40, 8, 56), (2048, 64, 4096 + 8)])
def test_row_major(M, first, N):
    dev = require_gpu()
    X, W, idx = make(dev, 1, M, 96, N, 50, first)
    V = own(W)
    for f in (rmm.rmm_reduced_gemm, rmm.rmm_reduced_gemm_epilogue):
        Y, Z = (torch.empty(1, M, N, dtype=BF, device=dev) for _ in range(2))
        f(X, W, idx, Y)
        f(X, V, idx, Z)
        assert torch.equal(Y, Z), f.__name__


@pytest.mark.parametrize("B", [1, 7])
@pytest.mark.parametrize("first,N", [(8, 1000), (1024, 40), (24, 520)])
def test_decode_products(B, first, N):
    dev = require_gpu()
    X, W, idx = make(dev, B, 1, 1024, N, 500, first)
    V, X, idx = own(W), X.view(B, 1024), idx.view(-1)
    for f in (rmm.rmm_decode_products, rmm.rmm_decode_products_shared):
        Y, Z = (torch.empty(B, N, dtype=BF, device=dev) for _ in range(2))
        f([(X, W, 500, idx, Y)])
        f([(X, V, 500, idx, Z)])
        assert torch.equal(Y, Z), f.__name__
