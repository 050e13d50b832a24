"""More calls of the cache entry points that are refused before any HIP call (CPU)."""
import ctypes

import pytest
import torch

import paper_2608_13426_amd as rmm
from tests import test_cache_abi as abi

INVALID, UNSUPPORTED, WS_SMALL, P = abi.INVALID, abi.UNSUPPORTED, abi.WS_SMALL, abi.P


def attention(scale, ws=None):
    """Refused in any case: there is no workspace."""
    q, c = abi.heads(8), abi.cache()
    return rmm.lib.rmm_paged_attention(3, ctypes.byref(q), ctypes.byref(c), P, 5, 5, P, 3, None, None, 0, scale, 1,
                                       ctypes.byref(q), ws, 0, None)


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), -float("inf"), 3e38, -3e38])
def test_attention_scale(scale):
    """NaN, infinite, or infinite in the base-2 units of the softmax (3e38 log2(e) > 2^128)."""
    assert attention(scale) == INVALID


@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-45, -0.1, 2e38])
def test_attention_scale_in_range(scale):
    assert attention(scale) == WS_SMALL


@pytest.mark.parametrize("T,D", [(2 ** 27, 128), (2 ** 28, 64), (2 ** 28 - 1, 128)])
def test_gather_past_a_grid(T, D):
    """2^32 threads and more, of which a launch would run the low 32 bits' worth."""
    c, h = abi.cache(D=D), abi.heads()
    assert rmm.lib.rmm_kv_gather(ctypes.byref(c), P, T, ctypes.byref(h), ctypes.byref(h), None) == UNSUPPORTED


def test_binding_keys_alone():
    """What the binding asks of a call without queries (CPU tensors reach no launch)."""
    K = torch.zeros(1, 3, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        rmm.rmm_qk_norm_rope(None, None, K=K, Ko=K.transpose(1, 2))
    for args in (dict(), dict(K=K), dict(Ko=K)):
        with pytest.raises(ValueError, match="together"):
            rmm.rmm_qk_norm_rope(None, None, **args)
    for q, qo in ((K, None), (None, K.transpose(1, 2))):
        with pytest.raises(ValueError, match="together"):
            rmm.rmm_qk_norm_rope(q, qo, K=K, Ko=K.transpose(1, 2))
    with pytest.raises(ValueError, match="energies"):
        rmm.rmm_qk_norm_rope(None, None, K=K, Ko=K.transpose(1, 2), energy=torch.zeros(256, dtype=torch.float64))


def test_attention_workspace_size():
    """Not monotonous, and below what the header says."""
    f = rmm.rmm_paged_attention_workspace_size
    assert f(64, 64, 32, 8, 128) < f(64, 1, 32, 8, 128)
    # 512 pieces of 256 rows of D sums, two statistics and 32 bytes: 65.02 and 33.02 MiB
    for D, top in ((128, 66 << 20), (64, 34 << 20)):
        sizes = [f(T, B, 8 * g, 8, D) for T in (1, 7, 64, 300, 5000, 100000) for B in (1, 3, 64, 300, 5000) for g in (1, 4, 40)]
        assert 0 < min(sizes) and max(sizes) <= top
