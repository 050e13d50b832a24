"""More calls of the cache entry points that are refused before any HIP call (CPU)."""
import ctypes

import pytest

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
