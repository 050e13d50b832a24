"""Scratch memory that a call allocates for itself comes from the pool of the stream
it runs on (CPU: the library and the streams are stand-ins).  A block of another
stream's pool could still be in use by that stream's kernels."""
import contextlib

import pytest
import torch

import paper_2608_13426_amd as rmm

BF, F64, I32 = torch.bfloat16, torch.float64, torch.int32


class _Lib:
    """The real library's size functions; every launch is left out."""
    real = rmm.lib

    def __getattr__(self, name):
        return getattr(self.real, name) if name.endswith(("_size", "_count")) else lambda *args: 0


@pytest.fixture
def calls(monkeypatch):
    """[(stream that is current, ...)] of the binding's allocations; None: the caller's."""
    cur, seen, empty = [None], [], torch.empty

    @contextlib.contextmanager
    def stream(s):
        cur.append(s)
        yield
        cur.pop()

    def alloc(*args, **kw):
        seen.append(cur[-1])
        return empty(*args, **kw)

    monkeypatch.setattr(rmm, "lib", _Lib())
    monkeypatch.setattr(rmm, "_dev", lambda *ts: torch.device("cpu"))
    monkeypatch.setattr(rmm, "_device_index", lambda *ts: 0)
    monkeypatch.setattr(rmm, "_stream", lambda device, s: 0)
    monkeypatch.setattr(rmm, "_run", lambda *args: None)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: cur[-1])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: None)
    monkeypatch.setattr(torch, "empty", alloc)
    return seen


def z(*shape, dtype=BF):
    return torch.zeros(*shape, dtype=dtype)


def _decode_group():
    return [(z(2, 512), z(512, 256), 128, z(2, 128, dtype=I32), z(2, 256))]


def _heads():
    return z(1, 4, 64, 128), z(1, 2, 64, 128)


def _paged(s):
    q = z(3, 8, 128)
    cache = rmm.kv_cache(4, 2, 16, 128, device="cpu")
    return rmm.rmm_paged_attention(q, cache, z(3, 4, dtype=I32), z(3, dtype=I32), q, stream=s)


CALLS = {
    "check_indices": lambda s: rmm.rmm_check_indices(z(2, 8, dtype=I32), 64, stream=s),
    "gemv": lambda s: rmm.rmm_reduced_gemv(z(1, 2, 512), z(512, 256), z(1, 128, dtype=I32), z(1, 2, 256), stream=s),
    "swiglu": lambda s: rmm.rmm_reduced_gemm_swiglu_kmajor(z(1, 64, 32), z(64, 256), z(1, 32, dtype=I32), z(1, 128, 32),
                                                           z(1, 128, dtype=F64), stream=s),
    "attention": lambda s: rmm.rmm_reduced_attention(_heads()[0], _heads()[1], _heads()[1], z(1, 4, 64, dtype=I32),
                                                     _heads()[0], stream=s),
    "attention_kmajor": lambda s: rmm.rmm_reduced_attention_kmajor(_heads()[0], _heads()[1], _heads()[1],
                                                                   z(1, 4, 64, dtype=I32), z(1, 512, 64),
                                                                   z(1, 512, dtype=F64), stream=s),
    "pv": lambda s: rmm.rmm_reduced_pv(z(1, 4, 64, 64), _heads()[1], 32, _heads()[0], stream=s),
    "linear": lambda s: rmm.rmm_linear(z(1, 64, 512), z(512, 256), 0.5, z(1, 64, 256), stream=s),
    "rmsnorm": lambda s: rmm.rmm_rmsnorm_kmajor(z(1, 64, 512), z(512), 1e-6, z(1, 512, 64), z(512, dtype=F64), stream=s),
    "weights": lambda s: rmm.rmm_attention_weights_kmajor(z(1, 4, 64, 64), z(1, 4, 64, 64), z(256, dtype=F64), stream=s),
    "decode_products": lambda s: rmm.rmm_decode_products(_decode_group(), stream=s),
    "decode_products_shared": lambda s: rmm.rmm_decode_products_shared(_decode_group(), stream=s),
    "decode_step_shared": lambda s: rmm.rmm_decode_step_shared(_decode_group(), stream=s),
    "decode_step": lambda s: rmm.rmm_decode_step(_decode_group(), stream=s),
    "qk_norm_rope": lambda s: rmm.rmm_qk_norm_rope(z(1, 64, 4, 128), z(1, 4, 64, 128), energy=z(512, dtype=F64), stream=s),
    "paged_attention": _paged,
}


@pytest.mark.parametrize("name", CALLS)
def test_scratch_is_of_the_calls_stream(name, calls):
    s = object()
    CALLS[name](s)
    assert calls and all(c is s for c in calls)
    del calls[:]
    CALLS[name](None)
    assert calls and all(c is None for c in calls)


def test_every_wrapper_that_allocates_is_listed():
    """A new allocation elsewhere in the binding would not be seen above."""
    import inspect
    src = inspect.getsource(rmm)
    assert src.count("torch.empty(") == inspect.getsource(rmm._scratch).count("torch.empty(")
    assert src.count("_scratch(") - 1 == len(CALLS)


class _Stream:
    cuda_stream = 7

    def __init__(self, device):
        self.device = torch.device("cuda", device)


def test_stream_of_another_device(monkeypatch):
    """A kernel launched on another device's stream would run there, on pointers of this one."""
    ran = []
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(rmm, "lib", type("L", (), {"f": staticmethod(lambda *args: ran.append(args) or 0)}))
    assert rmm._stream(torch.device("cuda", 0), _Stream(0)) == 7
    rmm._run("f", 0, _Stream(0), 1)
    assert ran == [(1, 7)]
    with pytest.raises(ValueError, match="stream"):
        rmm._stream(torch.device("cuda", 0), _Stream(1))
    with pytest.raises(ValueError, match="stream"):
        rmm._run("f", 0, _Stream(1), 1)
    assert len(ran) == 1
