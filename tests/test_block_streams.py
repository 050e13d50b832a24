"""The scratch memory of the calls between a layer's products comes from the pool of
the stream it is used on (CPU: the library and the streams are stand-ins)."""
import contextlib
import inspect

import pytest
import torch

import paper_2608_13426_amd as rmm
from paper_2608_13426_amd import _block

BF = torch.bfloat16


@pytest.fixture
def calls(monkeypatch):
    """The stream that is current at each allocation; None: the caller's."""
    cur, seen, empty = [None], [], torch.empty

    @contextlib.contextmanager
    def stream(s):
        cur.append(s)
        yield
        cur.pop()

    def alloc(*args, **kw):
        seen.append(cur[-1])
        return empty(*args, **kw)

    monkeypatch.setattr(_block, "_device_index", lambda *ts: 0)
    monkeypatch.setattr(_block, "_run", lambda *args: None)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch, "empty", alloc)
    return seen


def z(*shape, dtype=BF):
    return torch.zeros(*shape, dtype=dtype)


CALLS = {
    "gemv": lambda s: rmm.rmm_reduced_gemv_epilogue(z(1, 2, 512), z(512, 256), z(1, 128, dtype=torch.int32), z(1, 2, 256),
                                                    stream=s),
    "join": lambda s: rmm.rmm_block_join(z(1, 64, 128), z(1, 64, 128), z(1, 64, 128), Xt=z(1, 128, 64),
                                         energy=z(128, dtype=torch.float64), stream=s),
    "logprobs": lambda s: rmm.rmm_token_logprobs(z(1, 100000), entropy=z(1, dtype=torch.float32), stream=s),
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
    src = inspect.getsource(_block)
    assert "torch.empty(" not in src and src.count("_scratch(") == len(CALLS)
