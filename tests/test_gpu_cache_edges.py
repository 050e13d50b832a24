"""Rotation, appending and reading back at the edges of what the cache entry points take."""
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
