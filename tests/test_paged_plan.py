"""How the attention over the paged cache lays its work on a line and cuts it (CPU):
the arithmetic that the kernels are built from, compiled for the host."""
import os
import random
import subprocess
from collections import namedtuple

import pytest
import torch

from tests import paged_cases as pc
from tests import paged_ref as pr
from tests import test_lds_order as lds

Plan = namedtuple("Plan", "rows host_whole whole units run piece most cut blocks")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("plan") / "plan")
    build = lds.build
    subprocess.run([build.HIPCC, "-x", "hip", f"--offload-arch={build.ARCH}", "-O1", "-std=c++17",
                    os.path.join(os.path.dirname(__file__), "paged_plan_host.cpp"), "-o", exe], check=True)

    def run(cases, T=None, q_start=None):
        text = []
        for mx, D, H, Hkv, causal, page, width, lens, news in cases:
            starts = q_start or (news and [sum(news[:b]) for b in range(len(news) + 1)]) or []
            n = T or (starts[-1] if starts else len(lens))
            text += [int(mx), D, H, Hkv, int(causal), page, width, n, len(lens), int(bool(starts)), *lens, *starts]
        out = subprocess.run([exe], input=" ".join(map(str, text)), text=True, check=True, stdout=subprocess.PIPE).stdout
        lines = out.splitlines()
        assert len(lines) == len(cases)
        for c, l in zip(cases, lines):
            assert not l.startswith("error"), (l, c)
        return [l if l == "over" else Plan(*map(int, l.split())) for l in lines]
    return run


def _case(mx, c):
    _, D, H, Hkv, causal, page, lens, news, _ = c
    return mx, D, H, Hkv, causal, page, -(-max(lens) // page), lens, news


def test_every_key_block_once(plan):
    """Random calls: each unit's blocks are covered once, its pieces lie where they are joined from."""
    rng = random.Random(5)
    cases = []
    for _ in range(400):
        B = rng.choice([1, 2, 3, 7, 63, 64, 65, 130, 300])
        Hkv, grp, page = rng.choice([1, 2, 3, 8]), rng.choice([1, 3, 4, 5, 16, 40]), rng.choice([16, 64, 1024])
        top = int(2 ** rng.uniform(0, 17 if B < 8 else 13))
        lens = [rng.choice([0, 1, rng.randint(1, top), rng.randint(1, top)]) for _ in range(B)]
        most = rng.choice([1, 2, 9, 70, 400 if B < 20 else 20, 3000 if B < 4 else 30])
        news = None if rng.random() < 0.3 else [rng.choice([0, 1, rng.randint(0, most)]) for _ in range(B)]
        if news is not None and sum(news) == 0:
            news[0] = 1
        width = max(1, -(-max(lens) // page) + rng.choice([0, 0, 1, 100, -1]))
        cases.append((rng.random() < 0.5, rng.choice([64, 128]), Hkv * grp, Hkv, rng.random() < 0.7, page, width, lens, news))
    plans = plan(cases)
    # the draws reach every kind of call
    assert {p.rows for p in plans} == {16, 32, 64, 256}
    assert any(p.host_whole for p in plans) and any(p.whole and not p.host_whole for p in plans)
    assert any(p.cut > 100 for p in plans) and any(p.cut and p.rows == 256 for p in plans)


def test_overlapping_sequences(plan):
    """A q_start that falls and rises again gives sequences of more tokens than there are: past what
    the line (and 32-bit places on it) was checked for, so such a call has no line."""
    T, B = 1000, 2000
    starts = [b % 2 * T for b in range(B + 1)]
    assert plan([(0, 64, 32, 8, 1, 1024, 1000, [10 ** 6] * B, None)], T=T, q_start=starts) == ["over"]
    starts = [0] * (B // 2) + [T] * (B // 2 + 1)               # one sequence with all, the others empty
    assert plan([(0, 64, 32, 8, 1, 1024, 1000, [10 ** 6] * B, None)], T=T, q_start=starts)[0].units == T * 32 // 16


def test_long_cases_reach_their_plans(plan):
    keys = [(n, t) for n, c in pc.CASES.items() for t in c[0]]
    for (n, t), p in zip(keys, plan([_case(t == "mx", pc.CASES[n]) for n, t in keys])):
        assert pc.CASES[n][-1](p), (n, t, p)


@pytest.mark.parametrize("name", pc.CASES)
def test_long_cases_notice_a_lost_run(name, plan):
    """Dropping or doubling the keys of one run of the longest sequence (of 256 keys, the
    shortest run there is, where units are kept whole) is refused by the limits that the GPU
    test of the case uses."""
    c = pc.CASES[name]
    (p,) = plan([_case("mx" in c[0], c)])
    D, L = c[1], max(c[6])
    n = 256 if p.whole else p.run * (64 if p.rows == 256 else 32)
    assert n < L
    g = torch.Generator().manual_seed(1)
    K = torch.randn(L, D, dtype=torch.float64, generator=g)
    V = torch.randn(L, D, dtype=torch.float64, generator=g)
    q = torch.randn(2, D, dtype=torch.float64, generator=g)
    see = torch.tensor([L, L])
    ref = pr.attend(q, K, V, see, D ** -0.5, True)
    assert pr.accepts(ref[0].bfloat16().double(), *ref)
    for at in (0, (L // 2) // n * n):
        for rest in (torch.cat([torch.arange(at), torch.arange(at + n, L)]), torch.cat([torch.arange(L), torch.arange(at, at + n)])):
            o = pr.attend(q, K[rest], V[rest], torch.tensor([len(rest)] * 2), D ** -0.5, True)[0]
            assert not pr.accepts(o, *ref), (name, at)
