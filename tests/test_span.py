"""The products' loads end with the last row of a matrix that is some columns of a wider one (CPU)."""
import os
import random
import re
import subprocess

from tests.test_lds_order import PKG, build


def test_span_ends_with_the_last_row(tmp_path):
    exe = str(tmp_path / "span")
    subprocess.run([build.HIPCC, "-x", "hip", f"--offload-arch={build.ARCH}", "-O1", "-std=c++17",
                    os.path.join(os.path.dirname(__file__), "span_host.cpp"), "-o", exe], check=True)
    rng, cases = random.Random(0), []
    for _ in range(2000):
        vec = rng.random() < 0.5
        ld, rows = rng.choice((8, 16, 72, 4096, 6144)) if vec else rng.randint(1, 5000), rng.choice((1, 2, 77, 14336))
        first = rng.randrange(0, ld, 8) if vec else rng.randrange(ld)
        cases.append((rows, ld, rng.randint(1, ld - first), vec, first))
    out = subprocess.run([exe], input="\n".join(f"{r} {ld} {n} {int(v)}" for r, ld, n, v, _ in cases), text=True,
                         capture_output=True, check=True).stdout.split()
    for (rows, ld, n, vec, first), got in zip(cases, map(int, out)):
        held = 2 * ((rows - 1) * ld + n)                             # to the end of the last element
        assert held <= got <= (held + 15) // 16 * 16 if vec else got == held
        assert 2 * first + got <= 2 * rows * ld                      # columns first .. of a [rows][ld] matrix


def test_descriptors_of_shared_operands_go_by_it():
    """No product reaches past a weight matrix by its rows' stride."""
    for src in ("gemm.hip", "gemm_mid.hip", "gemv.hip", "gemv_shared.hip"):
        with open(os.path.join(PKG, "csrc", src)) as f:
            text = re.sub(r"\s+", " ", f.read())
        assert "span_bytes(" in text, src
        for m in re.finditer(r"make_buffer_rsrc\( ?const_cast<uint16_t \*>\((?:q\.)?(?:W|Xt)\b[^;]*;", text):
            assert "ldw - n0" not in m.group(0), (src, m.group(0))
        assert not re.search(r"(xt|w)_bytes = K \* ld", text), src
