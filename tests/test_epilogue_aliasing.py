"""A product's output may be its residual: no kernel with an epilogue declares Y free of
aliases, from which the compiler could move the residual's loads behind Y's stores
(from the code as it is before optimisation, on the CPU)."""
import os
import re
import subprocess

import pytest

from tests.test_lds_order import PKG, build


def output_of_functions(src, tmp_path):
    """(function, its template arguments, its parameter Y) of every device function that takes one."""
    out = tmp_path / (src + ".ll")
    subprocess.run([build.HIPCC, *build.CFLAGS, "--cuda-device-only", "-S", "-emit-llvm", "-fno-discard-value-names", "-Xclang",
                    "-disable-llvm-passes", os.path.join(PKG, "csrc", src), "-o", str(out)], check=True, stderr=subprocess.DEVNULL)
    defs = re.findall(r"^define .*?@(_Z\w+)\((.*)\) .*\{$", out.read_text(), re.M)
    names = subprocess.run(["c++filt"], input="\n".join(n for n, _ in defs), text=True, capture_output=True, check=True).stdout
    for name, (_, params) in zip(names.split("\n"), defs):
        m = re.match(r"(?:void )?rmm::(ep_tile|gem[mv]_\w+)<(.*?)>\(", name.replace("(anonymous namespace)::", ""))
        y = [p for p in re.split(r", (?=ptr|i\d|float|double)", params) if re.search(r"%Y\b", p)]
        if m and y:
            yield m.group(1), [a.strip() for a in m.group(2).split(",")], y[0]


@pytest.mark.parametrize("src,at_least", [("gemm.hip", 24), ("gemm_mid.hip", 4), ("gemv.hip", 6)])
def test_y_may_be_the_residual(src, at_least, tmp_path):
    seen = 0
    for name, args, y in output_of_functions(src, tmp_path):
        # the variants with an epilogue: by their last argument, or the 256-row K-major kernel's fourth
        if name == "ep_tile" or (args[3] == "2" if name == "gemm_kmajor_tr_kernel" else args[-1] == "true"):
            assert "noalias" not in y, (name, args)
            seen += 1
    assert seen >= at_least
