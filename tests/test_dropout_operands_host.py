"""Which operands the backward pass of dropout hands to its kernel (csrc/train.h): the
kernel reads what it is given, in the type that the caller gave for an output, so an
operand of no output that was asked for must not reach it."""
import itertools
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUDA = os.path.join(os.environ.get("CUDA_HOME", "/usr/local/cuda"), "include")

pytestmark = pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists(os.path.join(CUDA, "cuda_runtime.h")),
                                reason="needs a host compiler and the CUDA headers")


def test_operands_of_the_outputs_asked_for(tmp_path):
    src = tmp_path / "o.cpp"
    src.write_text("""#include "train.h"
#include <cstdio>
int main() {
    int gx, gr, gg, relu;
    static float p[4];
    while (scanf("%d %d %d %d", &gx, &gr, &gg, &relu) == 4) {
        mnmt::DropoutArgs a{};
        a.x = p, a.r = p + 1;
        a.gx = gx ? p + 2 : nullptr, a.gr = gr ? p + 3 : nullptr, a.ggamma = gg ? p : nullptr, a.relu = relu;
        printf("%d %d\\n", a.backward_x() == a.x, a.backward_r() == a.r);
    }
}
""")
    exe = tmp_path / "o"
    subprocess.run(["g++", "-std=c++17", "-I", os.path.join(ROOT, "paper_2306_04235_gb300", "csrc"), "-I", os.path.join(ROOT, "include"), "-I", CUDA,
                    str(src), "-o", str(exe)], check=True)
    calls = list(itertools.product((0, 1), repeat=4))
    out = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in calls), capture_output=True, text=True, check=True).stdout
    got = [tuple(int(v) for v in line.split()) for line in out.splitlines()]
    assert got == [(int(relu and gx), gg) for gx, gr, gg, relu in calls]
