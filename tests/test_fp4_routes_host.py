"""The rules that choose the kernel of a product of 4-bit floating-point matrices
(csrc/routes.h), against measured times of all forms (tests/golden/fp4_routes.txt)."""
import math
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2306_04235_gb300", "csrc")
TABLE = os.path.join(ROOT, "tests", "golden", "fp4_routes.txt")

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host compiler")


def _rows(kind):
    return [l.split()[1:] for l in open(TABLE) if l.split()[:1] == [kind]]


def _decide(tmp_path, expr, rows):
    src = tmp_path / "r.cpp"
    src.write_text(f"""#include "routes.h"
#include <cstdio>
using namespace mnmt;
int main() {{
    int M, N, K;
    while (scanf("%d %d %d", &M, &N, &K) == 3) printf("%d\\n", (int)({expr}));
}}
""")
    exe = tmp_path / "r"
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    text = "\n".join(" ".join(str(x) for x in r) for r in rows)
    return [int(x) for x in subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True).stdout.split()]


def test_products_take_the_fastest_tiles(tmp_path):
    """FP4_PAIR, FP4_128, FP4_64 are 0, 1, 2; the times repeat to a few per cent, and to half a microsecond."""
    rows = [([int(x) for x in f[2:5]], [float(x) for x in f[5:]]) for f in _rows("fp4")]
    assert len(rows) >= 150
    got = _decide(tmp_path, "route_fp4_tiles(M, N, K, 152)", [r for r, _ in rows])
    total = 0.0
    for (size, t), g in zip(rows, got):
        mine = t[2 - g]
        assert mine <= 1.1 * min(t) + 1.3, (size, t, g)
        total += math.log(mine / min(t))
    assert total / len(rows) < 0.03


def test_a_few_rows_take_the_faster_kernel(tmp_path):
    rows = [([int(x) for x in f[:3]], [float(x) for x in f[3:]]) for f in _rows("small")]
    got = _decide(tmp_path, "route_fp4_small(M, N, K)", [r for r, _ in rows])
    for (size, (one, two)), g in zip(rows, got):
        assert (one if g else two) <= 1.05 * min(one, two), size
    # more than eight rows, or more of x than the kernel holds, never
    assert _decide(tmp_path, "route_fp4_small(M, N, K)", [[9, 64, 64], [2, 64, 16385], [1, 64, 32769], [1, 64, 32768]]) == [0, 0, 0, 1]
