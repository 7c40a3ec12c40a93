"""The rule for products of a few rows (csrc/routes.h) where x is large: every block of
the one-launch kernel quantises all of x.  Measured on a GB300, us a call back to back
with x to be quantised: one launch / quantisation and product, MX and NV."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2306_04235_gb300", "csrc")

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host compiler")

# M, N, K: MX one, two; NV one, two
TIMES = {
    (1, 64, 64): (2.50, 4.85, 2.12, 4.96), (1, 512, 512): (2.76, 5.06, 2.60, 5.78), (1, 512, 2048): (3.47, 7.31, 3.63, 8.69),
    (1, 8192, 8192): (17.71, 20.42, 18.50, 22.90), (1, 32000, 2048): (15.86, 16.58, 15.61, 16.43),
    (1, 32000, 8192): (54.11, 60.79, 50.47, 63.93), (1, 2048, 32768): (27.33, 33.42, 39.57, 38.67),
    (1, 64, 32768): (22.11, 32.89, 34.24, 37.95), (1, 128000, 4096): (105.23, 103.39, 101.19, 106.54),
    (1, 8192, 32768): (70.08, 65.12, 81.30, 74.79), (2, 2048, 2048): (4.44, 8.03, 4.75, 9.36), (2, 8192, 512): (4.24, 6.19, 4.09, 6.49),
    (2, 512, 16384): (15.96, 19.09, 20.06, 21.65), (4, 2048, 512): (3.63, 5.67, 3.37, 6.03), (4, 2048, 2048): (5.62, 7.26, 6.49, 8.13),
    (4, 512, 8192): (12.63, 12.07, 15.25, 13.46), (8, 512, 512): (4.55, 5.42, 4.34, 5.88), (8, 2048, 512): (4.70, 5.78, 4.39, 6.08),
    (8, 512, 2048): (7.16, 6.75, 8.23, 7.39), (8, 512, 4096): (11.61, 8.59, 13.40, 9.31),
}


def test_the_faster_form_to_a_tenth(tmp_path):
    src = tmp_path / "r.cpp"
    src.write_text("""#include "routes.h"
#include <cstdio>
int main() {
    int M, N, K;
    while (scanf("%d %d %d", &M, &N, &K) == 3) printf("%d\\n", (int)mnmt::route_fp4_small(M, N, K));
}
""")
    exe = tmp_path / "r"
    subprocess.run(["g++", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    text = "\n".join(" ".join(map(str, k)) for k in TIMES)
    got = [int(v) for v in subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True).stdout.split()]
    for (size, (m1, m2, n1, n2)), one in zip(TIMES.items(), got):
        for a, b in ((m1, m2), (n1, n2)):
            assert (a if one else b) <= 1.1 * min(a, b), size
