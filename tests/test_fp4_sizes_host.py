"""Sizes that the 4-bit floating-point operators report without a GPU: nothing to hold
is no bytes of codes or scales, and the scratch of a backward pass is asked for with any
of its sizes zero."""
import os
import subprocess
import sys

import pytest

from paper_2306_04235_gb300 import mnmt

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_packed_sizes():
    assert [mnmt.mnmt_fp4_pitch(k) for k in (-1, 0, 1, 32, 33)] == [0, 0, 16, 16, 32]
    assert [mnmt.mnmt_fp4_scale_bytes(m, 128, mnmt.FP4_MX) for m in (-1, 0, 1, 128, 129)] == [0, 0, 512, 512, 1024]
    assert mnmt.mnmt_fp4_scale_bytes(1, 129, mnmt.FP4_NV) == 3 * 512 and mnmt.mnmt_fp4_scale_bytes(1, 0, mnmt.FP4_NV) == 0


@pytest.mark.parametrize("M,N,K", [(0, 0, 1), (0, 8, 40), (8, 0, 40), (64, 0, 40), (65, 0, 40), (16384, 0, 512), (1 << 30, 0, 8), (0, 1 << 30, 8)])
def test_workspace_of_empty_sides(M, N, K):
    """Sums over nothing use no scratch, but a buffer has to be given.  In a process of its own: a division by zero would
    end it."""
    code = f"from paper_2306_04235_gb300 import mnmt; print(mnmt.mnmt_fp4_linear_backward_workspace({M}, {N}, {K}))"
    run = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=ROOT)
    assert run.returncode == 0, run.stderr
    assert int(run.stdout) > 0


@pytest.mark.parametrize("M,N,K", [(-1, 8, 8), (8, -1, 8), (8, 8, 0), ((1 << 30) + 1, 8, 8)])
def test_workspace_of_no_size(M, N, K):
    assert mnmt.mnmt_fp4_linear_backward_workspace(M, N, K) == 0
