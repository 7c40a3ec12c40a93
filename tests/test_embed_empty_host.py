"""The table gradient's scratch size: 0 stands for sizes that are invalid, and for no others."""
import pytest

from paper_2306_04235_gb300 import mnmt


@pytest.mark.parametrize("T,V,d", [(0, 1, 1), (0, 2490368, 8), (0, 2490369, 8), (0, 311297, 2048), (0, 1 << 30, 1), (0, 1 << 30, 1 << 30), (1, 1 << 30, 8),
                                   (4096, 2490369, 8), (4097, 10, 8)])
def test_valid_sizes(T, V, d):
    """No tokens among them, whatever the table's size (few tokens into a small table take one launch, others several)."""
    assert mnmt.mnmt_embed_backward_workspace(T, V, d) >= 16


@pytest.mark.parametrize("T,V,d", [(-1, 5, 5), (5, 0, 5), (0, 5, 0), ((1 << 30) + 1, 5, 5)])
def test_invalid_sizes(T, V, d):
    assert mnmt.mnmt_embed_backward_workspace(T, V, d) == 0
