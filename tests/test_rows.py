"""Row strides of the gradient block, as the binding reads them from a tensor (no GPU needed)."""
import pytest
import torch

from paper_1905_04374_b200 import binding


def test_rows_that_share_memory_are_refused():
    """One gradient expanded to n workers has row stride 0, which the library would take for d."""
    g = torch.zeros(64)
    with pytest.raises(ValueError, match="share memory"):
        binding._rows(g.expand(4, 64))
    with pytest.raises(ValueError, match="share memory"):
        binding._rows(g.as_strided((4, 8), (7, 1)))


def test_row_strides():
    g = torch.zeros(5, 64)
    assert binding._rows(g) == (5, 64, 64)
    assert binding._rows(g[:, 8:32]) == (5, 24, 64)
    assert binding._rows(g[::2]) == (3, 64, 128)
    assert binding._rows(g[0].expand(1, 64)) == (1, 64, 64)      # a single row may have any stride
