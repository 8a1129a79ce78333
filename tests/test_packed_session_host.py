"""What PackedSession refuses and how it lays its pools out, without a GPU."""
import numpy as np
import pytest
import torch

from paper_2505_13544_amd import session as S


def test_free_pages():
    assert S._free_pages(None, 5).tolist() == [0, 1, 2, 3, 4]
    for order in ([3, 1], np.array([3, 1], np.int64), torch.tensor([3, 1]), np.arange(8)[3::-2]):
        got = S._free_pages(order, 5)
        assert got.tolist() == [3, 1] and got.dtype == np.int32 and got.flags["C_CONTIGUOUS"]
    assert S._free_pages(np.zeros(0, np.int32), 5).size == 0
    for order in ([0, 1, 1], [0, 5], [-1, 2], [[0, 1]], [0.0, 1.0], list(range(6)), [True, False], 3):
        with pytest.raises(ValueError):
            S._free_pages(order, 5)
