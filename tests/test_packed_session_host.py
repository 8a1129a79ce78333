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


def session(max_batch):
    s = object.__new__(S.PackedSession)
    s.max_batch = max_batch
    return s


@pytest.mark.parametrize("batch,at", [(3, 1), (1, 3), (2, 2), (1, -1), (1 << 20, 1), (1, 1 << 20)])
def test_sequences_that_a_session_lacks(batch, at):
    # refused before a call is made (there is no GPU, and nothing else of a session, here)
    s = session(3)
    with pytest.raises(IndexError):
        s.fit(batch, at=at)
    with pytest.raises(IndexError):
        s.unpack(batch, 4, at=at)
    x = torch.zeros(batch if batch < 9 else 9, 5, 64)
    with pytest.raises(IndexError):
        s.prefill(x, x, x, x, out=None, at=at)


@pytest.mark.parametrize("call", ["fit", "unpack"])
def test_arrays_that_are_none_of_the_call(call):
    s = session(3)
    ints, longs = lambda *n: torch.zeros(*n, dtype=torch.int32), lambda *n: torch.zeros(*n, dtype=torch.int64)
    for kw in (dict(counts=longs(3)), dict(counts=[1, 2, 3]), dict(counts=ints(6)[::2]), dict(slot_map=ints(3, 4)), dict(slot_map=longs(4, 3).t())):
        with pytest.raises(TypeError):
            getattr(s, call)(3, 4, **kw)
    for kw in (dict(counts=ints(2)), dict(slot_map=longs(3, 3)), dict(slot_map=longs(11))):
        with pytest.raises(ValueError):
            getattr(s, call)(3, 4, **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_outputs_of_another_type(dtype):
    # refused before the tables are touched
    s = session(3)
    s.w_uv = None
    x, out = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(3, 4, 64, dtype=dtype)
    with pytest.raises(TypeError):
        s.decode(x, x, out=out)
    with pytest.raises(TypeError):
        s.step(x, x, x, x, out=out)
