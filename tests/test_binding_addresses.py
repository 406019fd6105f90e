"""What the binding takes for a buffer, on the CPU."""
import numpy as np
import pytest
import torch

from paper_2101_10761_b200 import binding as B


def test_tensors_arrays_integers_and_none():
    t, a = torch.zeros(4), np.zeros(4)
    assert B._ptr(None) is None and B._ptr(t) == t.data_ptr() and B._ptr(a) == a.ctypes.data
    assert B._ptr(4096) == 4096 and B._ptr(np.int64(4096)) == 4096


@pytest.mark.parametrize("bad", [4096.0, "4096", b"4096", [4096], np.float32(4096), object()])
def test_nothing_else(bad):
    with pytest.raises(TypeError):
        B._ptr(bad)
