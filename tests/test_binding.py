"""What the binding takes for an address, and what it refuses."""
import ctypes

import numpy as np
import pytest

from paper_2508_13716_amd import binding as B


@pytest.mark.parametrize("x", ["text", b"bytes", bytearray(8), 1.5, [1, 2], (1,), ctypes.c_void_p(64)])
def test_what_is_no_address_is_refused(x):
    with pytest.raises(AttributeError):
        B._p(x)
    with pytest.raises(AttributeError):        # before the library is called
        B.softmax_ce(4, 3, x, 3, None, None, 0.0, None, None, 3, B.F32, None, 0)
    with pytest.raises(AttributeError):
        B.distill(4, 3, x, 3, B.F32, None, None, 2, 2, 0, 1.0, None, 0.0, 1.0, None, None, None, 3, B.F32, 0, None, 0)


def test_addresses():
    import torch
    a, t = np.zeros(3), torch.zeros(3)
    assert B._p(None) is None and B._p(12) == 12 and B._p(np.int64(12).item()) == 12
    assert B._p(a) == a.ctypes.data and B._p(t) == t.data_ptr()
