"""What the binding takes for an address."""
import sys

import numpy as np
import pytest

from paper_2509_09090_b200 import binding as B


class Odd(int):
    pass


def test_addresses():
    torch = pytest.importorskip("torch")
    t, a = torch.zeros(4), np.zeros(4)
    assert B._ptr(None) is None and B._ptr(4096) == 4096 and B._ptr(Odd(4096)) == 4096 and B._ptr(2 ** 63) == 2 ** 63
    assert B._ptr(t) == t.data_ptr() and B._ptr(a) == a.ctypes.data
    with pytest.raises(TypeError):
        B._ptr("4096")


def test_an_address_raises_nothing_on_its_way():
    """A plain address is not first asked for what tensors have: the exception costs more than the call's other arguments."""
    seen = []

    def trace(frame, event, arg):
        if event == "exception":
            seen.append(arg[0])
        return trace

    sys.settrace(trace)
    try:
        B._ptr(4096)
    finally:
        sys.settrace(None)
    assert not seen
