"""What the Python binding takes for a pointer and for a stream, without a GPU."""
import ctypes
import enum

import pytest
import torch

from paper_2608_06628_gb300 import hybrid as H


class Address(int):
    pass


class Slab(enum.IntEnum):
    BASE = 1 << 20


@pytest.mark.parametrize("x", [0, 1 << 40, Address(1 << 20), Slab.BASE, True])
def test_every_int_is_an_address(x):
    """A subclass of int too: an enumeration of addresses, a type of the caller's."""
    assert H._ptr(x) == int(x) and ctypes.c_void_p(H._ptr(x)).value == (int(x) or None)


def test_tensors_and_none():
    t = torch.zeros(5)
    assert H._ptr(t) == t.data_ptr() and H._ptr(t[1:]) == t.data_ptr() + 4 and H._ptr(None) is None
    with pytest.raises(AttributeError):
        H._ptr("16")


@pytest.mark.parametrize("stream", [0, 7, Address(1 << 20)])
def test_streams_by_handle(stream):
    class Stream:
        cuda_stream = stream

    assert H._stream(stream) == H._stream(Stream()) == int(stream)
