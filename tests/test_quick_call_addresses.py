"""What the native calls of the binding take as an address is what ctypes takes as a c_void_p, or left to it.  No GPU."""
import ctypes
import enum
import os

import pytest

from paper_2603_14371_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.MARSHAL_PATH), reason="libmarshal.so is not built here")
A = 1 << 20      # an aligned address that no refused call reads


class Holder:
    def __init__(self, value):
        self.value = value


class Handle(ctypes.c_void_p):
    pass


@pytest.mark.parametrize("kind", [ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_bool, Holder,
                                  lambda x: enum.Enum("E", {"x": x}).x], ids=["int", "long", "size_t", "bool", "holder", "enum"])
@pytest.mark.parametrize("at,value", [(0, 0), (1, 0), (3, 0), (5, 1), (7, 1)])
def test_objects_with_a_value_are_refused_as_ctypes_refuses_them(kind, at, value):
    """They were taken as addresses, and the library was called with them."""
    args = [None, None, 0, A, A, None, 0.5, None]
    args[at] = kind(value)
    B.lib()
    assert B._quick.oxy_mixed_attention(*args) is None
    with pytest.raises(ctypes.ArgumentError):
        B.oxy_mixed_attention(*args)


@pytest.mark.parametrize("thing", [0, None, ctypes.c_void_p(None), ctypes.c_void_p(0)], ids=repr)
def test_null_addresses_are_taken(thing):
    B.lib()
    assert B._quick.oxy_mixed_attention(thing, thing, 0, A, A, thing, 0.5, thing) == B.ERR_INVALID_ARG


def test_a_handle_of_a_kind_of_its_own_is_left_to_ctypes():
    B.lib()
    assert B._quick.oxy_mixed_attention(Handle(0), None, 0, A, A, None, 0.5, None) is None
    with pytest.raises(B.OxyError):
        B.oxy_mixed_attention(Handle(0), None, 0, A, A, None, 0.5, None)
