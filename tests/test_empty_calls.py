"""Calls with nothing to do.  No GPU."""
import pytest

from paper_2603_14371_amd import binding as B

A = 1 << 20     # an address that no such call reads


def test_rotating_no_tokens_takes_what_an_empty_tensor_has():
    """Null pointers, any stride, any alignment; the configuration is still looked at."""
    good = B.make_rotary(A, 256)
    for args in ((0, 0, 0, 0, 0), (A, A, 4096, A, 4096), (0, A + 2, 7, 0, 3)):
        B.oxy_rotary(good, *args, 0, 8, 0)
    for rotary, heads in ((B.make_rotary(A, 7), 8), (B.make_rotary(0, 256), 8), (B.make_rotary(A, 256, 5), 8), (good, 0)):
        with pytest.raises(B.OxyError):
            B.oxy_rotary(rotary, 0, 0, 0, 0, 0, 0, heads, 0)
    with pytest.raises(B.OxyError):
        B.oxy_rotary(good, 0, 0, 0, 0, 0, -1, 8, 0)
