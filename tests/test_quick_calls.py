"""The calls that a program makes in every layer go through libmarshal.so where it is built and every argument is a
plain one, and through ctypes otherwise: the same statuses, messages and conversions.  No GPU."""
import ctypes
import os

import numpy as np
import pytest

from paper_2603_14371_amd import binding as B

pytestmark = pytest.mark.skipif(not os.path.exists(B.MARSHAL_PATH), reason="libmarshal.so is not built here")
A = 1 << 20      # an aligned address that no refused call reads


@pytest.fixture()
def batch():
    pool = B.oxy_pool_create(B.make_config(2, 8, flags=B.POOL_HOST_ONLY))
    sid = B.oxy_stream_create(pool, -1, B.KIND_DECODE)
    b = B.oxy_batch_build(pool, [(sid, 3)], 0, 0)
    yield pool, b
    B.oxy_batch_destroy(b)
    B.oxy_pool_destroy(pool)


def _refusals(pool, b):
    r = B.make_rotary(A, 256)
    return [(B.oxy_mixed_attention, (pool, b, 0, A, A, 0, 0.5, 0)), (B.oxy_mixed_attention_static, (pool, b, 0, A, A, A, 0.5, 0)),
            (B.oxy_stream_append, (pool, b, 5, A, A, 0)), (B.oxy_append_attention, (pool, b, 9, A, A, A, A, 0, 0.5, 0)),
            (B.oxy_append_attention, (pool, b, 0, A, A, A, A, 0, 0.5, 0)),
            (B.oxy_rotary, (B.make_rotary(A, 7), A, A, 4096, A, 4096, 3, 8, 0)),
            (B.oxy_rotary_append, (pool, b, 0, r, A, A, 4096, A, A, 512, A, 512, 0))]


def test_refusals_are_those_of_ctypes(batch, monkeypatch):
    said = []
    for quick in (True, False):
        if not quick:
            for name in [n for n in vars(B._Quick) if n.startswith("oxy_")]:
                monkeypatch.setattr(B._quick, name, B._not_bound)
        for fn, args in _refusals(*batch):
            with pytest.raises(B.OxyError) as e:
                fn(*args)
            said.append((fn.__name__, e.value.code, str(e.value)))
    n = len(said) // 2
    assert said[:n] == said[n:] and all(code == B.ERR_INVALID_ARG for _, code, _ in said)


def test_every_call_is_bound_and_called():
    B.lib()
    for name in [n for n in vars(B._Quick) if n.startswith("oxy_")]:
        assert getattr(B._quick, name) is not B._not_bound, name
    pool = ctypes.c_void_p(0)
    assert B._quick.oxy_mixed_attention(pool, pool, 0, A, A, 0, 0.5, None) == B.ERR_INVALID_ARG
    assert B._quick.oxy_mixed_attention(0, None, 0, A, A, None, 0.5, 0) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("at,value", [
    (0, "x"), (0, 1.5), (2, 1 << 31), (2, -(1 << 31) - 1), (2, np.int32(1)), (2, True), (2, 1.0), (3, -1), (3, 1 << 64), (3, 2.0),
    (3, np.int64(A)), (6, 1), (6, np.float32(0.5)), (6, "1"), (5, object()),
], ids=str)
def test_arguments_of_other_kinds_are_left_to_ctypes(at, value):
    """Nothing is called and no exception is left behind."""
    args = [0, 0, 0, A, A, 0, 0.5, 0]
    args[at] = value
    B.lib()
    assert B._quick.oxy_mixed_attention(*args) is None
    assert B._quick.oxy_mixed_attention(*args[:-1]) is None


def test_without_libmarshal_ctypes_does_it_all(batch, monkeypatch):
    monkeypatch.setattr(B, "MARSHAL_PATH", "/nowhere/libmarshal.so")
    monkeypatch.setattr(B, "_quick", B._Quick())
    B._bind_quick(B.lib())
    assert B._quick.oxy_mixed_attention is B._not_bound
    for fn, args in _refusals(*batch):
        with pytest.raises(B.OxyError):
            fn(*args)
