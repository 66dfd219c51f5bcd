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
            (B.oxy_rotary_append, (pool, b, 0, r, A, A, 4096, A, A, 512, A, 512, 0)),
            (B.oxy_gather_kv, (pool, 0, [0, 1], A, A, 0)), (B.oxy_gather_kv, (pool, 7, [0], A, A, 0)),
            (B.oxy_gather_kv, (pool, 0, [], A, A, 0)), (B.oxy_gather_kv, (None, 0, [1], A, A, 0)),
            (B.oxy_gather_kv_layers, (pool, 0, 2, [0, 1], A, A, 1024, 0)), (B.oxy_batch_slots, (None,)),
            (B.oxy_batch_info, (None,))]


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


def test_what_a_batch_answers_is_what_ctypes_gets(monkeypatch):
    pool = B.oxy_pool_create(B.make_config(2, 200, flags=B.POOL_HOST_ONLY))
    sids = [B.oxy_stream_create(pool, -1, B.KIND_DECODE) for _ in range(3)]
    for items in ([(sids[0], 1)], [(sids[1], 700), (sids[2], 900)]):
        b = B.oxy_batch_build(pool, items, B.BATCH_APPEND_ONLY, 0)
        quick = B.oxy_batch_info(b), B.oxy_batch_slots(b)
        assert B._quick.oxy_batch_info(b) == quick[0] and B._quick.oxy_batch_slots(b, quick[0][1]) == quick[1]
        assert B._quick.oxy_batch_slots(b, quick[0][1] - 1) is None and B._quick.oxy_batch_slots(b, 0) is None
        with monkeypatch.context() as m:
            m.setattr(B, "_quick", B._Quick())
            assert (B.oxy_batch_info(b), B.oxy_batch_slots(b)) == quick
        assert type(quick[1]) is list and all(type(x) is int for x in quick[1])
        assert len(quick[1]) == sum(n for _, n in items)
        B.oxy_batch_destroy(b)
    B.oxy_pool_destroy(pool)


@pytest.mark.parametrize("slots", [(1, 2), [1.0], [True], [np.int64(3)], [1 << 63], ["1"], [None], np.arange(3)], ids=str)
def test_slots_of_other_kinds_are_left_to_ctypes(slots):
    B.lib()
    assert B._quick.oxy_gather_kv(0, 0, slots, A, A, 0) is None
    assert B._quick.oxy_gather_kv_layers(0, 0, 1, slots, A, A, 512, 0) is None
    assert B._quick.oxy_gather_kv(0, 0, [1], A, A, 0) == B.ERR_INVALID_ARG
    assert B._quick.oxy_gather_kv(0, "0", [1], A, A, 0) is None and B._quick.oxy_gather_kv(0, 0, [1], A, A) is None
    assert B._quick.oxy_gather_kv_layers(0, 0, 1, [1], A, A, 512, 0) == B.ERR_INVALID_ARG
    assert B._quick.oxy_gather_kv_layers(0, 0, 1, [1], A, A, -1, 0) is None
