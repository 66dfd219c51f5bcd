"""Batches of a prefill on a host-only pool against the pool model, refusals, and pins of the oracle.  No GPU."""
import ctypes

import numpy as np
import pytest

from oracle import attention, prefill, rotary
from oracle.pool_model import PoolModel
from paper_2603_14371_amd import binding as B

A = 1 << 20      # an aligned address that no refused call reads


def refused(code, fn, *args):
    with pytest.raises(B.OxyError) as e:
        fn(*args)
    assert e.value.code == code, str(e.value)


def host_pool(blocks=64, layers=2, **kw):
    return B.oxy_pool_create(B.make_config(layers, blocks, flags=B.POOL_HOST_ONLY | kw.pop("flags", 0), **kw))


def same(pool, model, blocks):
    assert B.oxy_block_refcounts(pool, blocks) == list(model.ref)
    assert B.oxy_free_blocks(pool) == model.free[::-1]
    for pid, px in model.prefixes.items():
        assert B.oxy_prefix_info(pool, pid)[0] == px.length and list(B.oxy_prefix_blocks(pool, pid)) == list(px.blocks)


@pytest.mark.parametrize("seed", range(6))
def test_blocks_are_taken_as_by_appends(seed):
    rng = np.random.default_rng(seed)
    blocks = 120
    order = rng.permutation(blocks)
    pool, model = host_pool(blocks, free_order=order), PoolModel(blocks, 16, 2, order.tolist())
    pids = []
    for _ in range(60):
        r = rng.random()
        if r < 0.25 or not pids:
            pids.append(B.oxy_prefix_create(pool))
            assert model.prefix_create() == pids[-1]
        elif r < 0.35:
            parent = int(rng.choice(pids))
            n = model.prefixes[parent].length // 16 * 16
            pids.append(B.oxy_prefix_fork(pool, parent, n))
            assert model.prefix_fork(parent, n) == pids[-1]
        elif r < 0.45:
            pid = pids.pop(int(rng.integers(len(pids))))
            B.oxy_prefix_release(pool, pid)
            model.prefix_release(pid)
        else:
            some = [int(p) for p in rng.permutation(pids)[:int(rng.integers(1, 4))]]
            items = [(p, int(rng.integers(1, 70)), int(rng.integers(0, 200))) for p in some]
            need = sum(-(-(model.prefixes[p].length + n) // 16) - len(model.prefixes[p].blocks) for p, n, _ in items)
            if need > len(model.free):
                refused(B.ERR_NO_BLOCKS, B.oxy_prefix_batch_build, pool, items, 0, 0)
            else:
                b = B.oxy_prefix_batch_build(pool, items, 0 if rng.random() < 0.7 else B.BATCH_APPEND_ONLY, 0)
                slots = []
                for p, n, _ in items:
                    at = model.prefixes[p].length
                    model.prefix_append(p, 0, n, at)
                    slots += [model.prefixes[p].blocks[t // 16] * 16 + t % 16 for t in range(at, at + n)]
                assert B.oxy_batch_slots(b) == slots and B.oxy_batch_info(b)[:2] == (len(items), len(slots))
                B.oxy_batch_destroy(b)
        same(pool, model, blocks)
    B.oxy_pool_destroy(pool)


def test_refusals_of_the_builds():
    pool = host_pool(8, max_q_tokens=40, max_append_tokens=60, max_live_batches=1)
    a, b, sealed = (B.oxy_prefix_create(pool) for _ in range(3))
    B.oxy_prefix_append(pool, sealed, 0, 0, 0, 16, 0, 0)
    sid = B.oxy_stream_create(pool, sealed, B.KIND_DECODE)
    before = B.oxy_free_blocks(pool)
    build = lambda items, flags=0: B.oxy_prefix_batch_build(pool, items, flags, 0)  # noqa: E731
    bad = B.ERR_INVALID_ARG
    refused(bad, build, [])
    refused(bad, B.oxy_prefix_batch_build, None, [(a, 1, 0)], 0, 0)
    refused(bad, build, [(a, 1, 0)], 2)
    for n, full in ((0, 0), (-1, 0), (1, -1)):
        refused(bad, build, [(b, 1, 0), (a, n, full)])
    refused(bad, build, [(a, 1, 0), (b, 1, 0), (a, 1, 0)])
    refused(B.ERR_BAD_ID, build, [(a, 1, 0), (77, 1, 0)])
    refused(B.ERR_SEALED, build, [(a, 1, 0), (sealed, 1, 0)])
    refused(B.ERR_WORKSPACE, build, [(a, 41, 0)])
    refused(B.ERR_WORKSPACE, build, [(a, 61, 0)], B.BATCH_APPEND_ONLY)
    refused(B.ERR_NO_BLOCKS, build, [(a, 113, 0)])
    refused(B.ERR_NO_BLOCKS, build, [(a, 2**31 - 1, 0)])
    assert B.oxy_free_blocks(pool) == before and B.oxy_prefix_info(pool, a)[:2] == (0, 0)
    batch = build([(a, 60, 0)], B.BATCH_APPEND_ONLY)
    refused(B.ERR_BUSY, build, [(b, 1, 0)])
    assert B.oxy_prefix_info(pool, b)[:2] == (0, 0)
    refused(B.ERR_BUSY, B.oxy_prompt_batch_build, pool, [(3, 0)], 0)
    B.oxy_batch_destroy(batch)
    refused(bad, B.oxy_prompt_batch_build, pool, [], 0)
    refused(bad, B.oxy_prompt_batch_build, None, [(1, 0)], 0)
    refused(bad, B.oxy_prompt_batch_build, pool, [(1, 0), (-1, 0)], 0)
    refused(bad, B.oxy_prompt_batch_build, pool, [(1, -1)], 0)
    refused(B.ERR_WORKSPACE, B.oxy_prompt_batch_build, pool, [(20, 0), (21, 0)], 0)
    refused(B.ERR_WORKSPACE, B.oxy_prompt_batch_build, pool, [(2**31 - 1, 0), (2**31 - 1, 0)], 0)
    B.oxy_prefix_release(pool, b)
    refused(B.ERR_BAD_ID, build, [(b, 1, 0)])
    B.oxy_stream_release(pool, sid)
    B.oxy_pool_destroy(pool)


def test_too_few_work_items():
    """What cannot be cut into fewer records is refused and changes nothing."""
    pool = host_pool(64, max_work_items=3)
    pid = B.oxy_prefix_create(pool)
    refused(B.ERR_WORKSPACE, B.oxy_prefix_batch_build, pool, [(pid, 49, 0)], 0, 0)
    assert B.oxy_prefix_info(pool, pid)[:2] == (0, 0) and len(B.oxy_free_blocks(pool)) == 64
    b = B.oxy_prefix_batch_build(pool, [(pid, 48, 900)], 0, 0)
    assert B.oxy_batch_info(b) == (1, 48, 3, 0)
    B.oxy_batch_destroy(b)
    B.oxy_pool_destroy(pool)


def test_refusals_of_the_calls():
    """A host-only pool refuses everything that would touch the device; the messages say what is wrong first."""
    pool = host_pool()
    pid = B.oxy_prefix_create(pool)
    b = B.oxy_prefix_batch_build(pool, [(pid, 5, 0)], 0, 0)
    c = B.oxy_prompt_batch_build(pool, [(5, 0)], 0)
    refused(B.ERR_INVALID_ARG, B.oxy_prefix_attention, pool, b, 0, A, 4096, A, 4096, 0, 1.0, 0)
    refused(B.ERR_INVALID_ARG, B.oxy_prompt_attention, pool, c, A, 4096, A, 512, A, 512, A, 4096, 0, 1.0, 0)
    refused(B.ERR_INVALID_ARG, B.oxy_batch_slots, c)
    refused(B.ERR_INVALID_ARG, B.oxy_batch_work, b)
    refused(B.ERR_INVALID_ARG, B.oxy_batch_records, c)
    B.oxy_batch_destroy(b)
    B.oxy_batch_destroy(c)
    B.oxy_pool_destroy(pool)


def test_rotary_axes_refusals():
    good = B.make_rotary(A, 8), B.make_rotary_axes([0, 1, 2, 0], 3)
    call = lambda cfg, axes, *args: B.oxy_rotary_axes(cfg, axes, *args)  # noqa: E731
    rows = (A, A, 4096, 2 * A, 4096, 3, 8, 0)
    bad = B.ERR_INVALID_ARG
    for axes in (B.make_rotary_axes([0, 1, 3, 0], 3), B.make_rotary_axes([0, 1, 2, 0], 0), B.make_rotary_axes([0, 1, 2, 0], 5),
                 B.make_rotary_axes([0, 0, 0, 0], -1), B.make_rotary_axes([0, 0, 0, 255], 4), B.RotaryAxisMap(3, None)):
        refused(bad, call, good[0], axes, *rows)
    for rot in (0, 7, 258, -2):
        refused(bad, call, B.make_rotary(A, rot), good[1], *rows)
    refused(bad, call, B.make_rotary(0, 8), good[1], *rows)
    refused(bad, call, good[0], good[1], 0, *rows[1:])
    refused(bad, call, good[0], good[1], A, A + 8, *rows[2:])
    refused(bad, call, good[0], good[1], A, A, 4080, *rows[3:])
    refused(bad, call, good[0], good[1], A, A, 4096, A, 5120, 3, 8, 0)
    refused(bad, call, good[0], good[1], *rows[:5], -1, 8, 0)
    refused(bad, call, good[0], good[1], *rows[:6], 0, 0)
    call(good[0], good[1], 0, 0, 1, 0, 3, 0, 8, 0)          # no tokens: nothing to do
    pool = host_pool()
    pid = B.oxy_prefix_create(pool)
    b = B.oxy_prefix_batch_build(pool, [(pid, 5, 0)], 0, 0)
    refused(bad, B.oxy_rotary_axes_append, pool, b, 0, good[0], good[1], A, A, 5120, A, A, 5120, A, 5120, 0)
    refused(bad, B.oxy_rotary_axes_append, pool, b, 0, good[0], B.make_rotary_axes([4] * 4, 4), A, A, 5120, A, A, 5120, A, 5120, 0)
    B.oxy_batch_destroy(b)
    B.oxy_pool_destroy(pool)


def test_wrong_argument_types_are_those_of_ctypes():
    with pytest.raises((ctypes.ArgumentError, TypeError)):
        B.oxy_prefix_attention(None, None, "0", A, 4096, A, 4096, 0, 1.0, 0)
    with pytest.raises((ctypes.ArgumentError, TypeError)):
        B.oxy_prompt_attention(None, None, A, 4096.5, A, 512, A, 512, A, 4096, 0, 1.0, 0)


def test_oracle_of_the_attention():
    """Causal: what a decode stream sees on a prefix; all: an action chunk; between: row by row from the definition."""
    rng = np.random.default_rng(0)
    past, n, d = 7, 6, 16
    raw = lambda *s: (rng.standard_normal(s).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)  # noqa: E731
    q, k, v = raw(n, 8, d), raw(past + n, d), raw(past + n, d)
    wide = [attention.widen_bf16(x) for x in (q, k, v)]
    for kind, full in ((attention.DECODE, 0), (attention.ACTION, past + n), (attention.ACTION, 10**6)):
        o, lse = attention.attend_item(kind, q, k[:past], v[:past], k[past:], v[past:], 0.3)
        got = prefill.attend(*wide, past, full, 0.3)
        assert np.allclose(o, got[0], atol=1e-12) and np.allclose(lse, got[1], atol=1e-12)
    got = prefill.attend(*wide, past, 10, 0.3)
    for i in range(n):
        m = max(past + i + 1, 10)
        o, lse = attention.softmax_attend(wide[0][i], wide[1][:m], wide[2][:m], 0.3)
        assert np.allclose(o, got[0][i], atol=1e-12) and np.allclose(lse, got[1][i], atol=1e-12)
        assert np.all(got[2][i] >= np.abs(o) - 1e-12)
    assert list(prefill.sees(3, 4, 0)) == [4, 5, 6, 7] and list(prefill.sees(0, 3, 2)) == [2, 2, 3]
    assert list(prefill.sees(2, 2, 99)) == [4, 4]


def test_oracle_of_the_rotation():
    rng = np.random.default_rng(1)
    x, freqs = rng.standard_normal((5, 3, 32)), rng.random(12)
    pos = rng.integers(0, 100, (3, 5))
    axis = rng.integers(0, 3, 12)
    for layout in ("halves", "pairs"):
        each = [rotary.turned(x, pos[a], freqs, layout, 1.5) for a in range(3)]
        got = prefill.turned(x, pos, axis, freqs, layout, 1.5)
        for i in range(12):
            pair = (i, i + 12) if layout == "halves" else (2 * i, 2 * i + 1)
            assert np.allclose(got[..., pair], each[axis[i]][..., pair], atol=1e-12)
        assert np.array_equal(got[..., 24:], x[..., 24:])
