"""Pins of the oracles of 8-bit rows and rotary positions, and what the library decides on the host about
both: sizes, indexing, frequencies, refusals.  No GPU."""
import math

import numpy as np
import pytest

from oracle import kv8, rotary
from oracle.attention import widen_bf16
from oracle.pool_model import PoolModel
from paper_2603_14371_amd import binding as B


def _bits(x):
    return (np.asarray(x, dtype=np.float32).view(np.uint32) >> 16).astype(np.uint16)


def test_grid_is_e4m3():
    assert kv8._GRID[-1] == 448.0 and kv8._GRID[1] == 2.0 ** -9 and kv8._GRID[8] == 2.0 ** -6
    assert np.all(np.diff(kv8._GRID) > 0) and len(kv8._GRID) == 127
    torch = pytest.importorskip("torch")
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn)
    assert np.array_equal(codes.double().numpy(), kv8._GRID)


def test_nearest_code_against_a_cast():
    torch = pytest.importorskip("torch")
    every = widen_bf16(np.arange(0x7f80, dtype=np.uint16))      # every finite magnitude of bf16
    y = every[every <= 448.0]
    want = torch.from_numpy(y.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(kv8.nearest_code(y), want)


@pytest.mark.parametrize("top,e", [(448.0, 0), (449.0, 1), (1.75, -8), (1.7578125, -7), (1.0, -8), (2.0, -7),
                                   (0.0, -126), (2.0 ** -133, -126), (448 * 2.0 ** -126, -126),
                                   (450 * 2.0 ** -126, -125), (3.3895e38, 120)])
def test_row_exponent(top, e):
    row = np.zeros(256)
    row[3], row[9] = -top, top / 2
    assert kv8.row_exponent(row) == e
    row[5], row[6] = np.inf, np.nan
    assert kv8.row_exponent(row) == e


def test_cached_values_are_close_and_hold_still():
    """Half a step of e4m3 is 2^-4 of a value (2^-10 of its row's scale below the normal range), and what was
    held once is held again as it is."""
    rng = np.random.default_rng(5)
    x = rng.standard_normal((40, 256)) * 2.0 ** rng.integers(-30, 30, (40, 1))
    bits = _bits(x)
    x = widen_bf16(bits)
    y = kv8.cached_values(bits)
    unit = 2.0 ** np.array([kv8.row_exponent(r) for r in x])[:, None]
    assert np.all(np.abs(y - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * unit))
    assert np.array_equal(kv8.cached_values(kv8.bf16_bits(y)), y)


def test_rotation_of_a_single_pair_and_of_negated_positions():
    x = np.random.default_rng(1).standard_normal((3, 2, 256))
    f = np.array([0.5])
    for layout, (i, j) in (("halves", (0, 1)), ("pairs", (0, 1))):
        y = rotary.turned(x, [0, 1, 7], f, layout, 2.0)
        c, s = 2 * math.cos(3.5), 2 * math.sin(3.5)
        assert np.allclose(y[2, 1, i], x[2, 1, i] * c - x[2, 1, j] * s)
        assert np.allclose(y[2, 1, j], x[2, 1, j] * c + x[2, 1, i] * s)
        assert np.array_equal(y[:, :, 2:], x[:, :, 2:]) and np.allclose(y[0, :, :2], 2 * x[0, :, :2])
    f = rotary.frequencies(10000.0, 100)[0]
    for layout in ("halves", "pairs"):
        y = rotary.turned(x, [3, 1000, 5], f, layout)
        assert np.allclose(rotary.turned(y, [-3, -1000, -5], f, layout), x)


KINDS = {"plain": B.ROTARY_PLAIN, "linear": B.ROTARY_LINEAR, "base": B.ROTARY_BASE, "bands": B.ROTARY_BANDS,
         "ramp": B.ROTARY_RAMP}


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("rot", [2, 6, 64, 100, 256])
@pytest.mark.parametrize("factor,original", [(1.0, 4096), (8.0, 8192), (2.5, 1)])
def test_frequencies(kind, rot, factor, original):
    low, high = (1.0, 32.0) if kind == "ramp" else (1.0, 4.0)
    got, amplitude = B.oxy_rotary_freqs(10000.0, rot, KINDS[kind], factor, low, high, original)
    want, want_amplitude = rotary.frequencies(10000.0, rot, kind, factor, low, high, original)
    # a power of up to 2e4 in 64 bits: its exponent's rounding, times ln(1e4 * 8)
    assert np.allclose(got, want, rtol=1e-14 * 12, atol=0) and abs(amplitude - want_amplitude) < 1e-14
    if factor == 1.0:
        assert np.allclose(got, rotary.frequencies(10000.0, rot)[0], rtol=2e-13, atol=0)


def _refused(fn, *args, **kw):
    with pytest.raises(B.OxyError) as e:
        fn(*args, **kw)
    assert e.value.code == B.ERR_INVALID_ARG, e.value
    assert str(e.value)


@pytest.mark.parametrize("kw", [
    dict(rot_dims=0), dict(rot_dims=-2), dict(rot_dims=7), dict(rot_dims=258), dict(base=0.0), dict(base=math.nan),
    dict(base=math.inf), dict(kind=-1), dict(kind=5), dict(kind=1, factor=0.5), dict(kind=2, factor=math.nan),
    dict(kind=3, factor=2.0, low=1.0, high=1.0, original_len=100), dict(kind=3, factor=2.0, low=0.0, high=1.0, original_len=9),
    dict(kind=4, factor=2.0, low=1.0, high=4.0, original_len=0), dict(kind=4, base=1.0, factor=2.0, low=1.0, high=4.0, original_len=9),
    dict(kind=4, factor=2.0, low=1.0, high=math.inf, original_len=9),
], ids=str)
def test_frequencies_refuse(kw):
    _refused(B.oxy_rotary_freqs, **dict(dict(base=10000.0, rot_dims=64), **kw))


A16 = 1 << 20     # an aligned address that no refused call reads


@pytest.mark.parametrize("kw", [
    dict(rot=0), dict(rot=3), dict(rot=512), dict(layout=2), dict(layout=-1), dict(freqs=0), dict(positions=0), dict(x=0),
    dict(out=0), dict(x=A16 + 2), dict(out=A16 + 8), dict(x_stride=4096 + 8), dict(x_stride=4096 - 16),
    dict(out_stride=512), dict(n=(1 << 25) + 1), dict(out_stride=8192), dict(n=-1), dict(heads=0), dict(heads=1025, x_stride=1 << 20, out_stride=1 << 20),
], ids=str)
def test_rotary_refuses(kw):
    a = dict(dict(rot=256, layout=0, freqs=A16, positions=A16, x=A16, out=A16, x_stride=4096, out_stride=4096, n=4,
                  heads=8), **kw)
    r = B.make_rotary(a["freqs"], a["rot"], a["layout"])
    _refused(B.oxy_rotary, r, a["positions"], a["x"], a["x_stride"], a["out"], a["out_stride"], a["n"], a["heads"], 0)


def test_rotary_of_no_tokens_does_nothing():
    B.oxy_rotary(B.make_rotary(A16, 256), A16, A16, 4096, A16, 4096, 0, 8, 0)


def test_host_only_pools_refuse_device_work():
    cfg = B.make_config(2, 8, flags=B.POOL_HOST_ONLY | B.POOL_KV_FP8)
    pool = B.oxy_pool_create(cfg)
    sid = B.oxy_stream_create(pool, -1, B.KIND_DECODE)
    batch = B.oxy_batch_build(pool, [(sid, 3)], 0, 0)
    r = B.make_rotary(A16, 256)
    _refused(B.oxy_rotary_append, pool, batch, 0, r, A16, A16, 4096, A16, A16, 512, A16, 512, 0)
    _refused(B.oxy_gather_kv_layers, pool, 0, 2, [0, 1], A16, A16, 1024, 0)
    B.oxy_batch_destroy(batch)
    B.oxy_pool_destroy(pool)


def test_sizes_of_a_pool_in_8_bits():
    """Per layer 8 KiB of codes and 32 exponent bytes a block, rounded up to 256 bytes."""
    for layers, blocks in ((1, 1), (3, 7), (18, 8192)):
        cfg = B.make_config(layers, blocks, flags=B.POOL_KV_FP8)
        assert B.oxy_kv_bytes(cfg) == layers * (-(-blocks * 8224 // 256) * 256)
        assert B.oxy_workspace_bytes(cfg) == B.oxy_workspace_bytes(B.make_config(layers, blocks))
    cfg = B.make_config(2, 8, flags=B.POOL_KV_FP8, kv_base=A16, kv_bytes=2 * 8 * 8224 - 1, workspace=A16,
                        workspace_bytes=1 << 40)
    _refused(B.oxy_pool_create, cfg)


def test_indexing_of_a_pool_in_8_bits_is_that_of_any_pool():
    rng = np.random.default_rng(8)
    nb = 64
    order = rng.permutation(nb).tolist()
    model = PoolModel(nb, 16, 2, order)
    pool = B.oxy_pool_create(B.make_config(2, nb, free_order=order, flags=B.POOL_HOST_ONLY | B.POOL_KV_FP8))
    pid, mid = B.oxy_prefix_create(pool), model.prefix_create()
    assert pid == mid
    for layer in range(2):
        B.oxy_prefix_append(pool, pid, layer, 0, 0, 70, 0, 0)
        model.prefix_append(mid, layer, 70, 0)
    sids = [B.oxy_stream_create(pool, pid, k) for k in (B.KIND_ACTION, B.KIND_DECODE)]
    assert sids == [model.stream_create(mid, k) for k in (0, 1)]
    for step in range(6):
        items = [(sids[0], 50), (sids[1], 1 + step % 3)]
        batch = B.oxy_batch_build(pool, items, 0, 0)
        assert B.oxy_batch_slots(batch) == model.batch_build(items)
        B.oxy_batch_destroy(batch)
    assert B.oxy_free_blocks(pool) == model.free[::-1]
    B.oxy_pool_destroy(pool)
