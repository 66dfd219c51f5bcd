"""Rotary positions with several axes on the GPU: against the float64 oracle, and the append against the calls it stands
for, bit for bit."""
import numpy as np
import pytest

from oracle import prefill
from oracle.attention import widen_bf16
from prefill_util import Pool, bits, down, up

pytestmark = pytest.mark.gpu


class Turn:
    def __init__(self, rot, layout, axis_of_pair, n_axes, amplitude=1.0):
        import torch
        from paper_2603_14371_amd import binding as B
        self.B, self.layout, self.axis, self.n_axes, self.amplitude = B, layout, list(axis_of_pair), n_axes, amplitude
        self.freqs = B.oxy_rotary_freqs(10000.0, rot)[0]
        self.dev = torch.from_numpy(self.freqs).cuda()
        self.cfg = B.make_rotary(self.dev.data_ptr(), rot, {"halves": B.ROTARY_HALVES, "pairs": B.ROTARY_PAIRS}[layout],
                                 amplitude)
        self.map = B.make_rotary_axes(self.axis, n_axes)

    def check(self, x, positions, got):
        """As for one axis: the output's rounding (2^-8 of it), two products and a sum in 32 bits and cosines rounded to
        them (8 x 2^-24 of the products' sizes), an angle off by 2^-51 of it."""
        x = widen_bf16(x)
        ref = prefill.turned(x, positions, self.axis, self.freqs, self.layout, self.amplitude)
        half, rot = len(self.freqs), 2 * len(self.freqs)
        a, b = (slice(0, half), slice(half, rot)) if self.layout == "halves" else (slice(0, rot, 2), slice(1, rot, 2))
        size = np.zeros_like(x)
        size[..., a] = size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
        angle = np.abs(positions).max() * self.freqs.max()
        tol = 2.0 ** -8 * np.abs(ref) + abs(self.amplitude) * size * (2.0 ** -21 + angle * 2.0 ** -51)
        assert np.all(np.abs(widen_bf16(got) - ref) <= tol)
        assert np.array_equal(widen_bf16(got)[..., rot:], x[..., rot:])

    def rotate(self, x, positions, heads, x_stride=None, out=None, out_stride=None):
        import torch
        n = positions.shape[1]
        pos = torch.from_numpy(np.ascontiguousarray(positions, dtype=np.int32)).cuda()
        if out is None:
            out = torch.zeros((n, heads, 256), dtype=torch.int16, device="cuda")
        self.B.oxy_rotary_axes(self.cfg, self.map, pos.data_ptr(), x.data_ptr(), x_stride or heads * 512, out.data_ptr(),
                               out_stride or heads * 512, n, heads, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        return out


def _axes(rng, pairs, n, kind):
    if kind == "sections":
        return np.minimum(np.arange(pairs) * n // pairs, n - 1)
    if kind == "turns":
        return np.arange(pairs) % n
    return rng.integers(0, n, pairs)


@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("rot", [2, 6, 16, 34, 128, 254, 256])
@pytest.mark.parametrize("n_axes", [1, 2, 3, 4])
def test_every_form(layout, rot, n_axes):
    rng = np.random.default_rng(rot * 10 + n_axes)
    for kind, n, heads in (("sections", 5, 9), ("turns", 33, 1), ("random", 1, 8)):
        t = Turn(rot, layout, _axes(rng, rot // 2, n_axes, kind), n_axes, 1.0 if n > 1 else 1.3)
        x = bits(rng, n, heads, 256)
        pos = rng.integers(-5000, 100000, (n_axes, n))
        t.check(x, pos, down(t.rotate(up(x), pos, heads)))


@pytest.mark.parametrize("layout,rot", [("halves", 256), ("pairs", 128), ("halves", 100)])
def test_many_tokens(layout, rot):
    """Four tokens a workgroup, a last one of fewer."""
    rng = np.random.default_rng(rot)
    n = 2051
    t = Turn(rot, layout, _axes(rng, rot // 2, 3, "turns"), 3)
    x, pos = bits(rng, n, 3, 256), rng.integers(0, 1 << 20, (3, n))
    t.check(x, pos, down(t.rotate(up(x), pos, 3)))


def test_one_axis_is_the_plain_rotation():
    import torch
    rng = np.random.default_rng(1)
    t = Turn(256, "halves", [0] * 128, 1)
    same = Turn(256, "halves", _axes(rng, 128, 4, "random"), 4)
    x, pos = up(bits(rng, 70, 9, 256)), rng.integers(0, 1 << 25, (1, 70))
    want = torch.zeros_like(x)
    dev = torch.from_numpy(pos[0].astype(np.int32)).cuda()
    t.B.oxy_rotary(t.cfg, dev.data_ptr(), x.data_ptr(), 9 * 512, want.data_ptr(), 9 * 512, 70, 9,
                   torch.cuda.current_stream().cuda_stream)
    assert np.array_equal(down(t.rotate(x, pos, 9)), down(want))
    assert np.array_equal(down(same.rotate(x, np.repeat(pos, 4, 0), 9)), down(want))


def test_in_place_strided_and_back():
    """Out of a projection's output, in place; negated positions turn back (off by both roundings)."""
    rng = np.random.default_rng(2)
    t = Turn(256, "halves", _axes(rng, 128, 3, "sections"), 3)
    x = bits(rng, 20, 10, 256)
    pos = rng.integers(0, 1000, (3, 20))
    d = up(x)
    t.rotate(d, pos, 9, x_stride=5120, out=d, out_stride=5120)
    got = down(d)
    t.check(x[:, :9], pos, got[:, :9])
    assert np.array_equal(got[:, 9], x[:, 9])
    t.rotate(d, -pos, 9, x_stride=5120, out=d, out_stride=5120)
    a, b = widen_bf16(x[:, :9]), widen_bf16(got[:, :9])
    size = np.abs(b) + np.abs(np.roll(b, 128, axis=-1))       # what the first rounding was of, turned back
    assert np.all(np.abs(widen_bf16(down(d)[:, :9]) - a) <= 2.0 ** -8 * (np.abs(a) + size) * 1.01)


@pytest.mark.parametrize("kv8", [False, True], ids=["bf16", "fp8"])
@pytest.mark.parametrize("layout,rot,n_axes", [("halves", 256, 3), ("pairs", 128, 2), ("halves", 36, 4), ("pairs", 256, 1)])
def test_append(layout, rot, n_axes, kv8):
    """Into prefixes and into streams: the bits of the rotation of queries and keys, and of an append of the turned keys."""
    import torch
    rng = np.random.default_rng(rot + n_axes)
    t = Turn(rot, layout, _axes(rng, rot // 2, n_axes, "random"), n_axes)
    pool = Pool(2, 64, kv8, seed=1)
    B = pool.B
    try:
        for what in ("prefix", "stream"):
            sizes = [5, 16, 41]
            n = sum(sizes)
            x = bits(rng, n, 10, 256)
            pos = rng.integers(0, 5000, (n_axes, n))
            d, dpos = up(x), torch.from_numpy(pos.astype(np.int32)).cuda()
            turned = t.rotate(d, pos, 9, x_stride=5120)
            got = []
            for fused in (False, True):
                if what == "prefix":
                    ids = [B.oxy_prefix_create(pool.p) for _ in sizes]
                    batch = B.oxy_prefix_batch_build(pool.p, [(i, m, 0) for i, m in zip(ids, sizes)], B.BATCH_APPEND_ONLY,
                                                     pool.stream)
                else:
                    ids = [B.oxy_stream_create(pool.p, -1, B.KIND_DECODE) for _ in sizes]
                    batch = B.oxy_batch_build(pool.p, list(zip(ids, sizes)), B.BATCH_APPEND_ONLY, pool.stream)
                q_out = torch.zeros((n, 8, 256), dtype=torch.int16, device="cuda")
                if fused:
                    a = d.data_ptr()
                    B.oxy_rotary_axes_append(pool.p, batch, 1, t.cfg, t.map, dpos.data_ptr(), a, 5120, q_out.data_ptr(),
                                             a + 4096, 5120, a + 4608, 5120, pool.stream)
                else:
                    k, v = turned[:, 8].contiguous(), d[:, 9].contiguous()
                    q_out.copy_(turned[:, :8])
                    B.oxy_stream_append(pool.p, batch, 1, k.data_ptr(), v.data_ptr(), pool.stream)
                back = torch.zeros((2, n, 256), dtype=torch.int16, device="cuda")
                B.oxy_gather_kv(pool.p, 1, B.oxy_batch_slots(batch), back[0].data_ptr(), back[1].data_ptr(), pool.stream)
                got.append((down(q_out), down(back)))
                B.oxy_batch_destroy(batch)
                for i in ids:
                    (B.oxy_prefix_release if what == "prefix" else B.oxy_stream_release)(pool.p, i)
            assert np.array_equal(got[0][0], got[1][0]) and np.array_equal(got[0][1], got[1][1])
            t.check(x[:, :8], pos, got[1][0])
    finally:
        pool.close()


@pytest.mark.parametrize("kv8", [False, True], ids=["bf16", "fp8"])
@pytest.mark.parametrize("n_axes", [0, 3])
@pytest.mark.parametrize("n", [127, 128, 129, 255, 256, 300, 1100])
def test_append_of_whole_rounds_and_others(n, n_axes, kv8):
    """Around multiples of 128 tokens, from which on they run in another order; n_axes 0: the call of one axis."""
    import torch
    rng = np.random.default_rng(n)
    t = Turn(256, "halves", _axes(rng, 128, max(n_axes, 1), "turns"), max(n_axes, 1))
    pool = Pool(1, 160, kv8, seed=2, max_q_tokens=1200, max_append_tokens=1200)
    B = pool.B
    try:
        x = bits(rng, n, 10, 256)
        pos = rng.integers(0, 5000, (max(n_axes, 1), n))
        d, dpos = up(x), torch.from_numpy(pos.astype(np.int32)).cuda()
        turned = t.rotate(d, pos, 9, x_stride=5120)
        got = []
        for fused in (False, True):
            pid = pool.prefix(bits(np.random.default_rng(1), 5, 256), bits(np.random.default_rng(2), 5, 256))
            batch = B.oxy_prefix_batch_build(pool.p, [(pid, n, 0)], B.BATCH_APPEND_ONLY, pool.stream)
            q_out = torch.zeros((n + 1, 8, 256), dtype=torch.int16, device="cuda")
            rows = (d.data_ptr(), 5120, q_out.data_ptr(), d.data_ptr() + 4096, 5120, d.data_ptr() + 4608, 5120, pool.stream)
            if fused and n_axes:
                B.oxy_rotary_axes_append(pool.p, batch, 0, t.cfg, t.map, dpos.data_ptr(), *rows)
            elif fused:
                B.oxy_rotary_append(pool.p, batch, 0, t.cfg, dpos.data_ptr(), *rows)
            else:
                k, v = turned[:, 8].contiguous(), d[:, 9].contiguous()
                q_out[:n].copy_(turned[:, :8])
                B.oxy_stream_append(pool.p, batch, 0, k.data_ptr(), v.data_ptr(), pool.stream)
            back = torch.zeros((2, n, 256), dtype=torch.int16, device="cuda")
            B.oxy_gather_kv(pool.p, 0, B.oxy_batch_slots(batch), back[0].data_ptr(), back[1].data_ptr(), pool.stream)
            got.append((down(q_out), down(back)))
            B.oxy_batch_destroy(batch)
            B.oxy_prefix_release(pool.p, pid)
        assert np.array_equal(got[0][0], got[1][0]) and np.array_equal(got[0][1], got[1][1])
    finally:
        pool.close()
