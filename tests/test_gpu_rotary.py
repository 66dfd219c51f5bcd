"""Rotary positions on the GPU against the float64 oracle, and the rotating append against the calls it
stands for, bit for bit."""
import numpy as np
import pytest

from oracle import kv8, rotary
from oracle.attention import widen_bf16
from oracle.replay import OracleWorld
from paper_2603_14371_amd import synth
from paper_2603_14371_amd.synth import ACTION, DECODE
from parity_util import assert_lse_close, assert_o_close

pytestmark = pytest.mark.gpu


def _bits(rng, *shape):
    x = rng.standard_normal(shape).astype(np.float32)
    return (x.view(np.uint32) >> 16).astype(np.uint16)


def _up(bits):
    import torch
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda()


def _down(t):
    import torch
    torch.cuda.synchronize()
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


class Turn:
    """Frequencies on the device with their configuration."""

    def __init__(self, rot, layout, base=10000.0, amplitude=None, **kw):
        import torch
        from paper_2603_14371_amd import binding as B
        self.layout = layout
        self.freqs, self.amplitude = B.oxy_rotary_freqs(base, rot, **kw)
        self.amplitude = self.amplitude if amplitude is None else amplitude
        self.dev = torch.from_numpy(self.freqs).cuda()
        self.cfg = B.make_rotary(self.dev.data_ptr(), rot, {"halves": B.ROTARY_HALVES, "pairs": B.ROTARY_PAIRS}[layout],
                                 self.amplitude)

    def check(self, bits, positions, got):
        """got [n, heads, 256] bits.  An output is a rounding to bf16 (half a step, 2^-8 of it), behind two products and
        a sum of 32-bit numbers of 2^-24 each and cosines rounded to 2^-24 (8 x 2^-24 of the products' sizes together), of
        an angle whose error is 2^-51 of it at most (frequency times position times 1 / 2 pi, each 2^-53)."""
        x = widen_bf16(bits)
        ref = rotary.turned(x, positions, self.freqs, self.layout, self.amplitude)
        rot, half = 2 * len(self.freqs), len(self.freqs)
        size = np.zeros_like(x)
        if self.layout == "halves":
            size[..., :half] = size[..., half:rot] = np.abs(x[..., :half]) + np.abs(x[..., half:rot])
        else:
            size[..., 0:rot:2] = size[..., 1:rot:2] = np.abs(x[..., 0:rot:2]) + np.abs(x[..., 1:rot:2])
        angle = np.abs(np.asarray(positions, dtype=np.float64)).max() * self.freqs.max()
        tol = 2.0 ** -8 * np.abs(ref) + abs(self.amplitude) * size * (2.0 ** -21 + angle * 2.0 ** -51)
        assert np.all(np.abs(widen_bf16(got) - ref) <= tol)
        assert np.array_equal(got[..., rot:], bits[..., rot:])      # copied


def _rotate(turn, x, positions, n, heads, x_stride=None, out=None, out_stride=None):
    import torch
    from paper_2603_14371_amd import binding as B
    pos = torch.tensor(np.asarray(positions, dtype=np.int32), device="cuda")
    if out is None:
        out = torch.zeros((n, heads, 256), dtype=torch.int16, device="cuda")
    B.oxy_rotary(turn.cfg, pos.data_ptr(), x.data_ptr(), x_stride or heads * 512, out.data_ptr(),
                 out_stride or heads * 512, n, heads, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("rot", [2, 6, 14, 16, 32, 34, 100, 128, 240, 254, 256])
def test_part_of_the_head(layout, rot):
    rng = np.random.default_rng(rot)
    turn = Turn(rot, layout)
    for n, heads in ((1, 1), (1, 8), (3, 1), (5, 9), (4, 2), (33, 3)):
        bits, pos = _bits(rng, n, heads, 256), rng.integers(0, 5000, n)
        turn.check(bits, pos, _down(_rotate(turn, _up(bits), pos, n, heads)))


@pytest.mark.parametrize("layout", ["halves", "pairs"])
def test_far_and_negative_positions(layout):
    rng = np.random.default_rng(2)
    turn = Turn(256, layout)
    pos = np.array([0, 1, -1, 65536, 1 << 20, (1 << 20) + 1, -(1 << 20), 2**31 - 1, -2**31])
    bits = _bits(rng, len(pos), 4, 256)
    turn.check(bits, pos, _down(_rotate(turn, _up(bits), pos, len(pos), 4)))
    assert np.array_equal(_down(_rotate(turn, _up(bits), [0] * 9, 9, 4)), bits)       # no turn, no change


@pytest.mark.parametrize("kind", [0, 1, 2, 3, 4])
def test_scaled_contexts(kind):
    rng = np.random.default_rng(kind)
    turn = Turn(128, "halves", kind=kind, factor=8.0, low=1.0, high=32.0, original_len=4096)
    pos = rng.integers(0, 32768, 40)
    bits = _bits(rng, 40, 2, 256)
    turn.check(bits, pos, _down(_rotate(turn, _up(bits), pos, 40, 2)))


@pytest.mark.parametrize("layout,rot", [("halves", 256), ("halves", 100), ("pairs", 128)])
def test_views_of_a_projection_and_in_place(layout, rot):
    """Rows out of a wider row into a wider row: what lies between them stays; and onto themselves."""
    import torch
    rng = np.random.default_rng(3)
    turn = Turn(rot, layout)
    n, pos = 21, rng.integers(0, 9000, 21)
    wide = _bits(rng, n, 10, 256)
    x = _up(wide)
    out = torch.full((n, 12, 256), 77, dtype=torch.int16, device="cuda")
    _rotate(turn, x[:, 2:], pos, n, 5, 10 * 512, out[:, 1:], 12 * 512)
    got = _down(out)
    turn.check(wide[:, 2:7], pos, got[:, 1:6])
    assert np.all(got[:, :1] == 77) and np.all(got[:, 6:] == 77) and np.array_equal(_down(x), wide)
    _rotate(turn, x, pos, n, 9, 10 * 512, x, 10 * 512)
    turn.check(wide[:, :9], pos, _down(x)[:, :9])
    assert np.array_equal(_down(x)[:, 9], wide[:, 9])


def test_many_tokens_and_heads():
    rng = np.random.default_rng(4)
    turn = Turn(256, "halves", amplitude=1.25)
    for n, heads in ((4099, 1), (517, 40), (2, 1024)):
        bits, pos = _bits(rng, n, heads, 256), np.arange(n) + 17
        turn.check(bits, pos, _down(_rotate(turn, _up(bits), pos, n, heads)))


def test_numbers_that_are_not_finite_stay_in_their_pair():
    rng = np.random.default_rng(5)
    turn = Turn(256, "halves")
    bits = _bits(rng, 2, 1, 256)
    bits[0, 0, 5], bits[1, 0, 200] = 0x7f80, 0x7fc0
    got = widen_bf16(_down(_rotate(turn, _up(bits), [3, 4], 2, 1)))
    bad = ~np.isfinite(got)
    assert bad.sum() == 4 and bad[0, 0, [5, 133]].all() and bad[1, 0, [72, 200]].all()


def _pool(bits8, n_layers=2, blocks=64, max_tokens=512):
    import torch
    from paper_2603_14371_amd import binding as B
    cfg = B.make_config(n_layers, blocks, flags=B.POOL_KV_FP8 if bits8 else 0, max_q_tokens=max_tokens,
                        max_append_tokens=max_tokens)
    kv = torch.full((B.oxy_kv_bytes(cfg),), 0xFF, dtype=torch.uint8, device="cuda")
    ws = torch.empty(B.oxy_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    cfg.kv_base, cfg.kv_bytes = kv.data_ptr(), kv.numel()
    cfg.workspace, cfg.workspace_bytes = ws.data_ptr(), ws.numel()
    return B.oxy_pool_create(cfg), (kv, ws)


@pytest.mark.parametrize("bits8", [True, False], ids=["kv8", "bf16"])
@pytest.mark.parametrize("layout,rot", [("halves", 256), ("halves", 100), ("pairs", 64), ("halves", 32)])
@pytest.mark.parametrize("queries", [True, False], ids=["queries", "keys_only"])
def test_rotating_append_is_the_calls_it_stands_for(bits8, layout, rot, queries):
    import torch
    from paper_2603_14371_amd import binding as B
    rng = np.random.default_rng(rot)
    turn = Turn(rot, layout, amplitude=0.75)
    s = torch.cuda.current_stream().cuda_stream
    lens = [1, 50, 3, 16, 1]
    n = sum(lens)
    wide = _bits(rng, n, 10, 256)
    x = _up(wide)
    pos = torch.tensor(rng.integers(0, 4000, n).astype(np.int32), device="cuda")
    stored = []
    for fused in (False, True):
        pool, keep = _pool(bits8)
        sids = [B.oxy_stream_create(pool, -1, ACTION if m == 50 else DECODE) for m in lens]
        first = B.oxy_batch_build(pool, [(sids[0], 5), (sids[3], 21)], B.BATCH_APPEND_ONLY, s)
        B.oxy_stream_append(pool, first, 1, x.data_ptr(), x.data_ptr(), s)
        B.oxy_batch_destroy(first)
        batch = B.oxy_batch_build(pool, list(zip(sids, lens)), 0, s)
        q = torch.full((n, 8, 256), 77, dtype=torch.int16, device="cuda")
        if fused:
            B.oxy_rotary_append(pool, batch, 1, turn.cfg, pos.data_ptr(), x.data_ptr() if queries else 0, 5120,
                                q.data_ptr() if queries else 0, x[:, 8].data_ptr(), 5120, x[:, 9].data_ptr(), 5120, s)
        else:
            k, v = torch.zeros((n, 256), dtype=torch.int16, device="cuda"), x[:, 9].contiguous()
            if queries:
                B.oxy_rotary(turn.cfg, pos.data_ptr(), x.data_ptr(), 5120, q.data_ptr(), 4096, n, 8, s)
            B.oxy_rotary(turn.cfg, pos.data_ptr(), x[:, 8].data_ptr(), 5120, k.data_ptr(), 512, n, 1, s)
            B.oxy_stream_append(pool, batch, 1, k.data_ptr(), v.data_ptr(), s)
        torch.cuda.synchronize()
        stored.append((_down(q), keep[0].cpu().numpy()))
        B.oxy_batch_destroy(batch)
        B.oxy_pool_destroy(pool)
    assert np.array_equal(stored[0][0], stored[1][0])
    assert np.array_equal(stored[0][1], stored[1][1])
    if queries:
        turn.check(wide[:, :8], pos.cpu().numpy(), stored[1][0])
    assert np.array_equal(_down(x), wide)


def test_rotating_append_refuses():
    import torch
    from paper_2603_14371_amd import binding as B
    turn = Turn(256, "halves")
    pool, keep = _pool(True)
    other, keep2 = _pool(True)
    s = torch.cuda.current_stream().cuda_stream
    sid = B.oxy_stream_create(pool, -1, DECODE)
    batch = B.oxy_batch_build(pool, [(sid, 4)], 0, s)
    buf = torch.zeros(4 * 5120, dtype=torch.uint8, device="cuda")
    p = buf.data_ptr()
    pos = torch.zeros(4, dtype=torch.int32, device="cuda")
    good = dict(pool=pool, batch=batch, layer=0, rotary=turn.cfg, pos=pos.data_ptr(), q=p, qs=5120, qo=p, k=p, ks=5120, v=p,
                vs=5120)
    d = turn.dev.data_ptr()
    for bad in (dict(pool=other), dict(layer=2), dict(layer=-1), dict(rotary=B.make_rotary(0, 256)),
                dict(rotary=B.make_rotary(d, 255)), dict(rotary=B.make_rotary(d, 258)), dict(rotary=B.make_rotary(d, 0)),
                dict(rotary=B.make_rotary(d, 256, 2)), dict(pos=0), dict(qo=0), dict(k=0), dict(v=0), dict(q=p + 2),
                dict(k=p + 8), dict(v=p + 4), dict(qo=p + 8), dict(qs=4088), dict(qs=4080), dict(ks=504), dict(ks=496),
                dict(vs=16), dict(qo=p)):
        a = dict(good, **bad)
        with pytest.raises(B.OxyError) as e:
            B.oxy_rotary_append(a["pool"], a["batch"], a["layer"], a["rotary"], a["pos"], a["q"], a["qs"], a["qo"], a["k"],
                                a["ks"], a["v"], a["vs"], s)
        assert e.value.code == B.ERR_INVALID_ARG
    B.oxy_batch_destroy(batch)
    for x in (pool, other):
        B.oxy_pool_destroy(x)


@pytest.mark.parametrize("bits8", [True, False], ids=["kv8", "bf16"])
def test_a_decode_loop_with_drafts(bits8):
    """The operators together, as a serving loop uses them: an observation's keys are turned and stored; every step turns
    and stores the new tokens of a chunk and of requests with one to five drafts, attends, and the drafts that were
    not taken are rewound.  Everything against the oracle, which turns, stores and attends in 64 bits."""
    import torch
    from paper_2603_14371_amd import binding as B
    rng = np.random.default_rng(31)
    turn = Turn(128, "halves", kind=B.ROTARY_BANDS, factor=4.0, low=1.0, high=4.0, original_len=256)
    s = torch.cuda.current_stream().cuda_stream
    P, chunk = 205, 20
    pool, keep = _pool(bits8, n_layers=1, blocks=128)
    model = {}

    def bf16(x):         # 64-bit numbers to the nearest bf16, as bits
        u = np.asarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
        return ((u + 0x7fff + ((u >> 16) & 1)) >> 16).astype(np.uint16)

    def held(bits):
        return kv8.bf16_bits(kv8.cached_values(bits)) if bits8 else bits

    wide = _bits(rng, P, 10, 256)
    x, pos = _up(wide), np.arange(P)
    k = _rotate(turn, x[:, 8:], pos, P, 1, 5120)
    turn.check(wide[:, 8:9], pos, _down(k))
    pid = B.oxy_prefix_create(pool)
    v = x[:, 9].contiguous()
    B.oxy_prefix_append(pool, pid, 0, k.data_ptr(), v.data_ptr(), P, 0, s)
    prefix = held(_down(k)[:, 0]), held(wide[:, 9])
    act = B.oxy_stream_create(pool, pid, ACTION)
    decs = [B.oxy_stream_create(pool, pid, DECODE) for _ in range(3)]
    model = {d: (np.zeros((0, 256), np.uint16),) * 2 for d in decs}
    from oracle.attention import attend_item
    for step in range(8):
        items = [(act, chunk)] + [(d, 1 + (step * (i + 1)) % 5) for i, d in enumerate(decs)]
        n = sum(m for _, m in items)
        wide = _bits(rng, n, 10, 256)
        x = _up(wide)
        pos = np.concatenate([P + np.arange(chunk)] + [P + len(model[d][0]) + np.arange(m) for d, m in items[1:]])
        dpos = torch.tensor(pos.astype(np.int32), device="cuda")
        batch = B.oxy_batch_build(pool, items, 0, s)
        q = torch.zeros((n, 8, 256), dtype=torch.int16, device="cuda")
        o, lse = torch.zeros_like(q), torch.zeros((n, 8), device="cuda")
        B.oxy_rotary_append(pool, batch, 0, turn.cfg, dpos.data_ptr(), x.data_ptr(), 5120, q.data_ptr(),
                            x[:, 8].data_ptr(), 5120, x[:, 9].data_ptr(), 5120, s)
        B.oxy_mixed_attention(pool, batch, 0, q.data_ptr(), o.data_ptr(), lse.data_ptr(), 0.0625, s)
        slots = B.oxy_batch_slots(batch)
        kb, vb = (torch.zeros((n, 256), dtype=torch.int16, device="cuda") for _ in range(2))
        B.oxy_gather_kv(pool, 0, slots, kb.data_ptr(), vb.data_ptr(), s)
        q, kb, vb = _down(q), _down(kb), _down(vb)
        B.oxy_batch_destroy(batch)
        turn.check(wide[:, :8], pos, q)
        assert np.array_equal(vb, held(wide[:, 9]))
        # the kernel rounds keys that it turned in 32 bits: those within that of a border may fall either way
        exact = rotary.turned(widen_bf16(wide[:, 8:9]), pos, turn.freqs, "halves", turn.amplitude)[:, 0]
        want = held(bf16(exact))
        assert np.mean(kb != want) < 1e-3
        assert np.all(np.abs(widen_bf16(kb) - widen_bf16(want)) <= (2.0 ** -3 if bits8 else 2.0 ** -7) * np.abs(exact) + 2.0 ** -18)
        t = 0
        for sid, m in items:
            old = (np.zeros((0, 256), np.uint16),) * 2 if sid == act else model[sid]
            own = np.concatenate([old[0], kb[t:t + m]]), np.concatenate([old[1], vb[t:t + m]])
            ref, ref_lse = attend_item(0 if sid == act else 1, q[t:t + m], prefix[0], prefix[1], own[0], own[1], 0.0625)
            assert_o_close(_down(o)[t:t + m], ref, "step %d" % step)
            assert_lse_close(lse.cpu().numpy()[t:t + m], ref_lse, "step %d" % step)
            if sid != act:
                keep_n = len(old[0]) + max(1, m - step % 3)       # the drafts that are taken
                B.oxy_stream_rewind(pool, sid, keep_n)
                model[sid] = own[0][:keep_n], own[1][:keep_n]
            t += m
    B.oxy_pool_destroy(pool)
