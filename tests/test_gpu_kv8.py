"""A pool in 8 bits on the GPU: rows held as the oracle says, bit for bit, however they came in; attention
over them against the float64 oracle on the held values (same rounding chain behind the values as a
bf16 pool: probabilities as hi + lo bf16, split results in 16 bits, so the same tolerances); the
invariants of the method, bit for bit."""
import numpy as np
import pytest

from oracle import kv8
from oracle.attention import widen_bf16
from oracle.replay import OracleWorld
from paper_2603_14371_amd import synth
from paper_2603_14371_amd.synth import ACTION, DECODE, _TraceBuilder, _workload
from parity_util import assert_lse_close, assert_o_close, assert_pool_contents_equal

pytestmark = pytest.mark.gpu


def run_both8(w, compare=True, oracle_steps=None, layers=None, source=None, **kw):
    """One trace through a pool in 8 bits and through the oracle on what such a pool holds."""
    from paper_2603_14371_amd.harness import GpuWorld
    src = source or synth.DataSource(w["seed"], w["sigma"])
    order = None if w["free_order"] is None else list(w["free_order"])
    ow = OracleWorld(w["num_blocks"], w["n_layers"], kv8.cached_source(src), w["scale"], free_order=order,
                     layers=layers)
    gw = GpuWorld(w, src, layers=layers, kv8=True, **kw)
    for i, op in enumerate(w["trace"]):
        g = gw.apply(op)
        skip = oracle_steps is not None and op["op"] == "step" and i not in oracle_steps
        o = ow.apply(dict(op, attend=False) if skip else op)
        if "slots" in o:
            assert g["slots"] == o["slots"], i
        if compare and op["op"] == "step":
            for layer, ref in o["O"].items():
                assert_o_close(g["O"][layer], ref, "op %d layer %d" % (i, layer))
                if layer in g["LSE"]:
                    assert_lse_close(g["LSE"][layer], o["LSE"][layer], "op %d layer %d" % (i, layer))
    return gw, ow


def _same_rows(got, want):
    """Bit patterns, any NaN for any NaN."""
    nan = (want & 0x7fff) > 0x7f80
    assert np.array_equal((got & 0x7fff) > 0x7f80, nan)
    assert np.array_equal(got[~nan], want[~nan])


class Cache:
    """A pool in 8 bits, driven by hand."""

    def __init__(self, n_layers=2, blocks=40, fill=0xFF, order=None):
        import torch
        from paper_2603_14371_amd import binding as B
        self.torch, self.B = torch, B
        cfg = B.make_config(n_layers, blocks, free_order=order, flags=B.POOL_KV_FP8, max_q_tokens=1024)
        self.kv = torch.full((B.oxy_kv_bytes(cfg),), fill, dtype=torch.uint8, device="cuda")
        self.ws = torch.empty(B.oxy_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        cfg.kv_base, cfg.kv_bytes = self.kv.data_ptr(), self.kv.numel()
        cfg.workspace, cfg.workspace_bytes = self.ws.data_ptr(), self.ws.numel()
        self.pool = B.oxy_pool_create(cfg)
        self.n_layers, self.blocks = n_layers, blocks
        self.stream = torch.cuda.current_stream().cuda_stream

    def up(self, bits):
        return self.torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda()

    def back(self, t):
        self.torch.cuda.synchronize()
        return t.view(self.torch.int16).cpu().numpy().view(np.uint16)

    def gather(self, layer, slots):
        k = self.torch.zeros((len(slots), 256), dtype=self.torch.bfloat16, device="cuda")
        v = self.torch.zeros_like(k)
        self.B.oxy_gather_kv(self.pool, layer, slots, k.data_ptr(), v.data_ptr(), self.stream)
        return self.back(k), self.back(v)

    def prefix_slots(self, pid):
        n = self.B.oxy_prefix_info(self.pool, pid)[0]
        blocks = self.B.oxy_prefix_blocks(self.pool, pid)
        return [blocks[t // 16] * 16 + t % 16 for t in range(n)]

    def close(self):
        self.torch.cuda.synchronize()
        self.B.oxy_pool_destroy(self.pool)


def _rows(kind, n, seed):
    """bf16 bit patterns [n, 256]."""
    rng = np.random.default_rng(seed)
    f32 = lambda x: (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16)  # noqa: E731
    if kind == "normal":
        return f32(rng.standard_normal((n, 256)) * 2.0 ** rng.integers(-4, 5, (n, 1)))
    if kind == "any":                # every finite bit pattern is as likely
        return rng.choice(np.r_[0:0x7f80, 0x8000:0xff80].astype(np.uint16), (n, 256))
    if kind == "subnormal":          # rows below 448 * 2^-126, and rows of bf16 subnormals
        x = rng.integers(0, 0x0a00, (n, 256)).astype(np.uint16) | (rng.integers(0, 2, (n, 256)) << 15).astype(np.uint16)
        x[::2] &= 0x807f
        return x
    if kind == "borders":            # largest elements around 448 * 2^e, ties of e4m3, zeros
        x = f32(rng.integers(-256, 257, (n, 256)) / 16.0)
        x[:, 0] = f32(np.array([27.875, 28.0, 28.125, 31.875, 32.0, 14.0, 14.0625, 0.0])[rng.integers(0, 8, n)])
        x[::5] = 0
        x[1::5] |= 0x8000
        return x
    x = f32(rng.standard_normal((n, 256)))
    for i, bits in enumerate((0x7f80, 0xff80, 0x7fc0, 0xffc1, 0x7f81)):
        x[i::7, 10 * i + 3] = bits
    x[n // 2] = 0x7f80               # a row with nothing finite
    return x


@pytest.mark.parametrize("kind", ["normal", "any", "subnormal", "borders", "nonfinite"])
@pytest.mark.parametrize("n", [1, 15, 16, 17, 203])
def test_prefix_rows_come_back_as_the_oracle_says(kind, n):
    c = Cache(order=np.random.default_rng(n).permutation(40).tolist())
    k, v = _rows(kind, 2 * n, n).reshape(2, n, 256), _rows(kind, 2 * n, n + 1).reshape(2, n, 256)
    dk, dv = c.up(k), c.up(v)
    pid = c.B.oxy_prefix_create(c.pool)
    c.B.oxy_prefix_append_layers(c.pool, pid, 0, 2, dk.data_ptr(), dv.data_ptr(), n * 512, n, 0, c.stream)
    for layer in range(2):
        gk, gv = c.gather(layer, c.prefix_slots(pid))
        _same_rows(gk, kv8.bf16_bits(kv8.cached_values(k[layer])))
        _same_rows(gv, kv8.bf16_bits(kv8.cached_values(v[layer])))
    c.close()


@pytest.mark.parametrize("kind", ["normal", "any", "borders", "nonfinite"])
def test_rows_depend_on_nothing_but_themselves(kind):
    """The same tokens in one call, in ragged pieces, layer by layer, or token by token as a stream: the same
    bytes in the pool, over whatever was there before, and nothing else is touched."""
    n = 75
    k, v = _rows(kind, n, 3), _rows(kind, n, 4)
    want = None
    for way in ("whole", "pieces", "stream", "tokens"):
        for fill in (0xFF, 0x00):
            c = Cache(n_layers=2, blocks=8, fill=fill)
            dk, dv = c.up(k), c.up(v)
            if way in ("whole", "pieces"):
                cuts = [0, n] if way == "whole" else [0, 5, 16, 17, 30, 64, 74, 75]
                pid = c.B.oxy_prefix_create(c.pool)
                for a, b in zip(cuts, cuts[1:]):
                    c.B.oxy_prefix_append(c.pool, pid, 1, dk[a:].data_ptr(), dv[a:].data_ptr(), b - a, a, c.stream)
            else:
                sid = c.B.oxy_stream_create(c.pool, -1, DECODE)
                step = n if way == "stream" else 1
                for a in range(0, n, step):
                    b = c.B.oxy_batch_build(c.pool, [(sid, step)], c.B.BATCH_APPEND_ONLY, c.stream)
                    c.B.oxy_stream_append(c.pool, b, 1, dk[a:].data_ptr(), dv[a:].data_ptr(), c.stream)
                    c.B.oxy_batch_destroy(b)
            gk, gv = c.gather(1, list(range(n)))          # blocks are handed out in order
            _same_rows(gk, kv8.bf16_bits(kv8.cached_values(k)))
            _same_rows(gv, kv8.bf16_bits(kv8.cached_values(v)))
            raw = c.kv.cpu().numpy().reshape(2, -1)
            assert np.all(raw[0] == fill)                 # the other layer
            codes, exps = raw[1][:8 * 8192].reshape(8, 8192), raw[1][8 * 8192:8 * 8224].reshape(8, 32)
            assert np.all(codes[5:] == fill) and np.all(exps[5:] == fill)
            # the page of the last tokens: 11 of its 16 rows are written
            touched = codes[4] != fill
            assert np.count_nonzero(touched) <= 2 * 11 * 256 and np.count_nonzero(exps[4] != fill) <= 2 * 11
            if want is None:
                want = codes[:4].copy(), exps[:4].copy()
            assert np.array_equal(codes[:4], want[0]) and np.array_equal(exps[:4], want[1]), way
            c.close()


def test_appending_beside_rows_leaves_them_as_they_were():
    c = Cache(n_layers=1, blocks=4, fill=0xFF)
    k, v = _rows("normal", 64, 1), _rows("normal", 64, 2)
    dk, dv = c.up(k), c.up(v)
    pid = c.B.oxy_prefix_create(c.pool)
    c.B.oxy_prefix_append(c.pool, pid, 0, dk.data_ptr(), dv.data_ptr(), 64, 0, c.stream)
    k2, v2 = _rows("any", 64, 5), _rows("any", 64, 6)
    d2, e2 = c.up(k2), c.up(v2)
    for a, n in ((3, 1), (20, 6), (37, 20)):
        c.B.oxy_prefix_append(c.pool, pid, 0, d2[a:].data_ptr(), e2[a:].data_ptr(), n, a, c.stream)
        k[a:a + n], v[a:a + n] = k2[a:a + n], v2[a:a + n]
        gk, gv = c.gather(0, list(range(64)))
        _same_rows(gk, kv8.bf16_bits(kv8.cached_values(k)))
        _same_rows(gv, kv8.bf16_bits(kv8.cached_values(v)))
    c.close()


@pytest.mark.parametrize("bits8", [True, False], ids=["kv8", "bf16"])
def test_read_back_of_several_layers_is_that_of_each(bits8):
    import torch
    from paper_2603_14371_amd import binding as B
    from paper_2603_14371_amd.harness import GpuWorld
    b = _TraceBuilder()
    pid = b.prefix(700)
    d = b.stream(pid, DECODE)
    b.step([(d, 37)], attend=False)
    w = _workload("read_back", 61, 4, 64, b.trace)
    gw = GpuWorld(w, synth.DataSource(61), kv8=bits8)
    gw.run(w["trace"])
    rng = np.random.default_rng(0)
    live = gw.prefix_slots(pid) + gw.stream_slots(d)
    for slots in (live, live[::-1], list(rng.permutation(live)), [live[5]] * 3, live * 7, [live[-1]]):
        n, stride = len(slots), len(slots) * 512 + 256
        k = torch.zeros(4 * stride, dtype=torch.uint8, device="cuda")
        v = torch.zeros_like(k)
        B.oxy_gather_kv_layers(gw.pool, 1, 4, slots, k.data_ptr(), v.data_ptr(), stride, gw._stream())
        torch.cuda.synchronize()
        for layer in range(1, 4):
            gk, gv = gw.gather(layer, slots)
            at = (layer - 1) * stride
            for got, want in ((k, gk), (v, gv)):
                rows = got[at:at + n * 512].cpu().numpy().view(np.uint16).reshape(n, 256)
                assert np.array_equal(rows, want)
                assert not got[at + n * 512:at + stride].any()
    for bad in (dict(layer_begin=2, layer_end=2), dict(layer_begin=-1, layer_end=2), dict(layer_end=5),
                dict(stride=100), dict(stride=len(live) * 512 + 8), dict(slots=[64 * 16]), dict(slots=[-1])):
        a = dict(dict(layer_begin=0, layer_end=4, slots=live, stride=len(live) * 512), **bad)
        with pytest.raises(B.OxyError):
            B.oxy_gather_kv_layers(gw.pool, a["layer_begin"], a["layer_end"], a["slots"], k.data_ptr(), v.data_ptr(),
                                   a["stride"], gw._stream())
    gw.close()


def test_tiny_config():
    gw, ow = run_both8(synth.tiny())
    assert assert_pool_contents_equal(gw, ow) == 64 + 10 + 5
    gw.close()


@pytest.mark.parametrize("kw", [
    dict(prefix_len=70), dict(prefix_len=0), dict(prefix_len=1, chunk=1, prior=0), dict(prefix_len=33, chunk=1, prior=0),
    dict(prefix_len=64, chunk=50, prior=40), dict(prefix_len=832, chunk=50, prior=300, n_layers=3),
    dict(sigma=1.0 / 16.0), dict(prefix_len=70, chunk=13, prior=21),
], ids=str)
@pytest.mark.parametrize("split", [0, 32, 64])
def test_tiny_variants_in_a_pool_full_of_nan(kw, split):
    gw, ow = run_both8(synth.tiny(**kw), poison=True, split_tokens=split)
    assert_pool_contents_equal(gw, ow)
    gw.close()


def test_several_new_tokens_are_causal():
    b = _TraceBuilder()
    pid = b.prefix(40)
    d0, d1 = b.stream(pid, DECODE), b.stream(-1, DECODE)
    b.step([(d0, 7), (d1, 37)])
    b.step([(d1, 3), (d0, 5)])
    b.step([(d0, 70)])
    b.step([(d0, 1), (d1, 2)])
    gw, ow = run_both8(_workload("multi_token", 99, 2, 64, b.trace), split_tokens=32, poison=True)
    assert_pool_contents_equal(gw, ow)
    gw.close()


@pytest.mark.parametrize("tile,stream", [(512, 512), (1024, 1024), (32, 32), (96, 160), (0, 0)])
def test_split_sizes(tile, stream):
    """Also splits longer than the 16 pages that a work record lists."""
    gw, ow = run_both8(synth.tiny(prefix_len=1100, chunk=37, prior=1700, n_layers=2), split_tokens=tile,
                       stream_split_tokens=stream, max_partials=8192, poison=True)
    assert_pool_contents_equal(gw, ow)
    gw.close()


@pytest.mark.parametrize("n_new", [1, 2, 5])
def test_histories_around_page_step_round_and_split_boundaries(n_new):
    b = _TraceBuilder()
    pid = b.prefix(70)
    lens = [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 255, 256, 257, 384, 511, 512, 513, 640]
    sids = [b.stream(pid if i % 3 else -1, DECODE) for i in range(len(lens))]
    b.step(list(zip(sids, lens)), attend=False)
    b.step([(s, n_new) for s in sids])
    gw, ow = run_both8(_workload("boundaries", 77, 1, 600, b.trace), poison=True)
    assert_pool_contents_equal(gw, ow)
    gw.close()


@pytest.mark.parametrize("chunk", [1, 2, 3, 16, 31, 32, 33, 50, 63, 64, 65, 100, 130])
def test_chunks_of_every_width(chunk):
    b = _TraceBuilder()
    pids = [b.prefix(n, b.recipe(n, tag=50 + n)) for n in (300, 832)]
    acts = [b.stream(p, ACTION) for p in pids + [-1]]
    for _ in range(2):                       # a chunk is rewound and written anew
        b.step([(a, chunk) for a in acts])
    gw, ow = run_both8(_workload("chunks", 12, 1, 200, b.trace), poison=True)
    assert_pool_contents_equal(gw, ow)
    gw.close()


def test_frame_of_the_pi05_shape():
    w = synth.pi05_frame(n_layers=2, denoise_steps=3, decode_tokens=20)
    steps = [i for i, op in enumerate(w["trace"]) if op["op"] == "step"]
    gw, ow = run_both8(w, oracle_steps=set(steps[::5]))
    assert_pool_contents_equal(gw, ow)
    gw.close()


def test_frames_with_requests_carried_over():
    w = synth.cross_frame(n_frames=7, n_layers=1)
    steps = [i for i, op in enumerate(w["trace"]) if op["op"] == "step"]
    gw, ow = run_both8(w, oracle_steps=set(steps[::9]))
    assert_pool_contents_equal(gw, ow)
    gw.close()


def test_many_requests_on_shared_prefixes():
    """The stress geometry: items of eight tokens, own pages past the caches, results written through."""
    w = synth.stress(n_layers=1)
    steps = [i for i, op in enumerate(w["trace"]) if op["op"] == "step"]
    gw, ow = run_both8(w, oracle_steps=set(steps[-1:]))
    gw.close()


def test_own_pages_past_the_caches():
    """Requests whose pages in all layers are more than what non-temporal loads begin at; one layer is run."""
    b = _TraceBuilder()
    sids = [b.stream(-1, DECODE) for _ in range(24)]
    b.step([(s, 530 + 17 * i) for i, s in enumerate(sids)], attend=False)
    b.step([(s, 1 + i % 2) for i, s in enumerate(sids)])
    w = _workload("once", 21, 24, 1400, b.trace)
    assert sum(530 + 17 * i for i in range(24)) * 24 * 514 > 128 << 20
    gw, ow = run_both8(w, layers=[23], poison=True)
    gw.close()


def _only(prefixes, chunks, requests, take):
    """One step; the outputs of item `take` in it, by the bits of its rows."""
    from paper_2603_14371_amd.harness import GpuWorld
    b = _TraceBuilder()
    pids = [b.prefix(n, b.recipe(n, tag=30 + i)) for i, n in enumerate(prefixes)]
    items = [(b.stream(pids[p], ACTION), n, tag) for p, n, tag in chunks]
    reqs = [(b.stream(pids[p], DECODE), h, n, tag) for p, h, n, tag in requests]
    for sid, h, n, tag in reqs:
        if h:
            b.step([(sid, h)], attend=False, recipe={"tag": 500 + tag, "tok0": 0, "n_total": h})
    items += [(sid, n, tag) for sid, h, n, tag in reqs]
    w = _workload("only", 4, 1, 4000, b.trace)
    data = synth.DataSource(4)
    gw = GpuWorld(w, data, kv8=True, max_q_tokens=2048, max_append_tokens=32768, max_partials=40000)
    gw.run(w["trace"])

    def stitched(recipe, layer, what, n):
        return np.concatenate([data({"tag": 900 + tag, "tok0": 0, "n_total": m}, layer, what, m) for _, m, tag in items])
    gw.data_fn = stitched
    r = gw.step({"op": "step", "items": [(s, n) for s, n, _ in items], "attend": True, "data": None})
    gw.close()
    t = 0
    for _, n, tag in items:
        if tag == take:
            return r["O"][0][t:t + n], r["LSE"][0][t:t + n]
        t += n


@pytest.mark.parametrize("n_new,hist", [(1, 0), (1, 40), (1, 700), (2, 300), (6, 100)])
def test_a_request_gives_the_same_bits_alone_and_among_others(n_new, hist):
    me = (0, hist, n_new, 7)
    alone = _only([900], [], [me], 7)
    few = _only([900], [(0, 50, 1)], [(0, 33, 1, 2), me], 7)
    many = _only([900, 300], [(0, 50, 1), (1, 50, 3)], [(i % 2, 20 * i, 1, 20 + i) for i in range(60)] + [me], 7)
    for other in (few, many):
        assert np.array_equal(alone[0], other[0]) and np.array_equal(alone[1], other[1])


@pytest.mark.parametrize("chunk,prefix", [(50, 832), (13, 2048), (70, 200)])
def test_a_chunk_gives_the_same_bits_alone_and_among_others(chunk, prefix):
    me = (0, chunk, 7)
    alone = _only([prefix], [me], [], 7)
    few = _only([prefix, 64], [(1, 3, 1), me], [(0, 33, 1, 2)], 7)
    many = _only([prefix, 300], [(1, 50, 1), me] + [(1, 50, 60 + i) for i in range(5)],
                 [(i % 2, 20 * i, 1, 20 + i) for i in range(60)], 7)
    for other in (few, many):
        assert np.array_equal(alone[0], other[0]) and np.array_equal(alone[1], other[1])


def test_every_form_of_a_step_gives_the_same_bits():
    """Per-layer calls, append + attention of a layer, all layers in a call, recorded; the forms that fold or fuse the
    append are not covered and give the plain one.  Recordings are replayed with eager work between them."""
    import torch
    from paper_2603_14371_amd import binding as B
    from paper_2603_14371_amd.harness import GpuWorld, bits_of, to_device_bf16
    w = synth.tiny(prefix_len=200, chunk=50, prior=77, n_layers=3)
    data = synth.DataSource(17)
    results = {}
    modes = {"calls": None, "append_attention": None, "static": None, "plain": 0, "fuse": B.STEP_FUSE_ACROSS_LAYERS,
             "fold": B.STEP_FOLD_APPEND, "graph": B.STEP_GRAPH, "fold_graph": B.STEP_FOLD_APPEND | B.STEP_GRAPH}
    for mode, flags in modes.items():
        gw = GpuWorld(w, data, kv8=True, poison=True)
        gw.run(w["trace"][:-1])
        op = w["trace"][-1]
        n, L, s = sum(m for _, m in op["items"]), 3, gw._stream()
        k, v, q = (torch.stack([to_device_bf16(data(op["data"], l, x, n), gw.device) for l in range(L)]) for x in "kvq")
        o, lse = torch.zeros_like(q), torch.zeros((L, n, 8), device=gw.device)
        batch = B.oxy_batch_build(gw.pool, op["items"], 0, s)
        for again in range(3):
            o.zero_()
            if flags is None:
                for l in range(L):
                    args = (k[l].data_ptr(), v[l].data_ptr())
                    tail = (q[l].data_ptr(), o[l].data_ptr(), lse[l].data_ptr(), gw.scale, s)
                    if mode == "append_attention":
                        B.oxy_append_attention(gw.pool, batch, l, *args, *tail)
                    else:
                        B.oxy_stream_append(gw.pool, batch, l, *args, s)
                        (B.oxy_mixed_attention if mode == "calls" else B.oxy_mixed_attention_static)(
                            gw.pool, batch, l, *tail)
            else:
                B.oxy_step_layers(gw.pool, batch, 0, L, k.data_ptr(), v.data_ptr(), k.stride(0) * 2, q.data_ptr(),
                                  o.data_ptr(), q.stride(0) * 2, lse.data_ptr(), lse.stride(0) * 4, gw.scale, flags, None, s)
            torch.cuda.synchronize()
            got = (bits_of(o), lse.cpu().numpy())
            if again:
                assert np.array_equal(got[0], results[mode][0]) and np.array_equal(got[1], results[mode][1])
            results[mode] = got
        if flags is not None and flags & B.STEP_GRAPH:
            assert B.oxy_step_graph_stats(gw.pool) == (1, 0, 3)
        B.oxy_batch_destroy(batch)
        gw.close()
    for mode in modes:
        assert np.array_equal(results[mode][0], results["calls"][0]), mode
        assert np.array_equal(results[mode][1], results["calls"][1]), mode
    assert np.isfinite(results["calls"][1]).all() and results["calls"][0].any()


@pytest.mark.parametrize("scale", [1.0 / 16, -0.11, 0.0, 3.0])
def test_softmax_scales(scale):
    w = dict(synth.tiny(prefix_len=150, chunk=20, prior=90), scale=scale)
    src = synth.DataSource(w["seed"], 0.5)
    gw, ow = run_both8(w, source=src)
    gw.close()


@pytest.mark.parametrize("where", ["prefix", "chunk", "history"])
@pytest.mark.parametrize("bits", [0x7f80, 0xff80, 0x7fc0], ids=["inf", "-inf", "nan"])
def test_a_value_that_is_not_finite_gives_no_wrong_finite_output(where, bits):
    """Held as NaN: lost are the dim, or its 64 (the sums that share an exponent), of the queries that see it."""
    from paper_2603_14371_amd.harness import GpuWorld
    b = _TraceBuilder()
    pid = b.prefix(300, b.recipe(300, tag=100))
    act, dec = b.stream(pid, ACTION), b.stream(pid, DECODE)
    b.tag = 10
    b.step([(dec, 150)], attend=False)                 # tag 10
    b.step([(act, 50), (dec, 1)])                      # tag 11
    w = _workload("nonfinite", 5180, 1, 512, b.trace)
    src = synth.DataSource(w["seed"])
    tag, row = {"prefix": (100, 17), "chunk": (11, 9), "history": (10, 70)}[where]

    def planted(recipe, layer, what, n):
        x = src(recipe, layer, what, n).copy()
        if what == "v" and recipe["tag"] == tag:
            x[row - recipe["tok0"], 133] = bits
        return x

    def without(recipe, layer, what, n):      # the row's other elements as the cache holds them beside the planted one
        x = planted(recipe, layer, what, n)
        x = x if what == "q" else kv8.bf16_bits(kv8.cached_values(x))
        return np.where((x & 0x7fff) > 0x7f80, np.uint16(0), x)

    gw = GpuWorld(w, planted, poison=True, kv8=True)
    ow = OracleWorld(w["num_blocks"], 1, without, w["scale"])
    for op in w["trace"]:
        g, o = gw.apply(op), ow.apply(op)
    gw.close()
    got, ref = g["O"][0], o["O"][0]
    sees = {"prefix": list(range(51)), "chunk": list(range(50)), "history": [50]}[where]
    assert not np.isfinite(widen_bf16(got[sees][:, :, 133])).any()
    part = np.arange(256) // 64 == 133 // 64
    assert_o_close(got[:, :, ~part], ref[:, :, ~part], where)
    lost = ~np.isfinite(widen_bf16(got[:, :, part]))
    assert np.all(lost.all(axis=2) | (lost.sum(axis=2) <= 1))
    assert_o_close(got[:, :, part][~lost], ref[:, :, part][~lost], where)
    rest = np.setdiff1d(np.arange(len(ref)), sees)
    if len(rest):
        assert_o_close(got[rest], ref[rest], where)
    assert_lse_close(g["LSE"][0], o["LSE"][0], where)


def test_values_of_very_different_size():
    """Exponents of one round's values 2^60 apart: a row's output is that of its largest values."""
    b = _TraceBuilder()
    d = b.stream(-1, DECODE)
    b.step([(d, 200)], attend=False)
    b.step([(d, 1)])
    w = _workload("sizes", 9, 1, 40, b.trace)
    src = synth.DataSource(9)

    def sized(recipe, layer, what, n):
        x = src(recipe, layer, what, n).copy()
        if what == "v":                       # rows times 2^-30, 1 and 2^30 in turn: exponent bits shifted
            x = (x.astype(np.int32) + (((np.arange(n) + recipe["tok0"]) % 3 - 1) * 30 * 128)[:, None]).astype(np.uint16)
        return x

    from paper_2603_14371_amd.harness import GpuWorld
    gw = GpuWorld(w, sized, kv8=True)
    ow = OracleWorld(w["num_blocks"], 1, kv8.cached_source(sized), w["scale"])
    for op in w["trace"]:
        g, o = gw.apply(op), ow.apply(op)
    gw.close()
    # the tolerance of outputs of the order of one, in units of 2^30
    assert_o_close_scaled(g["O"][0], o["O"][0], 2.0 ** 30)


def assert_o_close_scaled(bits, ref, unit):
    got = widen_bf16(bits) / unit
    assert np.all(np.abs(got - ref / unit) <= 2e-3 + 1e-2 * np.abs(ref / unit))


def test_another_stream():
    """All work goes to the stream that is handed in."""
    import torch
    from paper_2603_14371_amd.harness import GpuWorld
    w = synth.tiny(prefix_len=300, chunk=20, prior=60, n_layers=2)
    src = synth.DataSource(w["seed"])
    outs = []
    for own_stream in (False, True):
        s = torch.cuda.Stream() if own_stream else torch.cuda.current_stream()
        with torch.cuda.stream(s):
            gw = GpuWorld(w, src, kv8=True)
            outs.append([r.get("O") for r in gw.run(w["trace"])][-1])
            gw.close()
    for layer in outs[0]:
        assert np.array_equal(outs[0][layer], outs[1][layer])


@pytest.mark.parametrize("hist", [4200, 9001])
def test_long_histories_are_merged_by_many(hist):
    """Tokens of more than 32 split results take another merge; beside them, tokens of fewer give the bits that they
    give in any other launch."""
    b = _TraceBuilder()
    pid = b.prefix(300)
    d, e, a = b.stream(pid, DECODE), b.stream(-1, DECODE), b.stream(pid, ACTION)
    b.step([(d, hist), (e, 700)], attend=False)
    b.step([(a, 5), (d, 1), (e, 2)])
    b.step([(d, 2)])
    w = _workload("long", 11, 1, 800, b.trace)
    gw, ow = run_both8(w, poison=True, max_partials=4096, stream_split_tokens=32)
    gw.close()
    gw, ow = run_both8(w, poison=True)
    gw.close()


def test_short_tokens_beside_a_long_one_give_the_same_bits():
    me = (0, 700, 1, 7)
    alone = _only([900], [], [me], 7)
    beside = _only([900], [(0, 13, 1)], [(0, 20000, 1, 2), me], 7)
    assert np.array_equal(alone[0], beside[0]) and np.array_equal(alone[1], beside[1])


@pytest.mark.parametrize("n,blocks,first", [(16 * 1920 + 40, 2000, 0), (16 * 1920 + 40, 2000, 7), (16 * 960 + 21, 65600, 0)])
def test_more_tokens_than_a_launch_takes(n, blocks, first):
    """Ids of 1920 blocks travel with a launch, or of 960 where one of the pool's needs more than 16 bits."""
    order = np.random.default_rng(blocks).permutation(blocks)
    order = np.roll(order, -int(np.argmax(order == blocks - 1)) + 3).tolist()      # the largest id is among them
    c = Cache(n_layers=1, blocks=blocks, order=order)
    k, v = _rows("normal", n, 1), _rows("normal", n, 2)
    dk, dv = c.up(k), c.up(v)
    pid = c.B.oxy_prefix_create(c.pool)
    if first:
        c.B.oxy_prefix_append(c.pool, pid, 0, dk.data_ptr(), dv.data_ptr(), first, 0, c.stream)
    c.B.oxy_prefix_append(c.pool, pid, 0, dk[first:].data_ptr(), dv[first:].data_ptr(), n - first, first, c.stream)
    slots = c.prefix_slots(pid)
    assert max(slots) // 16 == blocks - 1
    gk, gv = c.gather(0, slots)
    pick = np.unique(np.r_[0:40, n - 60:n, 16 * 960 - 20:16 * 960 + 20, np.random.default_rng(0).integers(0, n, 500)])
    _same_rows(gk[pick], kv8.bf16_bits(kv8.cached_values(k[pick])))
    _same_rows(gv[pick], kv8.bf16_bits(kv8.cached_values(v[pick])))
    backwards, _ = c.gather(0, slots[::-1])                  # another path reads the same rows
    assert np.array_equal(backwards[::-1], gk)
    c.close()


@pytest.mark.parametrize("where", ["prefix", "chunk", "history", "only"])
@pytest.mark.parametrize("bits", [0x7f80, 0xff80, 0x7fc0], ids=["inf", "-inf", "nan"])
def test_a_key_that_is_not_finite_leaves_no_finite_output(where, bits):
    """Held as NaN, it makes the logits of the queries that see it NaN, also where a split has no other key; all others
    equal the oracle's."""
    from paper_2603_14371_amd.harness import GpuWorld
    b = _TraceBuilder()
    pid = b.prefix(300, b.recipe(300, tag=100))
    act, dec, one = b.stream(pid, ACTION), b.stream(pid, DECODE), b.stream(pid, DECODE)
    b.tag = 10
    b.step([(dec, 150)], attend=False)                 # tag 10
    b.step([(act, 50), (dec, 1), (one, 1)])            # tag 11
    w = _workload("nan_key", 5181, 1, 512, b.trace)
    src = synth.DataSource(w["seed"])
    tag, row = {"prefix": (100, 17), "chunk": (11, 9), "history": (10, 70), "only": (11, 51)}[where]

    def planted(recipe, layer, what, n):
        x = src(recipe, layer, what, n).copy()
        if what == "k" and recipe["tag"] == tag:
            x[row - recipe["tok0"], 77] = bits
        return x

    gw = GpuWorld(w, planted, poison=True, kv8=True)
    ow = OracleWorld(w["num_blocks"], 1, kv8.cached_source(src), w["scale"])
    for op in w["trace"]:
        g, o = gw.apply(op), ow.apply(op)
    gw.close()
    got, ref = g["O"][0], o["O"][0]
    sees = {"prefix": list(range(52)), "chunk": list(range(50)), "history": [50], "only": [51]}[where]
    assert np.isnan(widen_bf16(got[sees])).all() and np.isnan(g["LSE"][0][sees]).all()
    rest = np.setdiff1d(np.arange(len(ref)), sees)
    if len(rest):
        assert_o_close(got[rest], ref[rest], where)
        assert_lse_close(g["LSE"][0][rest], o["LSE"][0][rest], where)


def test_a_query_that_is_not_finite_leaves_the_others_alone():
    from paper_2603_14371_amd.harness import GpuWorld
    b = _TraceBuilder()
    pid = b.prefix(300)
    act, dec = b.stream(pid, ACTION), b.stream(pid, DECODE)
    b.step([(act, 9), (dec, 1)])
    w = _workload("nan_query", 77, 1, 64, b.trace)
    src = synth.DataSource(w["seed"])

    def planted(recipe, layer, what, n):
        x = src(recipe, layer, what, n).copy()
        if what == "q":
            x[3, 2, 100], x[9, 5, 0] = 0x7fc0, 0x7f80
        return x

    gw = GpuWorld(w, planted, kv8=True)
    ow = OracleWorld(w["num_blocks"], 1, kv8.cached_source(src), w["scale"])
    for op in w["trace"]:
        g, o = gw.apply(op), ow.apply(op)
    gw.close()
    bad = np.zeros((10, 8), dtype=bool)
    bad[3, 2] = bad[9, 5] = True
    got = widen_bf16(g["O"][0])
    assert not np.isfinite(got[bad]).any() and not np.isfinite(g["LSE"][0][bad]).any()
    for r in range(10):
        ok = ~bad[r]
        assert_o_close(g["O"][0][r][ok], o["O"][0][r][ok], "row %d" % r)


@pytest.mark.parametrize("sizes", ["zeros", "zeros_then_normal", "tiny", "huge"])
def test_values_at_the_ends_of_the_range(sizes):
    """Rows of zeros (the lowest exponent), of 2^-120 and of 2^120: the unit that an item's sums go by follows."""
    from paper_2603_14371_amd.harness import GpuWorld
    b = _TraceBuilder()
    pid = b.prefix(400, b.recipe(400, tag=100))
    act, dec = b.stream(pid, ACTION), b.stream(pid, DECODE)
    b.step([(dec, 600)], attend=False)
    b.step([(act, 20), (dec, 1)])
    w = _workload("ends", 13, 1, 128, b.trace)
    src = synth.DataSource(w["seed"])
    shift = {"tiny": -120, "huge": 120}.get(sizes, 0)

    def sized(recipe, layer, what, n):
        x = src(recipe, layer, what, n).copy()
        if what == "v":
            at = np.arange(n) + recipe["tok0"]
            if sizes == "zeros":
                x[:] = 0
            elif sizes == "zeros_then_normal":
                x[at % 256 < 128] = 0
            else:                                # exponents moved, as far as they stay those of normal numbers
                e = (x >> 7) & 0xff
                moved = np.clip(e.astype(np.int32) + shift, 1, 250)
                x = ((x & 0x807f) | (moved << 7)).astype(np.uint16)
        return x

    gw = GpuWorld(w, sized, kv8=True, poison=True)
    ow = OracleWorld(w["num_blocks"], 1, kv8.cached_source(sized), w["scale"])
    for op in w["trace"]:
        g, o = gw.apply(op), ow.apply(op)
    gw.close()
    if sizes == "zeros":
        assert not (g["O"][0] & 0x7fff).any()
    else:
        assert_o_close_scaled(g["O"][0], o["O"][0], 2.0 ** shift)
    assert_lse_close(g["LSE"][0], o["LSE"][0], sizes)


@pytest.mark.parametrize("own", [65536, 65537])
def test_histories_of_more_than_65536_tokens(own):
    """Longer ones are cut into splits of 512."""
    b = _TraceBuilder()
    d = b.stream(-1, DECODE)
    b.step([(d, own - 2)], attend=False)
    b.step([(d, 2)])
    w = _workload("longer", 23, 1, 4100, b.trace)
    gw, _ = run_both8(w, poison=True, max_partials=1024)
    gw.close()


@pytest.mark.parametrize("own", [40, 9000], ids=["short", "merged_by_many"])
def test_a_captured_layer_follows_its_inputs(own):
    """Turning, storing, attention and read-back captured twice (two graphs of one batch, and a second batch), replayed
    in turn with eager work and new inputs between: every replay gives what eager calls give."""
    import torch
    from paper_2603_14371_amd import binding as B
    from paper_2603_14371_amd.harness import GpuWorld
    b = _TraceBuilder()
    pid = b.prefix(500)
    act, dec = b.stream(pid, ACTION), b.stream(pid, DECODE)
    b.step([(dec, own)], attend=False)
    w = _workload("captured", 3, 2, 800, b.trace)
    gw = GpuWorld(w, synth.DataSource(3), kv8=True, poison=True, max_q_tokens=64)
    gw.run(w["trace"])
    freqs = torch.from_numpy(B.oxy_rotary_freqs(10000.0, 128)[0]).cuda()
    turn = B.make_rotary(freqs.data_ptr(), 128)
    batches, buffers, graphs = [], [], []
    for m in (1, 2):
        items = [(act, 20), (dec, m)]
        batches.append(B.oxy_batch_build(gw.pool, items, 0, gw._stream()))
        n = 20 + m
        buffers.append(dict(n=n, wide=torch.zeros((n, 10, 256), dtype=torch.bfloat16, device="cuda"),
                            pos=torch.zeros(n, dtype=torch.int32, device="cuda"),
                            q=torch.zeros((n, 8, 256), dtype=torch.bfloat16, device="cuda"),
                            o=torch.zeros((2, n, 8, 256), dtype=torch.bfloat16, device="cuda"),
                            lse=torch.zeros((2, n, 8), device="cuda"),
                            kv=torch.zeros((2, 2, n, 256), dtype=torch.bfloat16, device="cuda")))

    def layer_calls(i, s):
        t, batch = buffers[i], batches[i]
        wide = t["wide"]
        slots = B.oxy_batch_slots(batch)
        B.oxy_rotary(turn, t["pos"].data_ptr(), wide.data_ptr(), 5120, wide.data_ptr(), 5120, t["n"], 1, s)
        for layer in range(2):
            B.oxy_rotary_append(gw.pool, batch, layer, turn, t["pos"].data_ptr(), wide.data_ptr(), 5120, t["q"].data_ptr(),
                                wide[:, 8].data_ptr(), 5120, wide[:, 9].data_ptr(), 5120, s)
            B.oxy_mixed_attention(gw.pool, batch, layer, t["q"].data_ptr(), t["o"][layer].data_ptr(),
                                  t["lse"][layer].data_ptr(), 0.0625, s)
        B.oxy_gather_kv_layers(gw.pool, 0, 2, slots, t["kv"][0].data_ptr(), t["kv"][1].data_ptr(), t["n"] * 512, s)

    def fill(i, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        t = buffers[i]
        t["wide"].normal_(generator=g)
        t["pos"].random_(0, 9000, generator=g)
        for x in ("q", "o", "lse", "kv"):
            t[x].fill_(7)

    def results(i):
        torch.cuda.synchronize()
        return [buffers[i][x].clone() for x in ("wide", "q", "o", "lse", "kv")]

    side = torch.cuda.Stream()
    for i in (0, 0, 1):
        fill(i, 0)
        layer_calls(i, gw._stream())
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            layer_calls(i, torch.cuda.current_stream().cuda_stream)
        graphs.append((i, graph))
    for seed in range(1, 5):
        for i, graph in graphs:
            fill(i, seed)
            layer_calls(i, gw._stream())
            want = results(i)
            fill(i, seed)
            torch.cuda.synchronize()
            graph.replay()
            for x, y in zip(want, results(i)):
                assert torch.equal(x, y) and torch.isfinite(x).all()
    del graphs
    for batch in batches:
        B.oxy_batch_destroy(batch)
    gw.close()


def test_recordings_on_both_sides_of_the_merge_by_many():
    """A request whose split results pass 32 while its steps are recorded and replayed."""
    import torch
    from paper_2603_14371_amd import binding as B
    from paper_2603_14371_amd.harness import GpuWorld, bits_of, to_device_bf16
    b = _TraceBuilder()
    pid = b.prefix(100)
    dec = b.stream(pid, DECODE)
    b.step([(dec, 30 * 32 - 3)], attend=False)
    w = _workload("passes", 8, 2, 100, b.trace)
    data = synth.DataSource(8)
    outs = {}
    for flags in (0, B.STEP_GRAPH):
        gw = GpuWorld(w, data, kv8=True, stream_split_tokens=32, max_q_tokens=16)
        gw.run(w["trace"])
        s, parts = gw._stream(), []
        k, v, q = (torch.stack([to_device_bf16(data(b.recipe(1, tag=5), l, x, 1), gw.device) for l in range(2)]) for x in "kvq")
        o, lse, got = torch.zeros_like(q), torch.zeros((2, 1, 8), device="cuda"), []
        for step in range(8):
            batch = B.oxy_batch_build(gw.pool, [(dec, 1)], 0, s)
            parts.append(B.oxy_batch_info(batch)[3])
            o.zero_()
            B.oxy_step_layers(gw.pool, batch, 0, 2, k.data_ptr(), v.data_ptr(), 512, q.data_ptr(), o.data_ptr(), 4096,
                              lse.data_ptr(), 32, gw.scale, flags, None, s)
            torch.cuda.synchronize()
            got.append((bits_of(o), lse.cpu().numpy().copy()))
            B.oxy_batch_destroy(batch)
        outs[flags] = got
        assert min(parts) == 32 and max(parts) == 33
        gw.close()
    for a, c in zip(outs[0], outs[B.STEP_GRAPH]):
        assert np.array_equal(a[0], c[0]) and np.array_equal(a[1], c[1]) and a[0].any()


@pytest.mark.parametrize("lens,first", [([2049], [0]), ([2061], [3]), ([1] * 2100, [5]), (None, None)],
                         ids=["whole", "ragged", "single", "mixed"])
def test_large_appends_store_what_small_ones_do(lens, first):
    """More than 2048 tokens go by another kernel; an append that turns by nothing stores the same rows one by one."""
    import torch
    from paper_2603_14371_amd import binding as B
    rng = np.random.default_rng(5)
    if lens is None:
        lens = rng.integers(1, 60, 90).tolist()
        first = rng.integers(0, 30, 90).tolist()
    first = first * (len(lens) // len(first))
    n = sum(lens)
    assert n > 2048
    x = rng.standard_normal((2, n, 256)) * 2.0 ** rng.integers(-30, 30, (2, n, 1))
    x[0, 7], x[1, 9], x[0, 11, 3], x[1, 12, 200] = 0, 0, np.inf, np.nan
    rows = torch.from_numpy(x).cuda().to(torch.bfloat16)
    positions = torch.zeros(n, dtype=torch.int32, device="cuda")
    freqs = torch.ones(1, dtype=torch.float64, device="cuda")
    stored = []
    for turning in (False, True):
        blocks = sum((m + f + 15) // 16 for m, f in zip(lens, first))
        order = np.random.default_rng(1).permutation(blocks).tolist()
        cfg = B.make_config(2, blocks, flags=B.POOL_KV_FP8, max_q_tokens=16, max_append_tokens=16 * blocks, free_order=order)
        kv = torch.full((B.oxy_kv_bytes(cfg),), 0x5a, dtype=torch.uint8, device="cuda")
        ws = torch.empty(B.oxy_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        cfg.kv_base, cfg.kv_bytes, cfg.workspace, cfg.workspace_bytes = kv.data_ptr(), kv.numel(), ws.data_ptr(), ws.numel()
        pool, s = B.oxy_pool_create(cfg), torch.cuda.current_stream().cuda_stream
        sids = [B.oxy_stream_create(pool, -1, DECODE) for _ in lens]
        before = [(sid, f) for sid, f in zip(sids, first) if f]
        if before:                                   # these rows stay unwritten
            B.oxy_batch_destroy(B.oxy_batch_build(pool, before, B.BATCH_APPEND_ONLY, s))
        batch = B.oxy_batch_build(pool, list(zip(sids, lens)), B.BATCH_APPEND_ONLY, s)
        if turning:
            B.oxy_rotary_append(pool, batch, 1, B.make_rotary(freqs.data_ptr(), 2), positions.data_ptr(), 0, 0, 0,
                                rows[0].data_ptr(), 512, rows[1].data_ptr(), 512, s)
        else:
            B.oxy_stream_append(pool, batch, 1, rows[0].data_ptr(), rows[1].data_ptr(), s)
        torch.cuda.synchronize()
        stored.append(kv.cpu().numpy())
        B.oxy_batch_destroy(batch)
        B.oxy_pool_destroy(pool)
    assert np.array_equal(*stored)
    half = len(stored[0]) // 2
    assert (stored[0][:half] == 0x5a).all() and (stored[0][half:] != 0x5a).sum() > 500 * n


@pytest.mark.parametrize("seed", range(100, 108))
def test_random_traces(seed):
    """Forks, rewinds, releases, chunks, drafts and histories in any order, a pool full of NaN bytes; at the end every
    live row is read back."""
    from test_gpu_fuzz import random_trace
    gw, ow = run_both8(random_trace(seed), layers=[0, 2], poison=True, max_q_tokens=1024, max_append_tokens=4096)
    assert_pool_contents_equal(gw, ow)
    gw.close()


def test_blocks_beyond_4_gib():
    """Block ids whose bytes lie past 32 bits, codes and exponents: written by all three appends, read back, attended."""
    b = _TraceBuilder()
    pid = b.prefix(333)
    act, dec = b.stream(pid, ACTION), b.stream(pid, DECODE)
    b.step([(dec, 3000)], attend=False)
    b.step([(act, 30), (dec, 1)])
    n = (9 << 29) // 8192
    order = np.roll(np.arange(n, dtype=np.int32)[::-1], -3)
    gw, ow = run_both8(_workload("far", 41, 1, n, b.trace, free_order=order), max_partials=4096)
    assert gw.prefix_slots(pid)[0] * 512 > 1 << 32
    assert_pool_contents_equal(gw, ow)
    gw.close()


@pytest.mark.parametrize("hist", [50, 9000], ids=["short", "merged_by_many"])
def test_kernels_carry_their_events(hist):
    import ctypes
    import torch
    from paper_2603_14371_amd import binding as B
    from paper_2603_14371_amd.harness import GpuWorld
    b = _TraceBuilder()
    dec = b.stream(b.prefix(200), DECODE)
    b.step([(dec, hist)], attend=False)
    w = _workload("events", 8, 2, 800, b.trace)
    gw = GpuWorld(w, synth.DataSource(8), kv8=True, max_q_tokens=16)
    gw.run(w["trace"])
    x, s = torch.randn(2, 1, 8, 256, device="cuda").to(torch.bfloat16), gw._stream()
    outs = [torch.zeros_like(x) for _ in range(2)]
    events = [torch.cuda.Event(enable_timing=True) for _ in range(8)]
    for e in events:
        e.record()                                  # creates the handle
    raw = (ctypes.c_void_p * 8)(*[e.cuda_event for e in events])
    batch = B.oxy_batch_build(gw.pool, [(dec, 1)], 0, s)
    for out, ev in zip(outs, (None, raw)):
        B.oxy_step_layers(gw.pool, batch, 0, 2, x.data_ptr(), x.data_ptr(), 4096, x.data_ptr(), out.data_ptr(), 4096, 0, 0,
                          gw.scale, 0, ev, s)
    torch.cuda.synchronize()
    for i in range(0, 8, 2):
        assert 0 < events[i].elapsed_time(events[i + 1]) < 10
    assert torch.equal(*outs) and outs[0].any()
    B.oxy_batch_destroy(batch)
    gw.close()


@pytest.mark.parametrize("n_new,hist,bad", [(2, 0, 1), (3, 0, 2), (8, 0, 4), (13, 5, 6), (5, 125, 3), (6, 253, 4), (13, 250, 1),
                                            (50, 0, 20), (60, 700, 59), (4, 509, 2), (16, 1000, 1)])
def test_a_value_that_is_not_finite_does_not_reach_tokens_before_it(n_new, hist, bad):
    """Of several new tokens, some do not see the value of the token `bad`: their weight of it is zero, and zero times NaN
    is not."""
    from paper_2603_14371_amd.harness import GpuWorld
    b = _TraceBuilder()
    dec = b.stream(b.prefix(70), DECODE)
    b.tag = 10
    if hist:
        b.step([(dec, hist)], attend=False)
    b.tag = 20
    b.step([(dec, n_new)])
    w = _workload("later", 31, 1, 128, b.trace)
    src = synth.DataSource(w["seed"])

    def planted(recipe, layer, what, n):
        x = src(recipe, layer, what, n).copy()
        if what == "v" and recipe["tag"] == 20:
            x[bad, 133], x[bad, 200] = 0x7fc0, 0xff80
        return x

    def without(recipe, layer, what, n):
        x = planted(recipe, layer, what, n)
        x = x if what == "q" else kv8.bf16_bits(kv8.cached_values(x))
        return np.where((x & 0x7fff) > 0x7f80, np.uint16(0), x)

    gw = GpuWorld(w, planted, poison=True, kv8=True)
    ow = OracleWorld(w["num_blocks"], 1, without, w["scale"])
    for op in w["trace"]:
        g, o = gw.apply(op), ow.apply(op)
    gw.close()
    got, ref = g["O"][0], o["O"][0]
    assert_o_close(got[:bad], ref[:bad], "before")
    assert not np.isfinite(widen_bf16(got[bad:][:, :, [133, 200]])).any()
    assert_o_close(got[:, :, :128], ref[:, :, :128], "other dims")
    assert_lse_close(g["LSE"][0], o["LSE"][0], "all")
