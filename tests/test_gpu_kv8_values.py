"""Values of very different size in a pool in 8 bits: what a query does not see, or gives no weight, leaves its output alone.

Tolerances.  A key's weight times the power of two of its value is held as one fp16 number, whose unit goes by the largest
that any one key adds to the query: off by 2^-11 of itself or 2^-20 of that largest (at most 2^-12 for 256 keys).  A split's
sums are stored as fp16, off by 2^-11 of themselves or of the largest of 64 dims.  The output is rounded to bf16, 2^-8.
Where outputs are of the order of one these are within 2e-3 + 1e-2 |ref|, the bound of all attention tests; where they are
not, the same is asked in units of the row's largest output."""
import numpy as np
import pytest

from oracle import kv8
from oracle.attention import widen_bf16
from oracle.replay import OracleWorld
from paper_2603_14371_amd import synth
from paper_2603_14371_amd.synth import ACTION, DECODE, _TraceBuilder, _workload
from parity_util import assert_lse_close, assert_o_close

pytestmark = pytest.mark.gpu
LOWEST = 0xFF7F                      # of bf16


def scaled(bits, power):
    """bf16 numbers times 2^power, as far as they stay normal."""
    e = ((bits >> 7) & 0xff).astype(np.int32)
    return np.where(e == 0, bits, (bits & 0x807f) | (np.clip(e + power, 1, 254) << 7)).astype(np.uint16)


def outputs(w, source):
    """The last step's bits and log-sum-exps, and the oracle's on what the pool holds."""
    from paper_2603_14371_amd.harness import GpuWorld
    gw = GpuWorld(w, source, poison=True, kv8=True, max_partials=4096)
    ow = OracleWorld(w["num_blocks"], 1, kv8.cached_source(source), w["scale"])
    for op in w["trace"]:
        g, o = gw.apply(op), ow.apply(op)
    gw.close()
    return g["O"][0], g["LSE"][0], o["O"][0], o["LSE"][0]


def assert_close_by_row(bits, ref):
    unit = np.abs(ref).max(axis=-1, keepdims=True)
    assert np.all(np.abs(widen_bf16(bits) / unit - ref / unit) <= 2e-3 + 1e-2 * np.abs(ref / unit))


@pytest.mark.parametrize("size", [21, 28, 40, 100, "lowest", -60])
@pytest.mark.parametrize("n_new,hist,bad", [(2, 0, 1), (3, 0, 2), (8, 0, 4), (13, 5, 6), (5, 125, 3), (6, 253, 4), (13, 250, 1),
                                            (50, 0, 20), (60, 700, 59), (4, 509, 2), (16, 1000, 1)])
def test_a_finite_value_does_not_reach_tokens_before_it(n_new, hist, bad, size):
    """Of several new tokens those before `bad` do not see its value: their outputs are, bit for bit, what they are beside
    any other value there."""
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
            x[bad] = LOWEST if size == "lowest" else scaled(x[bad], size)
        return x

    got, lse, ref, ref_lse = outputs(w, planted)
    assert_o_close(got[:bad], ref[:bad], "before")
    if size != "lowest":             # its values are held as infinite
        assert_close_by_row(got, ref)
    assert_lse_close(lse, ref_lse, "all")
    plain = outputs(w, src)
    assert np.array_equal(got[:bad], plain[0][:bad]) and np.array_equal(lse, plain[1])


@pytest.mark.parametrize("size", [13, 25, 40, 90])
@pytest.mark.parametrize("where", ["prefix", "chunk", "history", "new"])
def test_a_large_value_of_no_weight_leaves_the_others(where, size):
    """One key, at a logit 2^-size and far less behind the others', has values 2^size as large."""
    b = _TraceBuilder()
    pid = b.prefix(420, b.recipe(420, tag=100))
    act, dec, few = b.stream(pid, ACTION), b.stream(pid, DECODE), b.stream(pid, DECODE)
    b.tag = 10
    b.step([(dec, 700)], attend=False)                 # tag 10
    b.step([(act, 50), (dec, 1), (few, 5)])            # tag 11
    w = _workload("no_weight", 17, 1, 512, b.trace)
    src = synth.DataSource(w["seed"])
    tag, row = {"prefix": (100, 130), "chunk": (11, 9), "history": (10, 300), "new": (11, 52)}[where]

    def planted(recipe, layer, what, n):
        x = src(recipe, layer, what, n).copy()
        if what == "q":
            x[:, :, 0] = 0x4200                        # 32: a key's first element counts twice in the logit
        if what == "k":
            x[:, 0] = 0
        if recipe["tag"] == tag and row - recipe["tok0"] < n:
            if what == "k":
                x[row - recipe["tok0"], 0] = 0xC2C8    # -100: a weight of 2^-288
            if what == "v":
                x[row - recipe["tok0"]] = scaled(x[row - recipe["tok0"]], size)
        return x

    got, lse, ref, ref_lse = outputs(w, planted)
    assert_o_close(got, ref, where)
    assert_lse_close(lse, ref_lse, where)


@pytest.mark.parametrize("logit", [-20, -60, -80])
@pytest.mark.parametrize("first", [True, False], ids=["before", "behind"])
def test_a_small_weight_and_a_large_value_count_by_their_product(logit, first):
    """A key at e^logit of the others' weight, with values that make up for it: its share of the output is that of the
    others together, whichever round of keys comes first."""
    power = int(round(-logit / np.log(2)))
    b = _TraceBuilder()
    pid = b.prefix(300, b.recipe(300, tag=100))
    act, dec = b.stream(pid, ACTION), b.stream(pid, DECODE)
    b.step([(act, 50), (dec, 3)])
    w = _workload("product", 19, 1, 128, b.trace)
    src = synth.DataSource(w["seed"])
    row = 3 if first else 297

    def planted(recipe, layer, what, n):
        x = src(recipe, layer, what, n).copy()
        if what == "q":
            x[:, :, 0] = 0x4180                        # 16: a key's first element is its logit's
        if what == "k":
            x[:, 0] = 0
        if recipe["tag"] == 100 and what != "q":
            if what == "k":
                x[row, 0] = (np.float32(logit).view(np.uint32) >> 16).astype(np.uint16)
            else:
                x[row] = scaled(x[row], power + 6)
        return x

    got, lse, ref, ref_lse = outputs(w, planted)
    assert_close_by_row(got, ref)
    assert_lse_close(lse, ref_lse, "all")


@pytest.mark.parametrize("spread", [10, 12, 13, 14, 24])
def test_sizes_that_differ_within_a_split(spread):
    """Rows of two sizes in turn, on both sides of where units go by the row; zeros among them."""
    b = _TraceBuilder()
    pid = b.prefix(333, b.recipe(333, tag=100))
    act, dec, few = b.stream(pid, ACTION), b.stream(pid, DECODE), b.stream(pid, DECODE)
    b.step([(dec, 400)], attend=False)
    b.step([(act, 50), (dec, 1), (few, 7)])
    w = _workload("two_sizes", 29, 1, 128, b.trace)
    src = synth.DataSource(w["seed"])

    def planted(recipe, layer, what, n):
        x = src(recipe, layer, what, n).copy()
        if what == "v":
            at = np.arange(n) + recipe["tok0"]
            x[at % 3 == 1] = scaled(x[at % 3 == 1], -spread)
            x[at % 50 == 7] = 0
        return x

    got, lse, ref, ref_lse = outputs(w, planted)
    assert_o_close(got, ref, "all")
    assert_lse_close(lse, ref_lse, "all")


@pytest.mark.parametrize("n_new", [1, 3, 9])
@pytest.mark.parametrize("keys", [1, 2, 3, 5, 17, 64, 100, 300, 700])
def test_outputs_within_what_each_rounding_may_cost(keys, n_new):
    """Element by element, also where the terms of a sum cancel.  With A = sum P |v| / sum P and M the largest A of the 64 dims
    that share an exponent: weights in fp16 cost 2^-11 A, split results 2^-11 M (the two together at most 2^-20 M more), the
    output 2^-8 |ref|.  Logits below 16 in 32 bits, eight products of 32 dims after one another: 16 * 8 * 2^-24 of each
    weight, and as much of their sum, 2^-16 A together."""
    import torch
    from test_gpu_kv8 import Cache
    c = Cache(n_layers=1, blocks=80)
    rng = np.random.default_rng(keys)
    bits = lambda *shape: (rng.standard_normal(shape).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)  # noqa: E731
    pk, pv, nk, nv, q = bits(keys, 256), bits(keys, 256), bits(n_new, 256), bits(n_new, 256), bits(n_new, 8, 256)
    up = [c.up(x) for x in (pk, pv, nk, nv, q)]
    pid = c.B.oxy_prefix_create(c.pool)
    c.B.oxy_prefix_append(c.pool, pid, 0, up[0].data_ptr(), up[1].data_ptr(), keys, 0, c.stream)
    sid = c.B.oxy_stream_create(c.pool, pid, DECODE)
    batch = c.B.oxy_batch_build(c.pool, [(sid, n_new)], 0, c.stream)
    c.B.oxy_stream_append(c.pool, batch, 0, up[2].data_ptr(), up[3].data_ptr(), c.stream)
    out = torch.zeros_like(up[4])
    c.B.oxy_mixed_attention(c.pool, batch, 0, up[4].data_ptr(), out.data_ptr(), 0, 1.0 / 16, c.stream)
    got = widen_bf16(c.back(out))
    c.B.oxy_batch_destroy(batch)
    c.close()
    k, v = (kv8.cached_values(np.concatenate(x)) for x in ((pk, nk), (pv, nv)))
    for t in range(n_new):
        n = keys + t + 1
        s = widen_bf16(q[t]) @ k[:n].T / 16
        assert np.abs(s).max() < 16
        p = np.exp(s - s.max(axis=1, keepdims=True))
        p /= p.sum(axis=1, keepdims=True)
        ref, a = p @ v[:n], p @ np.abs(v[:n])
        m = np.repeat(a.reshape(8, 4, 64).max(axis=2), 64, axis=1)
        bound = 2.0 ** -8 * np.abs(ref) + (2.0 ** -11 + 2.0 ** -16) * a + (2.0 ** -11 + 2.0 ** -20) * m
        assert np.all(np.abs(got[t] - ref) <= bound), (np.abs(got[t] - ref) / bound).max()


def _sized(data):
    """Values of sizes up to 2^45 apart, by their own bits, so that a row is the same in any batch."""
    def read(recipe, layer, what, n):
        x = data(recipe, layer, what, n)
        if what != "v":
            return x
        x = x.copy()
        for rest, power in ((0, 25), (1, -20)):
            rows = x[:, 1] % 7 == rest
            x[rows] = scaled(x[rows], power)
        x[x[:, 1] % 61 == 3] = 0
        return x
    return read


def _outputs_of(me, others, prefixes):
    """Items are (prefix, kind, history, new tokens, tag).  `me`'s outputs in one step with `others` before and behind it, and
    the oracle's; how many query tokens the widest record of the launch has."""
    from oracle.attention import attend_item
    from paper_2603_14371_amd import binding as B
    from paper_2603_14371_amd.harness import GpuWorld
    b = _TraceBuilder()
    pids = [b.prefix(n, b.recipe(n, tag=30 + i)) for i, n in enumerate(prefixes)]
    half = len(others) // 2
    items = []
    for p, kind, hist, n, tag in others[:half] + [me] + others[half:]:
        sid = b.stream(pids[p], kind)
        if hist:
            b.step([(sid, hist)], attend=False, recipe={"tag": 500 + tag, "tok0": 0, "n_total": hist})
        items.append((sid, n, tag))
    w = _workload("sized", 4, 1, 3000, b.trace)
    data = _sized(synth.DataSource(4))
    gw = GpuWorld(w, data, kv8=True, poison=True, max_q_tokens=2048, max_append_tokens=32768, max_partials=40000)
    gw.run(w["trace"])
    gw.data_fn = lambda recipe, layer, what, n: np.concatenate(
        [data({"tag": 900 + tag, "tok0": 0, "n_total": m}, layer, what, m) for _, m, tag in items])
    batch = B.oxy_batch_build(gw.pool, [(s, n) for s, n, _ in items], 0, gw._stream())
    widest = max(r[1] for r in B.oxy_batch_records(batch))
    B.oxy_batch_destroy(batch)
    for (sid, n, tag), it in zip(items, others[:half] + [me] + others[half:]):
        if it[1] == DECODE:
            B.oxy_stream_rewind(gw.pool, sid, it[2])
    r = gw.step({"op": "step", "items": [(s, n) for s, n, _ in items], "attend": True, "data": None})
    gw.close()
    at = sum(n for _, n, _ in items[:half])
    p, kind, hist, n, tag = me
    got = r["O"][0][at:at + n], r["LSE"][0][at:at + n]
    rec = lambda t, m: {"tag": t, "tok0": 0, "n_total": m}  # noqa: E731
    held = lambda t, m, what: kv8.bf16_bits(kv8.cached_values(data(rec(t, m), 0, what, m)))  # noqa: E731
    own = [np.concatenate([held(500 + tag, hist, x), held(900 + tag, n, x)]) if hist else held(900 + tag, n, x) for x in "kv"]
    ref = attend_item(0 if kind == ACTION else 1, data(rec(900 + tag, n), 0, "q", n), held(30 + p, prefixes[p], "k"),
                      held(30 + p, prefixes[p], "v"), own[0], own[1], w["scale"])
    return got, ref, widest


@pytest.mark.parametrize("me,prefix", [((0, ACTION, 0, 50, 7), 2048), ((0, ACTION, 0, 13, 7), 300), ((0, DECODE, 40, 1, 7), 900),
                                       ((0, DECODE, 1100, 30, 7), 300), ((0, DECODE, 0, 6, 7), 900)], ids=str)
def test_sizes_in_items_of_every_width(me, prefix):
    """The same bits whatever shares the launch, and as the oracle says; among many an item has eight query tokens."""
    chunks = [(i % 8, ACTION, 0, 50, 100 + i) for i in range(8)]
    alone, ref, _ = _outputs_of(me, [], [prefix])
    assert_close_by_row(alone[0], ref[0])
    assert_lse_close(alone[1], ref[1], "alone")
    widths = set()
    for others in (chunks[1:4], chunks[1:] + [(0, DECODE, 20 * i, 1, 20 + i) for i in range(20)]):
        got, _, widest = _outputs_of(me, others, [prefix] + [2048] * 7)
        widths.add(int(widest))
        assert np.array_equal(got[0], alone[0]) and np.array_equal(got[1], alone[1])
    assert 8 in widths
