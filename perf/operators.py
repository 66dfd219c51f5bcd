"""Workloads of the key/value cache held in 8 bits, the attention that reads it, and rotary positions.

Geometry is the library's: 8 query heads over one KV head, head_dim 256, pages of 16 tokens, bf16 in
and out.  A cached row x (the key or the value of a token) is held as 256 e4m3 codes and the exponent
of a power-of-two scale, e = the smallest integer >= -126 with max|x| <= 448 * 2^e:

    code_i = e4m3(x_i * 2^-e), round to nearest even        value_i = code_i * 2^e

Attention of a query over its visible tokens (its observation's prefix, then its own tokens, causal for
requests and all of the chunk for action chunks) is softmax(q k / 16) v on those values.  A rotation by
positions turns pairs of a row's first `rot` dims: (x1 c - x2 s, x2 c + x1 s), c and s the amplitude
times cosine and sine of position * frequency.

`own` false: elementary torch operations; true: the library's calls.
"""
import math
import random

import numpy as np
import torch

own = False

HEADS, DIM, PAGE = 8, 256, 16
SCALE = 1.0 / 16.0
ROW = DIM * 2                    # bytes of a bf16 row
ROW8 = DIM + 1                   # bytes of a row in 8 bits, its exponent among them
QKV = (HEADS + 2) * DIM          # elements of a token's projected queries, key and value


def _case(name, kind, **kw):
    """kind: "store" = rows brought into a cache of `layers` layers and read back, as one observation's
    prefill (decoders = 0: prefix_len tokens) or as the histories of requests that move in;
    "attend" = the attention of a step whose rows are in the cache and whose descriptor is in hand, one
    call per layer; "step" = a whole step: descriptor, and per layer queries and new keys rotated, new rows
    cached, attention; "append" = the rotating append alone, rows read back; "rotate" = the queries and
    keys of prefix_len tokens rotated.
    prefixes x prefix_len observations; chunks action chunks of chunk_len queries (chunk i on observation
    i, counted round); decoders requests with own histories of hist_lo..hist_hi tokens and n_new new tokens
    each (request i on observation i // ceil(decoders / prefixes)).
    rot dims are rotated, "halves" or "pairs"; scaling: see _frequencies; first: position of token 0."""
    c = dict(kind=kind, layers=18, prefixes=1, prefix_len=832, chunks=0, chunk_len=50, decoders=0,
             hist_lo=1, hist_hi=1, n_new=1, lse=False, lengths=1, rot=DIM, layout="halves",
             scaling="none", factor=1.0, first=0)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one observation's prefill cache goes into all layers, and is read back (moved, checked)
        _case("store_observation", "store"),
        # a long document's, ragged at its end
        _case("store_long_prefix", "store", layers=6, prefix_len=16391),
        # four requests' histories move in with their streams and are read back
        _case("store_histories", "store", layers=6, prefixes=0, decoders=4, hist_lo=100,
              hist_hi=700, lengths=7),
        # the smallest attention: one layer, a 64-token observation, a chunk of 10 and a request
        _case("attend_tiny", "attend", layers=1, prefix_len=64, chunks=1, chunk_len=10, decoders=1,
              hist_lo=4, hist_hi=4, lse=True),
        # a denoise step of the frame's chunk together with one decode token
        _case("attend_frame", "attend", chunks=1, decoders=1, hist_lo=9, hist_hi=9),
        # chunks of eight observations, no language: the dense side
        _case("attend_chunks", "attend", layers=6, prefixes=8, prefix_len=2048, chunks=8),
        # drafts of 13 tokens for six requests on three observations, causal, ragged everywhere
        _case("attend_drafts", "attend", layers=6, prefixes=3, prefix_len=771, decoders=6,
              hist_lo=30, hist_hi=900, n_new=13, lse=True, lengths=4),
        # 64 requests in groups of eight on long observations, two chunks
        _case("attend_many", "attend", prefixes=8, prefix_len=2048, chunks=2, decoders=64, hist_lo=1,
              hist_hi=2048, lengths=5),
        # one request far into a long history, no observation
        _case("attend_long_history", "attend", layers=2, prefixes=0, decoders=1, hist_lo=131071,
              hist_hi=131071, lse=True),
        # a prefill's queries and keys, out of the projection's output, far out in a scaled context
        _case("rotate_prefill", "rotate", prefix_len=8192, scaling="bands", factor=8.0, first=100000),
        # the rotating append of a step: two chunks and 64 requests, a quarter of the head rotated
        _case("append_step", "append", layers=4, prefixes=8, prefix_len=200, chunks=2, decoders=64,
              hist_lo=1, hist_hi=300, rot=64, layout="pairs", scaling="linear", factor=4.0, lengths=3),
        # a whole step of the cross-frame loop: eight requests on their observations, one new chunk
        _case("step_cross_frame", "step", prefixes=8, chunks=1, decoders=8, hist_lo=16, hist_hi=512,
              lengths=2),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    """The same ranges: prefills of 1..16384 tokens, histories of up to 131072, up to 64 requests, eight
    chunks of 1..64 queries, up to 16 new tokens per request, either layout, every scaling."""
    kind = rng.choice(["store", "attend", "attend", "attend", "rotate", "append", "step"])
    c = dict(layers=rng.randint(1, 18), lse=rng.random() < 0.4, lengths=rng.randint(100, 1 << 20),
             rot=2 * _log_int(rng, 1, 128), layout=rng.choice(["halves", "pairs"]),
             scaling=rng.choice(["none", "linear", "base", "bands", "ramp"]),
             factor=round(rng.uniform(1.5, 32.0), 2), first=_log_int(rng, 1, 1 << 20))
    if rng.random() < 0.4:
        c["rot"] = DIM
    if kind == "rotate":
        return _case(None, kind, **dict(c, prefix_len=_log_int(rng, 1, 8192)))
    if kind == "store":
        c["layers"] = rng.randint(1, 6)
        if rng.random() < 0.6:
            return _case(None, kind, **dict(c, prefix_len=_log_int(rng, 1, 16384)))
        hi = _log_int(rng, 1, 4096)
        return _case(None, kind, **dict(c, prefixes=0, decoders=_log_int(rng, 1, 8), hist_hi=hi,
                                        hist_lo=rng.randint(1, hi)))
    if kind == "attend" and rng.random() < 0.25:     # few requests with long histories
        hi = _log_int(rng, 2000, 131072)
        c.update(prefixes=rng.randint(0, 1), prefix_len=_log_int(rng, 16, 2048),
                 decoders=rng.randint(1, 2), hist_lo=hi // 2, hist_hi=hi, layers=rng.randint(1, 2))
        return _case(None, kind, **c)
    hi = _log_int(rng, 1, 2048)
    c.update(prefixes=_log_int(rng, 1, 16), prefix_len=_log_int(rng, 1, 2048), hist_hi=hi,
             hist_lo=rng.randint(0, hi), chunk_len=rng.randint(1, 64))
    mix = rng.choice(["mixed", "mixed", "requests", "chunks"])
    if mix != "chunks":
        c["decoders"] = _log_int(rng, 1, 64)
        if rng.random() < 0.3:
            c["n_new"] = rng.randint(2, 16)
            c["decoders"] = min(c["decoders"], 12)
    if mix != "requests":
        c["chunks"] = rng.randint(1, min(8, c["prefixes"]))
    if kind == "append":
        c["layers"] = rng.randint(1, 4)
    c = _case(None, kind, **c)
    tokens = c["prefixes"] * c["prefix_len"] + sum(_histories(c)) + 1
    c["layers"] = max(1, min(c["layers"], 1000000 // tokens))
    return c


def _histories(case):
    rng = random.Random(case["lengths"])
    return [rng.randint(case["hist_lo"], case["hist_hi"]) for _ in range(case["decoders"])]


def _items(case):
    """(observation, own history, new tokens, bidirectional) of every item, in batch order."""
    if case["kind"] in ("store", "rotate"):
        return []
    items = [(i % max(1, case["prefixes"]), 0, case["chunk_len"], True)
             for i in range(case["chunks"])]
    share = -(-case["decoders"] // max(1, case["prefixes"]))
    items += [(i // share if case["prefixes"] else -1, h, case["n_new"], False)
              for i, h in enumerate(_histories(case))]
    return items


# ------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------
def _generator(seed, tag, layer):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + tag) * 64 + layer)
    return g


def _shape_rows(x, g):
    """Rows as a model's: tokens of different size, and channels of the keys (x[0]) that stand out."""
    gain = torch.exp(0.4 * torch.randn(DIM, device="cuda", generator=g))
    size = torch.exp2(0.7 * torch.randn(x.shape[:-1], device="cuda", generator=g))
    x *= size[..., None]
    x[0] *= gain
    return x.to(torch.bfloat16)


def _kv_rows(seed, tag, layer, n):
    """Keys and values of n tokens, [2, n, 256] bf16."""
    g = _generator(seed, tag, layer)
    return _shape_rows(torch.randn((2, n, DIM), device="cuda", generator=g), g)


def _stored_rows(case, seed, layer):
    """What the cache of one layer holds before the pass: observations, then histories."""
    parts = [_kv_rows(seed, 10 + i, layer, case["prefix_len"]) for i in range(case["prefixes"])]
    if sum(_histories(case)):
        parts.append(_kv_rows(seed, 1, layer, sum(_histories(case))))
    return torch.cat(parts, dim=1) if parts else torch.empty((2, 0, DIM), dtype=torch.bfloat16,
                                                              device="cuda")


def _projected(seed, layer, n):
    """Queries, key and value of n new tokens side by side, as a projection writes them: [n, 10 * 256]."""
    g = _generator(seed, 2, layer)
    q = torch.randn((n, HEADS * DIM), device="cuda", generator=g)
    kv = _shape_rows(torch.randn((2, n, DIM), device="cuda", generator=g), g)
    return torch.cat([q.to(torch.bfloat16), kv[0], kv[1]], dim=1)


def _positions(case):
    """Position of every new token: behind its observation and its own history."""
    if case["kind"] == "rotate":
        return list(range(case["first"], case["first"] + case["prefix_len"]))
    pos = []
    for p, h, n, _ in _items(case):
        at = case["first"] + (case["prefix_len"] if p >= 0 else 0) + h
        pos += list(range(at, at + n))
    return pos


BASE, ORIGINAL, LOW, HIGH, SLOW, FAST = 10000.0, 8192, 1.0, 4.0, 1.0, 32.0


def _frequencies(case):
    """Frequencies (radians per position) and amplitude.  linear: positions divided by the factor; base:
    the base raised so that the slowest pair is divided by it; bands: wavelengths beyond ORIGINAL / LOW
    divided, below ORIGINAL / HIGH kept, blended between; ramp: pairs blended by how many turns they make
    in ORIGINAL positions (SLOW..FAST), with an amplitude of 1 + 0.1 ln(factor)."""
    rot, factor, kind = case["rot"], case["factor"], case["scaling"]
    pairs = np.arange(rot // 2, dtype=np.float64)
    base = BASE
    if kind == "base" and rot > 2:
        base = BASE * factor ** (rot / (rot - 2.0))
    f = base ** (-2.0 * pairs / rot)
    if kind == "linear":
        return f / factor, 1.0
    if kind == "bands":
        keep = np.clip((ORIGINAL * f / (2 * math.pi) - LOW) / (HIGH - LOW), 0.0, 1.0)
        return f * (keep + (1.0 - keep) / factor), 1.0
    if kind == "ramp":
        pair_of = lambda turns: rot * math.log(ORIGINAL / (2 * math.pi * turns)) / (2 * math.log(BASE))  # noqa: E731
        lo, hi = max(0, math.floor(pair_of(FAST))), min(rot - 1, math.ceil(pair_of(SLOW)))
        slow = np.clip((pairs - lo) / max(hi - lo, 0.001), 0.0, 1.0)
        return f * (1.0 - slow) + f / factor * slow, 1.0 + 0.1 * math.log(factor)
    return f, 1.0


# ------------------------------------------------------------------------------------------
# plain forms
# ------------------------------------------------------------------------------------------
def _power(exponent):
    """2^exponent in 32 bits, from its bits."""
    return ((exponent + 127) << 23).view(torch.float32)


def _quantise(x):
    """bf16 rows -> e4m3 codes, exponents."""
    x = x.float()
    mantissa, exponent = torch.frexp(x.abs().amax(dim=-1))
    e = torch.clamp(torch.where(mantissa > 0.875, exponent - 8, exponent - 9), min=-126)
    return (x * _power(-e)[..., None]).to(torch.float8_e4m3fn), e


def _values(codes, e):
    return codes.float() * _power(e)[..., None]


def _rotate(x, positions, freqs, amplitude, rot, layout):
    """Rows [n, heads, 256] bf16 rotated by their tokens' positions; angles in 64 bits."""
    angle = positions.double()[:, None] * freqs
    c = (torch.cos(angle) * amplitude).float()[:, None]
    s = (torch.sin(angle) * amplitude).float()[:, None]
    y = x.float()
    if layout == "halves":
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        turned = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    else:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    return torch.cat([turned, y[..., rot:]], dim=-1).to(torch.bfloat16)


def _attention(s, q, keys, values):
    """Items side by side, padded to the longest: q [tokens, 8, 256], keys and values [rows, 256] of the
    cache in 32 bits -> outputs and log-sum-exps of the tokens."""
    n_items, most = s.token_of.shape
    k, v = keys[s.row_of], values[s.row_of]                              # [items, keys, 256]
    rows = q.float()[s.token_of].reshape(n_items, most * HEADS, DIM)
    logits = (rows @ k.transpose(1, 2)).view(n_items, most, HEADS, -1) * SCALE
    logits = logits.masked_fill(s.hidden[:, :, None, :], -math.inf)
    top = logits.amax(dim=-1, keepdim=True)
    p = torch.exp(logits - top)
    total = p.sum(dim=-1, keepdim=True)
    o = (p.view(n_items, most * HEADS, -1) @ v).view(n_items, most, HEADS, DIM) / total
    lse = (top + torch.log(total))[..., 0]
    return o[s.real].to(torch.bfloat16), lse[s.real]


class _State:
    """A cache with what is stored in it, and a step's resident inputs."""


def _prepare_plain(s, case, seed):
    """The cache as codes and exponents of rows (observations, histories, new tokens), and for every item
    the rows that its keys lie in."""
    items, n = s.items, s.n
    if case["kind"] in ("attend", "step"):
        stored = [_quantise(torch.cat([_stored_rows(case, seed, l), s.new_rows(l)], dim=1))
                  for l in range(case["layers"])]
        s.codes = torch.stack([c for c, _ in stored])                    # [L, 2, rows, 256]
        s.exponents = torch.stack([e for _, e in stored])
        P, at = case["prefix_len"], case["prefixes"] * case["prefix_len"]
        new = at + sum(_histories(case))
        most_new = max(it[2] for it in items)
        lists, tokens, hidden, t = [], [], [], 0
        for p, h, m, both in items:
            rows = (list(range(p * P, p * P + P)) if p >= 0 else []) + list(range(at, at + h))
            lists.append(rows + list(range(new + t, new + t + m)))
            tokens.append([t + min(i, m - 1) for i in range(most_new)])
            at, t = at + h, t + m
        most = max(len(r) for r in lists)
        s.row_of = torch.tensor([r + [0] * (most - len(r)) for r in lists], device="cuda")
        s.token_of = torch.tensor(tokens, device="cuda")
        key = torch.arange(most, device="cuda")
        last = torch.tensor([[len(r) - 1 if it[3] else len(r) - it[2] + min(i, it[2] - 1)
                              for i in range(most_new)] for r, it in zip(lists, items)], device="cuda")
        s.hidden = key > last[..., None]
        s.real = torch.tensor([[i < it[2] for i in range(most_new)] for it in items], device="cuda")
    s.freqs = torch.tensor(_frequencies(case)[0], dtype=torch.float64, device="cuda")
    s.amplitude = _frequencies(case)[1]


def _prepare_own(s, case, seed):
    """A pool in 8 bits with observations and histories stored, streams attached, and outputs allocated."""
    from paper_2603_14371_amd import binding as B
    s.B, s.pool, s.batch = B, None, None
    s.stream = torch.cuda.current_stream().cuda_stream
    freqs, amplitude = B.oxy_rotary_freqs(
        BASE, case["rot"], {"none": B.ROTARY_PLAIN, "linear": B.ROTARY_LINEAR, "base": B.ROTARY_BASE,
                            "bands": B.ROTARY_BANDS, "ramp": B.ROTARY_RAMP}[case["scaling"]],
        factor=case["factor"], low=SLOW if case["scaling"] == "ramp" else LOW,
        high=FAST if case["scaling"] == "ramp" else HIGH, original_len=ORIGINAL)
    s.freqs = torch.tensor(freqs, dtype=torch.float64, device="cuda")
    s.rotary = B.make_rotary(s.freqs.data_ptr(), case["rot"],
                             {"halves": B.ROTARY_HALVES, "pairs": B.ROTARY_PAIRS}[case["layout"]], amplitude)
    L, P, n, hist = case["layers"], case["prefix_len"], s.n, _histories(case)
    if case["kind"] == "rotate":
        s.out = torch.empty((P, HEADS + 1, DIM), dtype=torch.bfloat16, device="cuda")
        return
    pages = lambda m: -(-m // PAGE)  # noqa: E731
    blocks = max(1, case["prefixes"]) * pages(P) + sum(pages(h + case["n_new"]) for h in hist)
    blocks += case["chunks"] * pages(case["chunk_len"]) + 64
    order = list(range(blocks))
    random.Random(seed).shuffle(order)
    cfg = B.make_config(L, blocks, free_order=order, max_q_tokens=max(16, n),
                        max_append_tokens=max(16, n, sum(hist)), flags=B.POOL_KV_FP8,
                        max_partials=max(32 * max(16, n), 2048))
    s.kv = torch.empty(B.oxy_kv_bytes(cfg), dtype=torch.uint8, device="cuda")
    s.ws = torch.empty(B.oxy_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    cfg.kv_base, cfg.kv_bytes = s.kv.data_ptr(), s.kv.numel()
    cfg.workspace, cfg.workspace_bytes = s.ws.data_ptr(), s.ws.numel()
    s.pool = B.oxy_pool_create(cfg)
    if case["kind"] == "store":
        s.hist = hist
        s.back = torch.empty_like(s.rows)
        return
    pids = [B.oxy_prefix_create(s.pool) for _ in range(case["prefixes"])]
    sids = []
    for l in range(L):
        kv = _stored_rows(case, seed, l)
        for i, pid in enumerate(pids):
            B.oxy_prefix_append(s.pool, pid, l, kv[0, i * P:].data_ptr(), kv[1, i * P:].data_ptr(), P, 0,
                                s.stream)
        torch.cuda.synchronize()
    sids = [B.oxy_stream_create(s.pool, pids[p] if p >= 0 else -1, B.KIND_ACTION if both else B.KIND_DECODE)
            for p, _, _, both in s.items]
    s.batch_items = [(sid, it[2]) for sid, it in zip(sids, s.items)]
    s.lengths = [(sid, it[1]) for sid, it in zip(sids, s.items) if not it[3]]
    moved = [it for it in s.lengths if it[1]]
    if moved:
        b = B.oxy_batch_build(s.pool, moved, B.BATCH_APPEND_ONLY, s.stream)
        for l in range(L):
            kv = _stored_rows(case, seed, l)[:, case["prefixes"] * P:]
            B.oxy_stream_append(s.pool, b, l, kv[0].data_ptr(), kv[1].data_ptr(), s.stream)
            torch.cuda.synchronize()
        B.oxy_batch_destroy(b)
    s.out = torch.empty((L, n, HEADS, DIM), dtype=torch.bfloat16, device="cuda")
    s.lse = torch.empty((L, n, HEADS), device="cuda") if case["lse"] else None
    s.q_out = torch.empty((L, n, HEADS, DIM), dtype=torch.bfloat16, device="cuda")
    s.back = torch.empty((2, L, n, DIM), dtype=torch.bfloat16, device="cuda")
    if case["kind"] in ("attend", "append"):
        s.batch = B.oxy_batch_build(s.pool, s.batch_items, 0, s.stream)
    if case["kind"] == "attend":
        for l in range(L):
            kv = s.new_rows(l).contiguous()
            B.oxy_stream_append(s.pool, s.batch, l, kv[0].data_ptr(), kv[1].data_ptr(), s.stream)
            torch.cuda.synchronize()


class _Handles(_State):
    def __del__(self):
        if getattr(self, "pool", None) is not None:
            torch.cuda.synchronize()
            if self.batch is not None:
                self.B.oxy_batch_destroy(self.batch)
            self.B.oxy_pool_destroy(self.pool)
            self.pool = None


def prepare(case, seed):
    s = _Handles()
    s.case, s.items = case, _items(case)
    L = case["layers"]
    if case["kind"] == "store":
        rows = [_stored_rows(case, seed, l) for l in range(L)]
        s.n = rows[0].shape[1]
        s.rows = torch.stack(rows, dim=1)                                # [2, L, n, 256]
    else:
        s.n = case["prefix_len"] if case["kind"] == "rotate" else sum(it[2] for it in s.items)
        if case["kind"] == "rotate":
            L = 1
        s.qkv = torch.stack([_projected(seed, l, s.n) for l in range(L)])
        s.positions = torch.tensor(_positions(case), dtype=torch.int32, device="cuda")
        s.q = s.qkv[:, :, :HEADS * DIM].contiguous().view(L, s.n, HEADS, DIM)
        s.new_rows = lambda l: s.qkv[l, :, HEADS * DIM:].view(s.n, 2, DIM).transpose(0, 1)
    if own:
        _prepare_own(s, case, seed)
    else:
        _prepare_plain(s, case, seed)
    return s


# ------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------
def _run_plain(s):
    case, kind = s.case, s.case["kind"]
    if kind == "store":
        codes, e = _quantise(s.rows)
        return {"kv": _values(codes, e).to(torch.bfloat16)}
    turn = lambda x: _rotate(x, s.positions, s.freqs, s.amplitude, case["rot"], case["layout"])  # noqa: E731
    if kind == "rotate":
        return {"out": turn(s.qkv[0, :, :(HEADS + 1) * DIM].unflatten(1, (HEADS + 1, DIM)))}
    new = s.n
    outs, lses, queries, rows = [], [], [], []
    for l in range(case["layers"]):
        q, codes_e = s.q[l], None
        if kind in ("step", "append"):
            x = s.qkv[l].unflatten(1, (HEADS + 2, DIM))
            turned = turn(x[:, :HEADS + 1])
            q = turned[:, :HEADS]
            codes_e = _quantise(torch.stack([turned[:, HEADS], x[:, HEADS + 1]]))
        if kind == "append":
            queries.append(q)
            rows.append(_values(*codes_e).to(torch.bfloat16))
            continue
        if kind == "step":
            s.codes[l, :, -new:], s.exponents[l, :, -new:] = codes_e
        values = _values(s.codes[l], s.exponents[l])
        o, lse = _attention(s, q, values[0], values[1])
        outs.append(o)
        lses.append(lse)
    if kind == "append":
        return {"q": torch.stack(queries), "kv": torch.stack(rows, dim=1)}
    got = {"out": torch.stack(outs)}
    if case["lse"]:
        got["lse"] = torch.stack(lses)
    return got


def _slots_of(blocks, n):
    return (np.asarray(blocks, dtype=np.int64)[:, None] * PAGE + np.arange(PAGE)).reshape(-1)[:n]


def _read_back(s, slots):
    case = s.case
    s.B.oxy_gather_kv_layers(s.pool, 0, case["layers"], slots, s.back[0].data_ptr(), s.back[1].data_ptr(),
                             s.n * ROW, s.stream)


def _run_own(s):
    B, case, kind, L, n = s.B, s.case, s.case["kind"], s.case["layers"], s.n
    if kind == "store" and not case["decoders"]:
        pid = B.oxy_prefix_create(s.pool)
        B.oxy_prefix_append_layers(s.pool, pid, 0, L, s.rows[0].data_ptr(), s.rows[1].data_ptr(), n * ROW, n,
                                   0, s.stream)
        _read_back(s, _slots_of(B.oxy_prefix_blocks(s.pool, pid), n))
        B.oxy_prefix_release(s.pool, pid)
        return {"kv": s.back}
    if kind == "store":
        sids = [B.oxy_stream_create(s.pool, -1, B.KIND_DECODE) for _ in s.hist]
        batch = B.oxy_batch_build(s.pool, list(zip(sids, s.hist)), B.BATCH_APPEND_ONLY, s.stream)
        for l in range(L):
            B.oxy_stream_append(s.pool, batch, l, s.rows[0, l].data_ptr(), s.rows[1, l].data_ptr(), s.stream)
        _read_back(s, B.oxy_batch_slots(batch))
        B.oxy_batch_destroy(batch)
        for sid in sids:
            B.oxy_stream_release(s.pool, sid)
        return {"kv": s.back}
    if kind == "rotate":
        B.oxy_rotary(s.rotary, s.positions.data_ptr(), s.qkv.data_ptr(), QKV * 2, s.out.data_ptr(),
                     (HEADS + 1) * ROW, n, HEADS + 1, s.stream)
        return {"out": s.out}
    batch = s.batch
    if kind == "step":
        for sid, length in s.lengths:       # the same step again: drop the tokens it appended
            B.oxy_stream_rewind(s.pool, sid, length)
        batch = B.oxy_batch_build(s.pool, s.batch_items, 0, s.stream)
    for l in range(L):
        q = s.q[l]
        if kind in ("step", "append"):
            x, q = s.qkv[l].data_ptr(), s.q_out[l]
            B.oxy_rotary_append(s.pool, batch, l, s.rotary, s.positions.data_ptr(), x, QKV * 2, q.data_ptr(),
                                x + HEADS * ROW, QKV * 2, x + (HEADS + 1) * ROW, QKV * 2, s.stream)
        if kind != "append":
            B.oxy_mixed_attention(s.pool, batch, l, q.data_ptr(), s.out[l].data_ptr(),
                                  0 if s.lse is None else s.lse[l].data_ptr(), SCALE, s.stream)
    if kind == "append":
        _read_back(s, B.oxy_batch_slots(batch))
        return {"q": s.q_out, "kv": s.back}
    if kind == "step":
        B.oxy_batch_destroy(batch)
    return {"out": s.out} if s.lse is None else {"out": s.out, "lse": s.lse}


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ------------------------------------------------------------------------------------------
# what a pass cannot do without, and what it computes
# ------------------------------------------------------------------------------------------
def _visible(case):
    """Sum over queries of the tokens each one sees."""
    total = 0
    for p, h, n, both in _items(case):
        pre = case["prefix_len"] if p >= 0 else 0
        total += n * (pre + n) if both else n * (pre + h) + n * (n + 1) // 2
    return total


def work(case):
    """Inputs read once, rows stored and read in 8 bits once, outputs written once; 4 * 256 flops per
    (query row, visible key), 6 per rotated pair."""
    L, kind = case["layers"], case["kind"]
    if kind == "store":
        n = case["prefixes"] * case["prefix_len"] + sum(_histories(case))
        return {"bytes": 2 * L * n * (2 * ROW + 2 * ROW8), "flops": 0}
    if kind == "rotate":
        rows = case["prefix_len"] * (HEADS + 1)
        return {"bytes": rows * 2 * ROW + 4 * case["prefix_len"], "flops": rows * 3 * case["rot"]}
    items = _items(case)
    n = sum(it[2] for it in items)
    turned = n * ((HEADS + 2) * ROW + 2 * ROW8 + 4)       # projection's output in, new rows out
    if kind == "append":
        return {"bytes": L * (turned + n * (HEADS * ROW + 2 * ROW8 + 2 * ROW)),
                "flops": L * n * (HEADS + 1) * 3 * case["rot"]}
    live = n + sum(it[1] for it in items)
    live += len({it[0] for it in items if it[0] >= 0}) * case["prefix_len"]
    bytes_ = live * 2 * ROW8 + n * HEADS * ROW + (n * HEADS * 4 if case["lse"] else 0)
    bytes_ += turned - n * 2 * ROW8 if kind == "step" else n * HEADS * ROW
    return {"bytes": L * bytes_, "flops": L * _visible(case) * HEADS * 4 * DIM}


def _round_to(x, bits, lowest):
    """64-bit numbers to `bits` significant ones, half to even; below 2^lowest with a fixed step."""
    _, exponent = torch.frexp(x)
    step = torch.exp2((torch.clamp(exponent - 1, min=lowest) - (bits - 1)).double())
    return torch.round(x / step) * step


def _exact_cached(x):
    """The values that a cache holds for 64-bit rows (that are bf16 numbers)."""
    top = x.abs().amax(dim=-1, keepdim=True)
    _, e = torch.frexp(top / 448.0)                        # top <= 448 * 2^e, equal at a power of two
    e = torch.where(top == 448.0 * torch.exp2((e - 1).double()), e - 1, e)
    unit = torch.exp2(torch.clamp(e, min=-126).double())
    return _round_to(x / unit, 4, -6) * unit


def _exact_turned(case, x, positions):
    """Rows [n, heads, 256] turned, in 64 bits."""
    freqs, amplitude = _frequencies(case)
    angle = torch.tensor(positions, dtype=torch.float64, device="cuda").view(-1, 1, 1)
    angle = angle * torch.tensor(freqs, dtype=torch.float64, device="cuda")
    turn = amplitude * torch.polar(torch.ones_like(angle), angle)
    y = x.double().clone()
    r, half = case["rot"], case["rot"] // 2
    first = slice(0, half) if case["layout"] == "halves" else slice(0, r, 2)
    second = slice(half, r) if case["layout"] == "halves" else slice(1, r, 2)
    z = torch.complex(y[..., first], y[..., second]) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    """The definitions in 64 bits; what is handed on in bf16 (rotated queries and keys) is rounded to it."""
    L, kind = case["layers"], case["kind"]
    if kind == "store":
        return {"kv": torch.stack([_exact_cached(_stored_rows(case, seed, l).double()) for l in range(L)], 1)}
    positions = _positions(case)
    items = _items(case)
    n = case["prefix_len"] if kind == "rotate" else sum(it[2] for it in items)
    if kind == "rotate":
        x = _projected(seed, 0, n).view(n, HEADS + 2, DIM)
        return {"out": _exact_turned(case, x[:, :HEADS + 1], positions)}
    outs, lses, queries, rows = [], [], [], []
    for l in range(L):
        x = _projected(seed, l, n).view(n, HEADS + 2, DIM).double()
        if kind != "attend":
            x[:, :HEADS + 1] = _exact_turned(case, x[:, :HEADS + 1], positions)
            queries.append(x[:, :HEADS].clone())
            x = _round_to(x, 8, -126)
        new = _exact_cached(x[:, HEADS:].transpose(0, 1))
        rows.append(new)
        if kind == "append":
            continue
        held = _exact_cached(_stored_rows(case, seed, l).double())
        P, at = case["prefix_len"], case["prefixes"] * case["prefix_len"]
        o = torch.empty((n, HEADS, DIM), dtype=torch.float64, device="cuda")
        z = torch.empty((n, HEADS), dtype=torch.float64, device="cuda")
        t = 0
        for p, h, m, both in items:
            seen = [held[:, p * P:p * P + P]] if p >= 0 else []
            k, v = torch.cat(seen + [held[:, at:at + h], new[:, t:t + m]], dim=1)
            logits = (x[t:t + m, :HEADS].reshape(m * HEADS, DIM) @ k.t()).view(m, HEADS, -1) * SCALE
            if not both:
                last = k.shape[0] - m + torch.arange(m, device="cuda")
                later = torch.arange(k.shape[0], device="cuda") > last[:, None]
                logits = logits.masked_fill(later[:, None], -math.inf)
            z[t:t + m] = torch.logsumexp(logits, dim=2)
            o[t:t + m] = (torch.softmax(logits, dim=2).view(m * HEADS, -1) @ v).view(m, HEADS, DIM)
            at, t = at + h, t + m
        outs.append(o)
        lses.append(z)
    if kind == "append":
        return {"q": torch.stack(queries), "kv": torch.stack(rows, dim=1)}
    got = {"out": torch.stack(outs)}
    if case["lse"]:
        got["lse"] = torch.stack(lses)
    return got
