"""Workloads of an observation's prefill: rotary positions with several axes, attention over whole prompts, and
attention of a prefix's new tokens over the paged cache.

Geometry is the library's: 8 query heads over one KV head, head_dim 256, pages of 16 tokens, bf16 in and out; the
cache in bf16, or in 8 bits (a row as 256 e4m3 codes and the exponent e of a power-of-two scale, e = the smallest
integer >= -126 with max|x| <= 448 * 2^e).

Attention of an item with `past` tokens before it and n new ones, len = past + n in all: the query of new token i,
at position p = past + i, sees tokens j < min(len, max(p + 1, n_full)) -- n_full = 0: causal; len: all see all;
between: what the observation begins with (its images) sees itself whole, what follows is causal.  The output is
softmax(q k / 16) v over them, the log-sum-exp of the logits an output on request.

A rotation with several axes turns pair i of a row's first `rot` dims by positions[axis of pair i][token] *
frequency i.

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
MOST_LOGITS, MOST_ROWS, MOST_KEYS = 1.07e9, 30000, 262144   # of a drawn case: per layer, in all layers


def _case(name, kind, **kw):
    """kind: "prompt" = attention over `items` whole prompts (past 0) straight from the projection's output, one
    call a layer; "chunk" = attention of `items` prefixes' new tokens, whose rows are in the cache and whose
    descriptor is in hand, one call a layer; "rotate" = queries and keys of `new_hi` tokens rotated; "append" =
    queries rotated, keys rotated and stored, values stored, as a prefix's new tokens, per layer, and the rows read
    back; "prefill" = a whole prefill: prefixes made (or forked), descriptor, and per layer the rotating append and
    the attention, prefixes released.
    Item i has past_lo..past_hi tokens before it and new_lo..new_hi new ones; fork: all items go on behind the same
    past_hi tokens (a multiple of the page) of one observation.  see: "causal", "all", or "part" (n_full a part of
    the item).  bits: 16 or 8, the cache's form.
    rot dims are rotated, "halves" or "pairs", over n_axes axes, whose pairs lie in sections side by side or
    interleaved; first: position of token 0; images are grids of side x side tokens."""
    c = dict(kind=kind, layers=1, items=1, past_lo=0, past_hi=0, new_lo=1, new_hi=1, fork=False, see="causal",
             bits=16, lse=False, lengths=1, rot=DIM, layout="halves", n_axes=3, sections=True, first=0, side=16)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a short instruction alone, no cache: the smallest call
        _case("prompt_tiny", "prompt", new_lo=24, new_hi=24, lse=True),
        # one observation of three 16 x 16 views and 64 words, all see all
        _case("prompt_observation", "prompt", layers=6, new_lo=832, new_hi=832, see="all"),
        # observations and instructions of different lengths side by side, images whole and words causal
        _case("prompt_packed", "prompt", layers=2, items=7, new_lo=1, new_hi=1500, see="part", lse=True, lengths=3),
        # a long document, causal, ragged at its end
        _case("prompt_long", "prompt", new_lo=16391, new_hi=16391),
        # one word behind an observation, the form of single tokens
        _case("chunk_token", "chunk", layers=18, past_lo=832, past_hi=832),
        # four frames' new views behind the history that they share
        _case("chunk_frames", "chunk", layers=6, items=4, past_lo=576, past_hi=576, new_lo=256, new_hi=256, fork=True,
              see="all"),
        # eight robots' next words behind observations in 8 bits, ragged everywhere
        _case("chunk_words8", "chunk", layers=6, items=8, past_lo=700, past_hi=900, new_lo=20, new_hi=90, bits=8,
              lse=True, lengths=2),
        # the next 2048 tokens of a long document
        _case("chunk_long", "chunk", past_lo=32781, past_hi=32781, new_lo=2048, new_hi=2048),
        # a question of 48 words about a document of 131071 tokens in 8 bits
        _case("chunk_question8", "chunk", layers=2, past_lo=131071, past_hi=131071, new_lo=48, new_hi=48, bits=8,
              lse=True),
        # queries and keys of a long multimodal prompt, out of the projection's output
        _case("rotate_long", "rotate", new_lo=8192, new_hi=8192, first=1000),
        # an observation's rows on their way into all layers of a bf16 cache, axes interleaved
        _case("append_observation", "append", layers=18, new_lo=832, new_hi=832, sections=False, layout="pairs"),
        # a frame's prefill: two observations, rotated, stored in 8 bits and attended over, layer by layer
        _case("prefill_frame8", "prefill", layers=18, items=2, new_lo=832, new_hi=832, see="part", bits=8),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    """The same ranges: up to 16 items; prompts of 1..16391 tokens, 1..2048 new tokens behind 0..131072, both forms
    of the cache, every mask; 1..4 axes, either layout, 2..256 rotated dims."""
    kind = rng.choice(["prompt", "prompt", "chunk", "chunk", "chunk", "rotate", "append", "prefill"])
    c = dict(layers=_log_int(rng, 1, 18), items=_log_int(rng, 1, 16), see=rng.choice(["causal", "all", "part"]),
             lse=rng.random() < 0.4, lengths=rng.randint(100, 1 << 20), bits=rng.choice([8, 16]),
             rot=DIM if rng.random() < 0.4 else 2 * _log_int(rng, 1, 128), layout=rng.choice(["halves", "pairs"]),
             n_axes=rng.randint(1, 4), sections=rng.random() < 0.5, first=_log_int(rng, 1, 1 << 20),
             side=rng.randint(2, 24))
    if kind == "rotate":
        return _case(None, kind, **dict(c, new_hi=_log_int(rng, 1, 8192)))
    hi = _log_int(rng, 1, 16391 if kind == "prompt" else 2048)
    c.update(new_hi=hi, new_lo=hi if rng.random() < 0.3 else rng.randint(1, hi))
    if kind == "append":
        c.update(layers=rng.randint(1, 18), items=rng.randint(1, 4))
        c["layers"] = max(1, min(c["layers"], MOST_ROWS // (c["items"] * hi)))
        return _case(None, kind, **c)
    if kind != "prompt":
        past = _log_int(rng, 1, 131072 if kind == "chunk" and rng.random() < 0.3 else 2048)
        c["fork"] = rng.random() < 0.3
        if c["fork"]:
            past = max(1, past // PAGE) * PAGE
        if rng.random() < 0.25 or (kind == "prefill" and not c["fork"]):
            past, c["fork"] = 0, False
        c.update(past_hi=past, past_lo=past if c["fork"] else rng.randint(0, past))
    most = lambda: c["items"] * c["new_hi"] * HEADS * (c.get("past_hi", 0) + c["new_hi"])  # noqa: E731
    keys = lambda: c["items"] * (c.get("past_hi", 0) + c["new_hi"])                        # noqa: E731
    logits = MOST_LOGITS * (2 if c["see"] == "causal" and kind == "prompt" else 1)    # half of them are masked
    while c["items"] > 1 and (most() > logits or keys() > MOST_KEYS or c["items"] * c["new_hi"] > MOST_ROWS):
        c["items"] -= 1
    while most() > logits:
        c["new_hi"] = c["new_hi"] * 15 // 16
        c["new_lo"] = min(c["new_lo"], c["new_hi"])
    c["layers"] = max(1, min(c["layers"], int(logits / most()), MOST_KEYS // keys(),
                             MOST_ROWS // (c["items"] * c["new_hi"])))
    return _case(None, kind, **c)


def _items(case):
    """(past, new, n_full) of every item."""
    rng = random.Random(case["lengths"])
    items = []
    for _ in range(case["items"]):
        past = rng.randint(case["past_lo"], case["past_hi"])
        new = rng.randint(case["new_lo"], case["new_hi"])
        full = {"causal": 0, "all": past + new, "part": past + new * rng.randint(1, 15) // 16}[case["see"]]
        items.append((past, new, full))
    return items


def _n_new(case):
    return case["new_hi"] if case["kind"] == "rotate" else sum(n for _, n, _ in _items(case))


def _n_past(case):
    return case["past_hi"] if case["fork"] else sum(p for p, _, _ in _items(case))


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
    x *= torch.exp2(0.7 * torch.randn(x.shape[:-1], device="cuda", generator=g))[..., None]
    x[0] *= gain
    return x.to(torch.bfloat16)


def _past_rows(case, seed, layer):
    """Keys and values that the cache of a layer holds before the pass, item by item: [2, n_past, 256] bf16."""
    g = _generator(seed, 1, layer)
    return _shape_rows(torch.randn((2, _n_past(case), DIM), device="cuda", generator=g), g)


def _projected(seed, layer, n):
    """Queries, key and value of n new tokens side by side, as a projection writes them: [n, 10 * 256]."""
    g = _generator(seed, 2, layer)
    q = torch.randn((n, HEADS * DIM), device="cuda", generator=g)
    kv = _shape_rows(torch.randn((2, n, DIM), device="cuda", generator=g), g)
    return torch.cat([q.to(torch.bfloat16), kv[0], kv[1]], dim=1)


def _grid_positions(case, first, n):
    """Positions of n tokens on every axis: three quarters of them images (view, row, column), then words, whose
    axes agree."""
    side = case["side"]
    views = n * 3 // 4 // (side * side)
    rows = []
    for t in range(n):
        v, at = divmod(t, side * side)
        if v < views:
            rows.append((first + v, first + at // side, first + at % side, first + at % 7))
        else:
            rows.append((first + max(views, side) + t - views * side * side,) * 4)
    return rows


def _positions(case):
    """[n_axes][tokens]"""
    if case["kind"] == "rotate":
        rows = _grid_positions(case, case["first"], case["new_hi"])
    else:
        rows = [r for past, n, _ in _items(case) for r in _grid_positions(case, case["first"] + past, n)]
    return [[r[a] for r in rows] for a in range(case["n_axes"])]


def _axis_of_pair(case):
    """The first axis has a quarter of the pairs, the others share the rest; or axes take turns."""
    pairs, n = case["rot"] // 2, case["n_axes"]
    if n == 1:
        return [0] * pairs
    if not case["sections"]:
        return [i % n for i in range(pairs)]
    lead = pairs // 4
    return [0 if i < lead else 1 + (i - lead) * (n - 1) // (pairs - lead) for i in range(pairs)]


BASE = 10000.0


def _frequencies(case):
    return BASE ** (-2.0 * np.arange(case["rot"] // 2, dtype=np.float64) / case["rot"])


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


def _rotate(s, x):
    """Rows [n, heads, 256] bf16 turned by their tokens' positions, each pair on its axis; angles in 64 bits."""
    rot = s.case["rot"]
    angle = s.positions[s.axis_of_pair].double().t() * s.freqs
    c, t = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    y = x.float()
    if s.case["layout"] == "halves":
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        turned = torch.cat([a * c - b * t, b * c + a * t], dim=-1)
    else:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack([a * c - b * t, b * c + a * t], dim=-1).flatten(-2)
    return torch.cat([turned, y[..., rot:]], dim=-1).to(torch.bfloat16)


def _attention(s, q, keys, values):
    """Items side by side, padded to the longest: q [tokens, 8, 256]; keys and values [rows, 256] in 32 bits."""
    n_items, most = s.token_of.shape
    k, v = keys[s.row_of], values[s.row_of]                              # [items, keys, 256]
    rows = q.float()[s.token_of].reshape(n_items, most * HEADS, DIM)
    logits = (rows @ k.transpose(1, 2).contiguous()).view(n_items, most, HEADS, -1)
    logits *= SCALE
    logits.masked_fill_(s.hidden[:, :, None, :], -math.inf)
    top = logits.amax(dim=-1, keepdim=True)
    p = logits.sub_(top).exp_()
    total = p.sum(dim=-1, keepdim=True)
    o = (p.view(n_items, most * HEADS, -1) @ v).view(n_items, most, HEADS, DIM) / total
    lse = (top + torch.log(total))[..., 0]
    return o[s.real].to(torch.bfloat16), lse[s.real]


class _State:
    """A cache with what is stored in it, and the resident inputs of a pass."""

    def __del__(self):
        if getattr(self, "pool", None) is not None:
            torch.cuda.synchronize()
            if self.batch is not None:
                self.B.oxy_batch_destroy(self.batch)
            self.B.oxy_pool_destroy(self.pool)
            self.pool = None


def _prepare_plain(s, case, seed):
    """Cached rows (past, then new ones), and for every item the rows that its keys lie in."""
    s.freqs = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
    s.axis_of_pair = torch.tensor(_axis_of_pair(case), device="cuda")
    if case["kind"] in ("rotate", "append"):
        return
    items, new0 = s.items, _n_past(case)
    if case["kind"] != "prompt":
        stored = [torch.cat([_past_rows(case, seed, l), s.new_rows(l)], dim=1) for l in range(case["layers"])]
        if case["bits"] == 8:
            coded = [_quantise(x) for x in stored]
            s.codes, s.exponents = (torch.stack([x[i] for x in coded]) for i in range(2))
        else:
            s.rows = torch.stack(stored)                                 # [L, 2, rows, 256]
    most_new, most = max(n for _, n, _ in items), max(p + n for p, n, _ in items)
    row_of, token_of = np.zeros((len(items), most), np.int64), np.zeros((len(items), most_new), np.int64)
    last = np.zeros((len(items), most_new), np.int64)
    at, t = 0, 0
    for i, (past, n, full) in enumerate(items):
        row_of[i, :past + n] = np.r_[at:at + past, new0 + t:new0 + t + n]
        new = np.minimum(np.arange(most_new), n - 1)
        token_of[i] = t + new
        last[i] = np.minimum(past + n, np.maximum(past + new + 1, full)) - 1
        at, t = at + (0 if case["fork"] else past), t + n
    s.row_of, s.token_of = torch.tensor(row_of, device="cuda"), torch.tensor(token_of, device="cuda")
    s.hidden = torch.arange(most, device="cuda") > torch.tensor(last, device="cuda")[..., None]
    s.real = torch.tensor([[i < n for i in range(most_new)] for _, n, _ in items], device="cuda")


def _prepare_own(s, case, seed):
    """A pool, with the past tokens stored as prefixes where there are any, and outputs allocated."""
    from paper_2603_14371_amd import binding as B
    s.B, s.pool, s.batch, s.pids = B, None, None, []
    s.stream = torch.cuda.current_stream().cuda_stream
    L, n, kind, items = case["layers"], s.n, case["kind"], s.items
    s.freqs = torch.tensor(B.oxy_rotary_freqs(BASE, case["rot"])[0], dtype=torch.float64, device="cuda")
    s.rotary = B.make_rotary(s.freqs.data_ptr(), case["rot"],
                             {"halves": B.ROTARY_HALVES, "pairs": B.ROTARY_PAIRS}[case["layout"]])
    s.axes = B.make_rotary_axes(_axis_of_pair(case), case["n_axes"])
    if kind == "rotate":
        s.out = torch.empty((n, HEADS + 1, DIM), dtype=torch.bfloat16, device="cuda")
        return
    s.out = torch.empty((L, n, HEADS, DIM), dtype=torch.bfloat16, device="cuda")
    s.lse = torch.empty((L, n, HEADS), device="cuda") if case["lse"] else None
    pages = lambda m: -(-m // PAGE)  # noqa: E731
    blocks = 16 + pages(case["past_hi"]) + sum(pages(p + m) for p, m, _ in items)
    if kind == "prompt":
        blocks = 1
    order = list(range(blocks))
    random.Random(seed).shuffle(order)
    cfg = B.make_config(1 if kind == "prompt" else L, blocks, free_order=order, max_q_tokens=max(16, n),
                        max_append_tokens=max(16, n), flags=B.POOL_KV_FP8 if case["bits"] == 8 else 0,
                        max_partials=max(32 * n, 2048) if n < 4096 else 4 * n + 16384)
    s.kv = torch.empty(B.oxy_kv_bytes(cfg), dtype=torch.uint8, device="cuda")
    s.ws = torch.empty(B.oxy_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    cfg.kv_base, cfg.kv_bytes = s.kv.data_ptr(), s.kv.numel()
    cfg.workspace, cfg.workspace_bytes = s.ws.data_ptr(), s.ws.numel()
    s.pool = B.oxy_pool_create(cfg)
    if kind == "prompt":
        s.batch = B.oxy_prompt_batch_build(s.pool, [(m, full) for _, m, full in items], s.stream)
        return
    s.q_out = torch.empty((L, n, HEADS, DIM), dtype=torch.bfloat16, device="cuda")
    s.back = torch.empty((2, L, n, DIM), dtype=torch.bfloat16, device="cuda")
    if kind == "append":
        return
    pasts = [items[0][0]] if case["fork"] else [p for p, _, _ in items]
    s.pids = [B.oxy_prefix_create(s.pool) for _ in pasts]
    for l in range(L):
        kv, at = _past_rows(case, seed, l), 0
        for pid, past in zip(s.pids, pasts):
            if past:
                B.oxy_prefix_append(s.pool, pid, l, kv[0, at:].data_ptr(), kv[1, at:].data_ptr(), past, 0, s.stream)
            at += past
        torch.cuda.synchronize()
    if kind == "chunk":
        pids = [B.oxy_prefix_fork(s.pool, s.pids[0], pasts[0]) for _ in items] if case["fork"] else s.pids
        s.batch = B.oxy_prefix_batch_build(s.pool, [(pid, m, full) for pid, (_, m, full) in zip(pids, items)], 0,
                                           s.stream)
        for l in range(L):
            kv = s.new_rows(l).contiguous()
            B.oxy_stream_append(s.pool, s.batch, l, kv[0].data_ptr(), kv[1].data_ptr(), s.stream)
            torch.cuda.synchronize()


def prepare(case, seed):
    s = _State()
    s.case, s.items = case, _items(case)
    L = 1 if case["kind"] == "rotate" else case["layers"]
    s.n = _n_new(case)
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
    if kind == "rotate":
        return {"out": _rotate(s, s.qkv[0, :, :(HEADS + 1) * DIM].unflatten(1, (HEADS + 1, DIM)))}
    outs, lses, queries, rows = [], [], [], []
    for l in range(case["layers"]):
        x, q = s.qkv[l].unflatten(1, (HEADS + 2, DIM)), s.q[l]
        if kind == "prompt":
            o, lse = _attention(s, x[:, :HEADS], x[:, HEADS].float(), x[:, HEADS + 1].float())
        else:
            if kind != "chunk":
                turned = _rotate(s, x[:, :HEADS + 1])
                q, new = turned[:, :HEADS], torch.stack([turned[:, HEADS], x[:, HEADS + 1]])
            if kind == "append":
                queries.append(q)
                rows.append(_values(*_quantise(new)).to(torch.bfloat16) if case["bits"] == 8 else new)
                continue
            if case["bits"] == 8:
                if kind == "prefill":
                    s.codes[l, :, -s.n:], s.exponents[l, :, -s.n:] = _quantise(new)
                kv = _values(s.codes[l], s.exponents[l])
            else:
                if kind == "prefill":
                    s.rows[l, :, -s.n:] = new
                kv = s.rows[l].float()
            o, lse = _attention(s, q, kv[0], kv[1])
        outs.append(o)
        lses.append(lse)
    if kind == "append":
        return {"q": torch.stack(queries), "kv": torch.stack(rows, dim=1)}
    return {"out": torch.stack(outs), "lse": torch.stack(lses)} if case["lse"] else {"out": torch.stack(outs)}


def _append(s, batch, l):
    x = s.qkv[l].data_ptr()
    s.B.oxy_rotary_axes_append(s.pool, batch, l, s.rotary, s.axes, s.positions.data_ptr(), x, QKV * 2,
                               s.q_out[l].data_ptr(), x + HEADS * ROW, QKV * 2, x + (HEADS + 1) * ROW, QKV * 2,
                               s.stream)


def _run_own(s):
    B, case, kind, n = s.B, s.case, s.case["kind"], s.n
    if kind == "rotate":
        B.oxy_rotary_axes(s.rotary, s.axes, s.positions.data_ptr(), s.qkv.data_ptr(), QKV * 2, s.out.data_ptr(),
                          (HEADS + 1) * ROW, n, HEADS + 1, s.stream)
        return {"out": s.out}
    lse_of = lambda l: 0 if s.lse is None else s.lse[l].data_ptr()  # noqa: E731
    if kind == "prompt":
        for l in range(case["layers"]):
            x = s.qkv[l].data_ptr()
            B.oxy_prompt_attention(s.pool, s.batch, x, QKV * 2, x + HEADS * ROW, QKV * 2, x + (HEADS + 1) * ROW,
                                   QKV * 2, s.out[l].data_ptr(), HEADS * ROW, lse_of(l), SCALE, s.stream)
    elif kind == "chunk":
        for l in range(case["layers"]):
            B.oxy_prefix_attention(s.pool, s.batch, l, s.q[l].data_ptr(), HEADS * ROW, s.out[l].data_ptr(),
                                   HEADS * ROW, lse_of(l), SCALE, s.stream)
    else:
        pids = [B.oxy_prefix_fork(s.pool, s.pids[0], s.items[0][0]) if case["fork"] else B.oxy_prefix_create(s.pool)
                for _ in s.items]
        batch = B.oxy_prefix_batch_build(s.pool, [(pid, m, full) for pid, (_, m, full) in zip(pids, s.items)],
                                         B.BATCH_APPEND_ONLY if kind == "append" else 0, s.stream)
        for l in range(case["layers"]):
            _append(s, batch, l)
            if kind == "prefill":
                B.oxy_prefix_attention(s.pool, batch, l, s.q_out[l].data_ptr(), HEADS * ROW, s.out[l].data_ptr(),
                                       HEADS * ROW, lse_of(l), SCALE, s.stream)
        if kind == "append":
            B.oxy_gather_kv_layers(s.pool, 0, case["layers"], B.oxy_batch_slots(batch), s.back[0].data_ptr(),
                                   s.back[1].data_ptr(), n * ROW, s.stream)
        B.oxy_batch_destroy(batch)
        for pid in pids:
            B.oxy_prefix_release(s.pool, pid)
        if kind == "append":
            return {"q": s.q_out, "kv": s.back}
    return {"out": s.out} if s.lse is None else {"out": s.out, "lse": s.lse}


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ------------------------------------------------------------------------------------------
# what a pass cannot do without, and what it computes
# ------------------------------------------------------------------------------------------
def _visible(case):
    """Sum over queries of the tokens that each one sees."""
    total = 0
    for past, n, full in _items(case):
        p = np.arange(past, past + n)
        total += int(np.minimum(past + n, np.maximum(p + 1, full)).sum())
    return total


def work(case):
    """Inputs read once, cached rows once in the cache's form, outputs written once; 4 * 256 flops per (query row,
    visible key), 6 per rotated pair."""
    L, kind, n = case["layers"], case["kind"], _n_new(case)
    held = ROW8 if case["bits"] == 8 else ROW
    turn_flops = n * (HEADS + 1) * 3 * case["rot"]
    if kind == "rotate":
        return {"bytes": n * (HEADS + 1) * 2 * ROW + 4 * case["n_axes"] * n, "flops": turn_flops}
    turned = n * ((HEADS + 2) * ROW + 4 * case["n_axes"])    # the projection's output and positions in
    if kind == "append":
        return {"bytes": L * (turned + n * (HEADS * ROW + 2 * held + 2 * ROW)), "flops": L * turn_flops}
    flops = _visible(case) * HEADS * 4 * DIM
    out = n * HEADS * ROW + (n * HEADS * 4 if case["lse"] else 0)
    if kind == "prompt":
        return {"bytes": L * (n * (HEADS + 2) * ROW + out), "flops": L * flops}
    live = (_n_past(case) + n) * 2 * held
    if kind == "chunk":
        return {"bytes": L * (live + n * HEADS * ROW + out), "flops": L * flops}
    return {"bytes": L * (turned + live + out), "flops": L * (flops + turn_flops)}


def _round_to(x, bits, lowest):
    """64-bit numbers to `bits` significant ones, half to even; below 2^lowest with a fixed step."""
    _, exponent = torch.frexp(x)
    step = torch.exp2((torch.clamp(exponent - 1, min=lowest) - (bits - 1)).double())
    return torch.round(x / step) * step


def _exact_cached(case, x):
    """The values that a cache holds for 64-bit rows (that are bf16 numbers)."""
    if case["bits"] == 16:
        return x
    top = x.abs().amax(dim=-1, keepdim=True)
    _, e = torch.frexp(top / 448.0)                        # top <= 448 * 2^e, equal at a power of two
    e = torch.where(top == 448.0 * torch.exp2((e - 1).double()), e - 1, e)
    unit = torch.exp2(torch.clamp(e, min=-126).double())
    return _round_to(x / unit, 4, -6) * unit


def _exact_turned(case, x):
    """Rows [n, heads, 256] turned, in 64 bits."""
    axis = torch.tensor(_axis_of_pair(case), device="cuda")
    at = torch.tensor(_positions(case), dtype=torch.float64, device="cuda")
    angle = (at.t()[:, axis] * torch.tensor(_frequencies(case), device="cuda"))[:, None]
    turn = torch.polar(torch.ones_like(angle), angle)
    y = x.double().clone()
    r, half = case["rot"], case["rot"] // 2
    first = slice(0, half) if case["layout"] == "halves" else slice(0, r, 2)
    second = slice(half, r) if case["layout"] == "halves" else slice(1, r, 2)
    z = torch.complex(y[..., first], y[..., second]) * turn
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    """The definitions in 64 bits; what is handed on in bf16 (rotated queries and keys) is rounded to it."""
    L, kind, n = case["layers"], case["kind"], _n_new(case)
    if kind == "rotate":
        return {"out": _exact_turned(case, _projected(seed, 0, n).view(n, HEADS + 2, DIM)[:, :HEADS + 1])}
    if _visible(case) * L > 2.5e8:
        return None
    outs, lses, queries, rows = [], [], [], []
    for l in range(L):
        x = _projected(seed, l, n).view(n, HEADS + 2, DIM).double()
        if kind in ("append", "prefill"):
            x[:, :HEADS + 1] = _exact_turned(case, x[:, :HEADS + 1])
            queries.append(x[:, :HEADS].clone())
            x = _round_to(x, 8, -126)
        new = x[:, HEADS:].transpose(0, 1)
        if kind != "prompt":
            new = _exact_cached(case, new)
        if kind == "append":
            rows.append(new)
            continue
        held = None if kind == "prompt" else _exact_cached(case, _past_rows(case, seed, l).double())
        o = torch.empty((n, HEADS, DIM), dtype=torch.float64, device="cuda")
        z = torch.empty((n, HEADS), dtype=torch.float64, device="cuda")
        at, t = 0, 0
        for past, m, full in _items(case):
            k, v = new[:, t:t + m] if held is None else torch.cat([held[:, at:at + past], new[:, t:t + m]], dim=1)
            for a in range(0, m, 2048):
                b = min(m, a + 2048)
                p = past + torch.arange(a, b, device="cuda")
                later = torch.arange(past + m, device="cuda") >= torch.clamp(p + 1, min=full)[:, None]
                for h in range(HEADS):
                    logits = (x[t + a:t + b, h] @ k.t() * SCALE).masked_fill(later, -math.inf)
                    z[t + a:t + b, h] = torch.logsumexp(logits, dim=1)
                    o[t + a:t + b, h] = torch.softmax(logits, dim=1) @ v
            at, t = at + (0 if case["fork"] else past), t + m
        outs.append(o)
        lses.append(z)
    if kind == "append":
        return {"q": torch.stack(queries), "kv": torch.stack(rows, dim=1)}
    return {"out": torch.stack(outs), "lse": torch.stack(lses)} if case["lse"] else {"out": torch.stack(outs)}
