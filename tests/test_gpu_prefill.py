"""Attention of a prefix's new tokens over the paged cache and over whole prompts, element by element against the float64
oracle."""
import numpy as np
import pytest

from prefill_util import Pool, bits, check, down, held, up

pytestmark = pytest.mark.gpu
SCALE = 1.0 / 16


def chunk(items, kv8=False, scale=SCALE, fork=False, lse=True, q_pad=0, out_pad=0, seed=0, sigma=1.0, parts=None,
          change=None, small=False):
    """items: (past, n_new, n_full).  One batch of them on a pool whose pages lie in random order; every row checked."""
    import torch
    rng = np.random.default_rng(seed)
    n = sum(it[1] for it in items)
    blocks = sum((p + m + 15) // 16 for p, m, _ in items) + 8
    kw = {} if parts is None else {"max_partials": parts}
    pool = Pool(2, blocks, kv8, seed, small, max_q_tokens=max(16, n), max_append_tokens=max(16, n), **kw)
    B = pool.B
    try:
        if fork:
            past = items[0][0]
            k0, v0 = bits(rng, past, 256, scale=sigma), bits(rng, past, 256)
            parent = pool.prefix(k0, v0, 1)
            pids, old = [B.oxy_prefix_fork(pool.p, parent, past) for _ in items], [(k0, v0)] * len(items)
        else:
            old = [(bits(rng, p, 256, scale=sigma), bits(rng, p, 256)) for p, _, _ in items]
            pids = [pool.prefix(k, v, 1) for k, v in old]
        q, k, v = bits(rng, n, 8, 256), bits(rng, n, 256, scale=sigma), bits(rng, n, 256)
        if change:
            change(q, k, v, old)
        batch = B.oxy_prefix_batch_build(pool.p, [(pid, m, f) for pid, (_, m, f) in zip(pids, items)], 0, pool.stream)
        dk, dv = up(k), up(v)
        B.oxy_stream_append(pool.p, batch, 1, dk.data_ptr(), dv.data_ptr(), pool.stream)
        dq = torch.zeros((n, 2048 + q_pad), dtype=torch.int16, device="cuda")
        dq[:, :2048] = up(q).view(n, 2048)
        out = torch.full((n + 1, 2048 + out_pad), 77, dtype=torch.int16, device="cuda")
        z = torch.full((n + 1, 8), 3.0, device="cuda")
        B.oxy_prefix_attention(pool.p, batch, 1, dq.data_ptr(), dq.stride(0) * 2, out.data_ptr(), out.stride(0) * 2,
                               z.data_ptr() if lse else 0, scale, pool.stream)
        got = down(out)
        assert np.all(got[:, 2048:] == 77) and np.all(got[n] == 77) and bool((z[n] == 3).all())
        z = z[:n].cpu().numpy().astype(np.float64) if lse else None
        info = B.oxy_batch_info(batch)
        assert info[:2] == (len(items), n)
        t = 0
        for i, (past, m, full) in enumerate(items):
            kk = held(np.concatenate([old[i][0], k[t:t + m]]), kv8)
            vv = held(np.concatenate([old[i][1], v[t:t + m]]), kv8)
            check(got[t:t + m, :2048].reshape(m, 8, 256), None if z is None else z[t:t + m], q[t:t + m], kk, vv, past, full,
                  scale, "item %d %s" % (i, (past, m, full)))
            t += m
        B.oxy_batch_destroy(batch)
        return info
    finally:
        pool.close()


def prompts(items, scale=SCALE, lse=True, pad=(0, 0, 0, 0), seed=0, sigma=1.0, parts=None, in8=False):
    """items: (tokens, n_full)."""
    import torch
    rng = np.random.default_rng(seed)
    n = sum(it[0] for it in items)
    kw = {} if parts is None else {"max_partials": parts}
    pool = Pool(1, 1, in8, max_q_tokens=max(16, n), **kw)
    B = pool.B
    try:
        q, k, v = bits(rng, n, 8, 256), bits(rng, n, 256, scale=sigma), bits(rng, n, 256)
        batch = B.oxy_prompt_batch_build(pool.p, items, pool.stream)
        dev = []
        for x, more in zip((q.reshape(n, 2048), k, v), pad):
            d = torch.full((n + 1, x.shape[1] + more), -1, dtype=torch.int16, device="cuda")    # NaN between and behind rows
            d[:n, :x.shape[1]] = up(x)
            dev.append(d)
        out = torch.full((n + 1, 2048 + pad[3]), 77, dtype=torch.int16, device="cuda")
        z = torch.full((n + 1, 8), 3.0, device="cuda")
        args = [a for d in dev for a in (d.data_ptr(), d.stride(0) * 2)]
        B.oxy_prompt_attention(pool.p, batch, *args, out.data_ptr(), out.stride(0) * 2, z.data_ptr() if lse else 0, scale,
                               pool.stream)
        got = down(out)
        assert np.all(got[:, 2048:] == 77) and np.all(got[n] == 77) and bool((z[n] == 3).all())
        z = z[:n].cpu().numpy().astype(np.float64) if lse else None
        info = B.oxy_batch_info(batch)
        t = 0
        for i, (m, full) in enumerate(items):
            check(got[t:t + m, :2048].reshape(m, 8, 256), None if z is None else z[t:t + m], q[t:t + m], held(k[t:t + m], False),
                  held(v[t:t + m], False), 0, full, scale, "prompt %d %s" % (i, (m, full)))
            t += m
        B.oxy_batch_destroy(batch)
        return info
    finally:
        pool.close()


FORMS = pytest.mark.parametrize("kv8", [False, True], ids=["bf16", "fp8"])


@FORMS
@pytest.mark.parametrize("past,n", [(0, 1), (1, 1), (15, 1), (16, 1), (31, 2), (32, 3), (0, 15), (0, 16), (0, 17), (5, 31), (17, 32),
                                    (33, 33), (100, 4), (100, 5), (0, 63), (0, 64), (1, 65), (63, 64), (250, 129)])
def test_small_items(past, n, kv8):
    for full in (0, past + n, past + n // 2):
        chunk([(past, n, full)], kv8, seed=past * 1000 + n)


@FORMS
@pytest.mark.parametrize("past,n", [(832, 1), (3000, 2), (1999, 7), (2048, 16), (4100, 20), (900, 100), (0, 700)])
def test_histories_cut_into_parts(past, n, kv8):
    info = chunk([(past, n, past + n)], kv8, seed=n)
    assert info[3] > 0
    chunk([(past, n, 0)], kv8, seed=n + 1, lse=False)


@FORMS
def test_ragged_items_side_by_side(kv8):
    items = [(0, 5, 3), (700, 1, 0), (31, 47, 60), (16, 16, 0), (1, 90, 1000), (333, 33, 400), (0, 1, 1), (64, 130, 100)]
    chunk(items, kv8, seed=3)
    chunk(items[::-1], kv8, seed=4, q_pad=512, out_pad=8)


@FORMS
def test_forks_share_their_history(kv8):
    chunk([(160, 40, 500), (160, 1, 0), (160, 77, 170)], kv8, fork=True, seed=5)


@FORMS
@pytest.mark.parametrize("scale", [1.0, -0.25, 0.0, 1e-3, 3.0])
def test_scales(scale, kv8):
    chunk([(40, 21, 50)], kv8, scale=scale, seed=6)


@FORMS
def test_room_for_split_results(kv8):
    """A prefill has room for 8192 split results however few a step of streams may have."""
    items = [(1500, 40, 0), (20, 30, 50)]
    n = [chunk(items, kv8, seed=7, parts=p)[3] for p in (1, 100000)]
    assert 0 < n[0] == n[1] <= 8192


@FORMS
@pytest.mark.parametrize("parts", [1, 7, 200])
def test_a_workspace_of_few_split_results(parts, kv8):
    info = chunk([(1500, 40, 0), (20, 30, 50), (900, 3, 0)], kv8, seed=7, parts=parts, small=True)
    assert info[3] <= parts


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 33, 64, 65, 130, 300])
def test_small_prompts(n):
    for full in (0, n, n // 2, 1):
        prompts([(n, full)], seed=n)


def test_prompts_side_by_side():
    items = [(5, 0), (0, 0), (130, 64), (1, 1), (77, 1000), (0, 3), (300, 200), (16, 16), (700, 0)]
    prompts(items, seed=1)
    prompts(items, seed=2, pad=(512, 2304, 8, 16), lse=False)
    prompts(items, seed=2, parts=1, in8=True)


def test_long_prompt():
    info = prompts([(1500, 700)], seed=9)
    assert info[3] > 0


def test_large_logits():
    """Maxima that move by far more than the threshold below which a reference is kept."""
    chunk([(300, 40, 0)], False, seed=11, sigma=8.0)
    chunk([(300, 40, 0)], True, seed=11, sigma=8.0)
    prompts([(200, 0)], seed=12, sigma=8.0)


def test_no_tokens():
    pool = Pool(1, 1)
    B = pool.B
    try:
        for items in ([(0, 0)], [(0, 5), (0, 0)]):
            batch = B.oxy_prompt_batch_build(pool.p, items, pool.stream)
            B.oxy_prompt_attention(pool.p, batch, 0, 0, 0, 0, 0, 0, 0, 0, 0, 1.0, pool.stream)
            B.oxy_batch_destroy(batch)
    finally:
        pool.close()


@FORMS
def test_few_long_items_among_others(kv8):
    """Tokens of more and of fewer split results than a wavefront joins at once, in one launch."""
    chunk([(200, 17, 0), (3000, 3, 0), (0, 1, 0), (330, 20, 400), (2500, 18, 0), (5, 2, 9)], kv8, seed=41)


@FORMS
def test_blocks_behind_four_gibibytes(kv8):
    """The prefix lies in blocks whose bytes in the layer begin behind 2^32."""
    import torch
    size = 8192 if kv8 else 16384
    blocks = 2 ** 32 // size + 200
    rng = np.random.default_rng(5)
    past, n = 700, 20
    from paper_2603_14371_amd import binding as B
    order = np.concatenate([np.arange(blocks - 150), blocks - 150 + rng.permutation(150)])
    at = {}
    for name in (order, order[::-1]):       # whichever end blocks are taken from
        cfg = B.make_config(1, blocks, free_order=name, flags=(B.POOL_KV_FP8 if kv8 else 0) | B.POOL_HOST_ONLY)
        p = B.oxy_pool_create(cfg)
        pid = B.oxy_prefix_create(p)
        B.oxy_prefix_append(p, pid, 0, 0, 0, past + n, 0, 0)
        at[min(B.oxy_prefix_blocks(p, pid))] = name
        B.oxy_prefix_release(p, pid)
        B.oxy_pool_destroy(p)
    assert max(at) * size >= 2 ** 32
    cfg = B.make_config(1, blocks, free_order=at[max(at)], flags=B.POOL_KV_FP8 if kv8 else 0)
    kv = torch.empty(B.oxy_kv_bytes(cfg), dtype=torch.uint8, device="cuda")
    ws = torch.empty(B.oxy_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
    cfg.kv_base, cfg.kv_bytes, cfg.workspace, cfg.workspace_bytes = kv.data_ptr(), kv.numel(), ws.data_ptr(), ws.numel()
    pool = B.oxy_pool_create(cfg)
    stream = torch.cuda.current_stream().cuda_stream
    k, v, q = bits(rng, past + n, 256), bits(rng, past + n, 256), bits(rng, n, 8, 256)
    dk, dv, dq = up(k), up(v), up(q)
    pid = B.oxy_prefix_create(pool)
    B.oxy_prefix_append(pool, pid, 0, dk.data_ptr(), dv.data_ptr(), past, 0, stream)
    batch = B.oxy_prefix_batch_build(pool, [(pid, n, 0)], 0, stream)
    assert min(B.oxy_prefix_blocks(pool, pid)) * size >= 2 ** 32
    B.oxy_stream_append(pool, batch, 0, dk.data_ptr() + past * 512, dv.data_ptr() + past * 512, stream)
    out, z = torch.zeros((n, 8, 256), dtype=torch.int16, device="cuda"), torch.zeros((n, 8), device="cuda")
    B.oxy_prefix_attention(pool, batch, 0, dq.data_ptr(), 4096, out.data_ptr(), 4096, z.data_ptr(), SCALE, stream)
    check(down(out), z.cpu().numpy().astype(np.float64), q, held(k, kv8), held(v, kv8), past, 0, SCALE)
    B.oxy_batch_destroy(batch)
    B.oxy_pool_destroy(pool)


def test_rows_as_far_apart_as_may_be():
    """Keys 256 MiB less 16 bytes apart, values a little less; from there on the call is refused."""
    import torch
    rng = np.random.default_rng(6)
    n, far, less = 17, 2 ** 28 - 16, 2 ** 28 - 4096
    pool = Pool(1, 1, max_q_tokens=32)
    B = pool.B
    q, k, v = bits(rng, n, 8, 256), bits(rng, n, 256), bits(rng, n, 256)
    dq, out = up(q), torch.zeros((n, 8, 256), dtype=torch.int16, device="cuda")
    big = torch.empty((n * far + 1024) // 2, dtype=torch.int16, device="cuda")
    for t in range(n):
        big[t * far // 2:t * far // 2 + 256] = up(k[t])
        big[t * less // 2 + 512:t * less // 2 + 768] = up(v[t])
    batch = B.oxy_prompt_batch_build(pool.p, [(n, 0)], pool.stream)
    a = big.data_ptr()
    args = lambda ks, vs: (pool.p, batch, dq.data_ptr(), 4096, a, ks, a + 1024, vs, out.data_ptr(), 4096, 0, SCALE,  # noqa: E731
                           pool.stream)
    B.oxy_prompt_attention(*args(far, less))
    check(down(out), None, q, held(k, False), held(v, False), 0, 0, SCALE)
    for ks, vs in ((far + 16, less), (less, far + 16), (far + 8, less), (496, less), (less, 0)):
        with pytest.raises(B.OxyError) as e:
            B.oxy_prompt_attention(*args(ks, vs))
        assert e.value.code == B.ERR_INVALID_ARG
    B.oxy_batch_destroy(batch)
    pool.close()
