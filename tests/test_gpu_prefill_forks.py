"""Attention of forks' new tokens on pools without a block to spare, where tables that list shared blocks once find them."""
import numpy as np
import pytest

from prefill_util import Pool, bits, check, down, held, up

pytestmark = pytest.mark.gpu
SCALE = 1.0 / 16
FORMS = pytest.mark.parametrize("kv8", [False, True], ids=["bf16", "fp8"])


def forks(kv8, past, own, n, seed):
    """Prefixes behind the same `past` tokens, own[i] more and then n[i] new ones; every row checked."""
    import torch
    rng = np.random.default_rng(seed)
    blocks = past // 16 + sum(-(-(a + b) // 16) for a, b in zip(own, n))
    total = sum(n)
    pool = Pool(1, blocks, kv8, seed, max_q_tokens=total, max_append_tokens=max(16, total))
    B = pool.B
    try:
        k0, v0 = bits(rng, past, 256), bits(rng, past, 256)
        parent = pool.prefix(k0, v0)
        pids, keys, values = [], [], []
        for more in own:
            pids.append(B.oxy_prefix_fork(pool.p, parent, past))
            k, v = bits(rng, more, 256), bits(rng, more, 256)
            if more:
                dk, dv = up(k), up(v)
                B.oxy_prefix_append(pool.p, pids[-1], 0, dk.data_ptr(), dv.data_ptr(), more, past, pool.stream)
                down(dk)
            keys.append(np.concatenate([k0, k]))
            values.append(np.concatenate([v0, v]))
        q, k, v = bits(rng, total, 8, 256), bits(rng, total, 256), bits(rng, total, 256)
        full = [int(rng.integers(0, past + 2 * m)) for m in n]
        batch = B.oxy_prefix_batch_build(pool.p, list(zip(pids, n, full)), 0, pool.stream)
        assert B.oxy_free_blocks(pool.p) == []
        dq, dk, dv = up(q), up(k), up(v)
        out, z = torch.zeros((total, 8, 256), dtype=torch.int16, device="cuda"), torch.zeros((total, 8), device="cuda")
        B.oxy_stream_append(pool.p, batch, 0, dk.data_ptr(), dv.data_ptr(), pool.stream)
        B.oxy_prefix_attention(pool.p, batch, 0, dq.data_ptr(), 4096, out.data_ptr(), 4096, z.data_ptr(), SCALE, pool.stream)
        got, z, t = down(out), z.cpu().numpy().astype(np.float64), 0
        for i, m in enumerate(n):
            kk, vv = held(np.concatenate([keys[i], k[t:t + m]]), kv8), held(np.concatenate([values[i], v[t:t + m]]), kv8)
            check(got[t:t + m], z[t:t + m], q[t:t + m], kk, vv, past + own[i], full[i], SCALE, "fork %d" % i)
            t += m
        B.oxy_batch_destroy(batch)
    finally:
        pool.close()


@FORMS
def test_frames_behind_one_history(kv8):
    forks(kv8, 576, [0] * 4, [256] * 4, 1)


@FORMS
def test_many_forks_of_a_long_history(kv8):
    """Records of more pages than they list themselves."""
    forks(kv8, 8192, [0] * 40, [1 + i % 3 for i in range(40)], 2)


@FORMS
def test_forks_that_have_tokens_of_their_own(kv8):
    """The shared pages end inside records."""
    forks(kv8, 4096, [0, 700, 33, 16, 5, 299, 0, 1], [17, 2, 40, 1, 3, 100, 33, 16], 3)
