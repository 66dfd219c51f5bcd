"""Softmax weights of a prefill on their way into the product with the values: rows that see few keys, whose weights are a
few large ones, or whose weights all round the same way, are as exact as a step's attention."""
import numpy as np
import pytest

from oracle import prefill
from oracle.attention import widen_bf16
from parity_util import assert_lse_close, assert_o_close
from prefill_util import HALF16, Pool, bits, down, held, up

pytestmark = pytest.mark.gpu
SCALE = 1.0 / 16
WAYS = pytest.mark.parametrize("way", ["rows", "pages", "pages8"])


def attend(way, q, k, v, past=0, full=0, scale=SCALE, whole=False):
    """One item of len(k) tokens, the last len(q) of them queries: outputs (bits), log-sum-exps, split results.  whole: on a
    workspace without room for split results, so that a row's keys have one reference."""
    import torch
    n = len(q)
    kw = {"max_partials": 1} if whole else {}
    pool = Pool(1, (len(k) + 15) // 16 + 1, way == "pages8", seed=1, small=whole, max_q_tokens=max(16, n),
                max_append_tokens=max(16, n), **kw)
    B = pool.B
    try:
        dq, dk, dv = up(q), up(k[past:]), up(v[past:])
        out, lse = torch.zeros((n, 8, 256), dtype=torch.int16, device="cuda"), torch.zeros((n, 8), device="cuda")
        if way == "rows":
            b = B.oxy_prompt_batch_build(pool.p, [(n, full)], pool.stream)
            B.oxy_prompt_attention(pool.p, b, dq.data_ptr(), 4096, dk.data_ptr(), 512, dv.data_ptr(), 512, out.data_ptr(),
                                   4096, lse.data_ptr(), scale, pool.stream)
        else:
            pid = pool.prefix(k[:past], v[:past])
            b = B.oxy_prefix_batch_build(pool.p, [(pid, n, full)], 0, pool.stream)
            B.oxy_stream_append(pool.p, b, 0, dk.data_ptr(), dv.data_ptr(), pool.stream)
            B.oxy_prefix_attention(pool.p, b, 0, dq.data_ptr(), 4096, out.data_ptr(), 4096, lse.data_ptr(), scale, pool.stream)
        got, info = down(out), B.oxy_batch_info(b)
        B.oxy_batch_destroy(b)
        return got, lse.cpu().numpy().astype(np.float64), info[3]
    finally:
        pool.close()


def both(way, q, k, v, past=0, full=0, scale=SCALE, whole=False):
    """Within the tolerance of a step's attention, and element by element within what the roundings may cost: a weight in
    two halves is off by 2^-16, split results by half a step of fp16, the output by half a step of bf16; a logit's 256
    products and a row's sum are 32-bit ones, and an exponential is off by a step."""
    got, lse, split = attend(way, q, k, v, past, full, scale, whole)
    wide = widen_bf16(q), held(k, way == "pages8"), held(v, way == "pages8")
    o, z, spread, reach = prefill.attend(*wide, past, full, scale)
    assert_o_close(got, o, way)
    assert_lse_close(lse, z, way)
    logit = abs(scale) * reach * (256 + 4) * 2.0 ** -24 + 2.0 ** -22
    each = 2.0 ** -16 + 2 * logit[..., None] + (len(k) + 64) * 2.0 ** -24 + (2.0 ** -11 if split else 0.0)
    tol = HALF16 * np.abs(o) + 1.01 * each * spread + 1e-37
    err = np.abs(widen_bf16(got) - o)
    assert np.all(err <= tol), "%s: worst %.3f of what the roundings allow" % (way, np.max(err / tol))
    return split


@WAYS
@pytest.mark.parametrize("sigma", [1.0, 3.0, 8.0])
@pytest.mark.parametrize("n", [2, 3, 7, 16, 24, 33, 64])
def test_few_keys(n, sigma, way):
    """A causal prompt; sigma: the keys' size, from even weights to a few large ones."""
    rng = np.random.default_rng(n)
    both(way, bits(rng, n, 8, 256), bits(rng, n, 256, scale=sigma), bits(rng, n, 256))


@WAYS
@pytest.mark.parametrize("sigma", [1.0, 3.0, 8.0])
@pytest.mark.parametrize("n,full", [(200, 0), (130, 130), (470, 300)])
def test_more_keys(n, full, sigma, way):
    rng = np.random.default_rng(n)
    both(way, bits(rng, n, 8, 256), bits(rng, n, 256, scale=sigma), bits(rng, n, 256), full=full)


@pytest.mark.parametrize("way", ["pages", "pages8"])
@pytest.mark.parametrize("sigma", [1.0, 3.0, 8.0])
@pytest.mark.parametrize("past,n", [(40, 1), (800, 3), (2000, 17)])
def test_behind_a_history(past, n, sigma, way):
    rng = np.random.default_rng(past + n)
    both(way, bits(rng, n, 8, 256), bits(rng, past + n, 256, scale=sigma), bits(rng, past + n, 256), past)


@WAYS
def test_a_row_does_not_go_by_keys_of_others(way):
    """A key that only later queries see becomes much larger: earlier rows keep every bit."""
    rng = np.random.default_rng(3)
    n = 60
    q, k, v = bits(rng, n, 8, 256), bits(rng, n, 256), bits(rng, n, 256)
    for at in (1, 17, 35, 58):
        other = k.copy()
        other[at] = bits(rng, 256, scale=30.0)
        a, b = (attend(way, q, x, v)[0] for x in (k, other))
        assert np.array_equal(a[:at], b[:at]) and not np.array_equal(a[at:], b[at:])


def _by_logit(log2_weights, n):
    """q of n tokens and one key for each weight: a logit is the first dim's alone."""
    q, k = np.zeros((n, 8, 256), np.float32), np.zeros((len(log2_weights), 256), np.float32)
    q[:, :, 0] = 1.0
    k[:, 0] = np.asarray(log2_weights) * np.log(2.0) / SCALE
    return [(x.view(np.uint32) >> 16).astype(np.uint16) for x in (q, k)]


@WAYS
@pytest.mark.parametrize("whole", [False, True])
@pytest.mark.parametrize("n", [40, 700])
@pytest.mark.parametrize("what", ["even", "random"])
def test_equal_values(what, n, whole, way):
    """Where all values are one row, the output is that row, bit for bit: 2^-16 of a weight, 2^-11 of a split result and
    two sums of n numbers (n 2^-23) together are less than the least half step of bf16, 2^-9.  Even: all keys behind the
    first tile have a weight a little above 1 + 2^-8 of the reference, which one rounding to bf16 takes up."""
    rng = np.random.default_rng(n)
    weights = np.r_[np.zeros(32), np.full(n - 32, np.log2(1.0045))] if what == "even" else rng.normal(0, 2, n)
    m = n if way == "rows" else 20
    q, k = _by_logit(weights, m)
    v = np.repeat(bits(rng, 1, 256), n, axis=0)
    got, _, split = attend(way, q, k, v, n - m, n, whole=whole)
    assert not (whole and split)
    want = held(v[:1], way == "pages8")[0]
    assert np.array_equal(widen_bf16(got), np.broadcast_to(want, got.shape))


@WAYS
@pytest.mark.parametrize("log2_weight", [7.3, 7.9, 1.005, 3.505])
def test_a_later_key_that_dominates(log2_weight, way):
    """Its logit is above the reference, but not by what moves it: a weight of up to 2^8 that is no power of two."""
    rng = np.random.default_rng(int(100 * log2_weight))
    n = 70
    weights = rng.normal(-6, 1, n)
    weights[:3] = 0.0
    weights[50] = log2_weight
    q, k = _by_logit(weights, n)
    both(way, q, k, bits(rng, n, 256), full=n, whole=True)
