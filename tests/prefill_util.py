"""What the tests of a prefill share: a pool with prefixes in it, a batch of their new tokens or of whole prompts, and
the comparison with the float64 oracle within what the roundings may cost."""
import numpy as np

from oracle import kv8, prefill
from oracle.attention import widen_bf16

HALF16 = 2.0 ** -8      # half a step of bf16, relative


def bits(rng, *shape, scale=1.0):
    x = (scale * rng.standard_normal(shape)).astype(np.float32)
    return (x.view(np.uint32) >> 16).astype(np.uint16)


def up(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a).view(np.int16)).cuda()


def down(t):
    import torch
    torch.cuda.synchronize()
    return t.view(torch.int16).cpu().numpy().view(np.uint16)


class Pool:
    """A pool on the device."""

    def __init__(self, layers, blocks, kv8=False, seed=None, small=False, **kw):
        """small: a workspace for max_partials split results and no more."""
        import torch
        from paper_2603_14371_amd import binding as B
        order = None if seed is None else np.random.default_rng(seed).permutation(blocks)
        cfg = B.make_config(layers, blocks, free_order=order, flags=B.POOL_KV_FP8 if kv8 else 0, **kw)
        # never-written slots hold NaN
        self.kv = torch.full((B.oxy_kv_bytes(cfg),), 0xff, dtype=torch.uint8, device="cuda")
        n_ws = B.oxy_workspace_bytes(cfg)
        if small:
            few = kw["max_partials"]
            n_ws -= 2 * ((8192 - few) * 4096 + 8192 * 128 - -(-few * 128 // 256) * 256)
        self.ws = torch.full((n_ws,), 0xff, dtype=torch.uint8, device="cuda")
        cfg.kv_base, cfg.kv_bytes = self.kv.data_ptr(), self.kv.numel()
        cfg.workspace, cfg.workspace_bytes = self.ws.data_ptr(), self.ws.numel()
        self.B, self.kv8, self.p = B, kv8, B.oxy_pool_create(cfg)
        self.stream = torch.cuda.current_stream().cuda_stream

    def prefix(self, k, v, layer=0):
        """A prefix that holds these rows (bits [n, 256])."""
        pid = self.B.oxy_prefix_create(self.p)
        if len(k):
            dk, dv = up(k), up(v)
            self.B.oxy_prefix_append(self.p, pid, layer, dk.data_ptr(), dv.data_ptr(), len(k), 0, self.stream)
            down(dk)
        return pid

    def close(self):
        import torch
        torch.cuda.synchronize()
        try:
            self.B.oxy_pool_destroy(self.p)
        except self.B.OxyError as e:       # a test that failed left its batch
            if e.code != self.B.ERR_BUSY:
                raise


def held(x, in8):
    """What a cache holds for rows of bits, in float64."""
    return kv8.cached_values(x) if in8 else widen_bf16(x)


def check(got, lse, q, k, v, past, full, scale, what=""):
    """One item: got, q bits [n, 8, 256]; lse [n, 8] or None; k, v float64 rows that the cache holds.

    A logit's 256 products are summed in 32 bits (256 half steps of the products' sizes together), scaled and
    subtracted from by one operation (half a step of the logit), and taken to the exponential, whose result is off by
    a step; a weight is then rounded to bf16 (half a step, 2^-8), sums over n keys to 32 bits, split results to fp16
    (2^-11), and the output to bf16."""
    n_keys = len(k)
    o, z, spread, reach = prefill.attend(widen_bf16(q), k, v, past, full, scale)
    logit = abs(scale) * reach * (256 + 4) * 2.0 ** -24 + 2.0 ** -22
    weight = HALF16 + 2 * logit[..., None] + (n_keys + 64) * 2.0 ** -24 + 2.0 ** -11
    tol = HALF16 * np.abs(o) + 1.01 * weight * spread + 1e-37
    err = np.abs(widen_bf16(got) - o)
    assert np.all(err <= tol), "%s: worst %.3f of what the roundings allow" % (what, np.nanmax(err / tol))
    assert np.all(np.isfinite(widen_bf16(got)))
    if lse is not None:
        tol = 2 * logit + (n_keys + 64) * 2.0 ** -24 + np.abs(z) * 2.0 ** -22
        assert np.all(np.abs(lse - z) <= tol), "%s: lse %.3e" % (what, np.abs(lse - z).max())
