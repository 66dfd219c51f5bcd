"""Recorded steps of a pool in 8 bits on both sides of 2048 new tokens, where the append becomes another kernel."""
import pytest

pytestmark = pytest.mark.gpu


def test_recordings_on_both_sides_of_large_appends():
    """More forms than recordings are held, so that they are updated in place; each step gives the bits of one that is
    not recorded, with eager work between them."""
    import torch
    from paper_2603_14371_amd import binding as B
    lens = [2040, 2049, 300, 2060, 2048, 2100, 310, 2044, 2055, 2047, 2064, 320, 2049, 2040]
    most = max(lens)
    gen = torch.Generator(device="cuda").manual_seed(3)
    rows = [torch.randn(2, most, 256, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2)]
    q = torch.randn(2, most, 8, 256, generator=gen, device="cuda").to(torch.bfloat16)
    outs = {}
    for flags in (0, B.STEP_GRAPH):
        cfg = B.make_config(2, 200, flags=B.POOL_KV_FP8, max_q_tokens=most, max_append_tokens=most)
        kv = torch.full((B.oxy_kv_bytes(cfg),), 0xFF, dtype=torch.uint8, device="cuda")
        ws = torch.empty(B.oxy_workspace_bytes(cfg), dtype=torch.uint8, device="cuda")
        cfg.kv_base, cfg.kv_bytes, cfg.workspace, cfg.workspace_bytes = kv.data_ptr(), kv.numel(), ws.data_ptr(), ws.numel()
        pool, s = B.oxy_pool_create(cfg), torch.cuda.current_stream().cuda_stream
        sid = B.oxy_stream_create(pool, -1, B.KIND_ACTION)
        out, lse, got = torch.zeros_like(q), torch.zeros(2, most, 8, device="cuda"), []
        for n in lens:
            out.zero_(), lse.zero_()
            batch = B.oxy_batch_build(pool, [(sid, n)], 0, s)
            B.oxy_step_layers(pool, batch, 0, 2, rows[0].data_ptr(), rows[1].data_ptr(), most * 512, q.data_ptr(), out.data_ptr(),
                              most * 4096, lse.data_ptr(), most * 32, 1.0 / 16, flags, None, s)
            B.oxy_batch_destroy(batch)
            got.append((out.clone(), lse.clone()))
        torch.cuda.synchronize()
        outs[flags] = got
        made, updated, replayed = B.oxy_step_graph_stats(pool)
        assert (replayed, updated > 0) == ((len(lens), True) if flags else (0, False))
        B.oxy_pool_destroy(pool)
    for n, plain, recorded in zip(lens, outs[0], outs[B.STEP_GRAPH]):
        assert torch.equal(plain[0], recorded[0]) and torch.equal(plain[1], recorded[1]), n
        assert plain[0][:, :n].float().abs().amax(dim=(0, 2, 3)).min() > 0 and not plain[0][:, n:].any(), n
