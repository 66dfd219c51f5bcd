"""Batches of forks compiled with gcc under AddressSanitizer + UndefinedBehaviorSanitizer, on pools without a block to
spare (tests/hostbuild/prefill_forks_main.cpp).  No GPU."""
import os

import pytest

from paper_2603_14371_amd import binding as B
from test_host_kv8 import HB, _build, _run


def test_every_page_of_every_fork(tmp_path):
    exe = str(tmp_path / "forks_asan")
    _build(exe, [os.path.join(HB, "prefill_forks_main.cpp")])
    _run(exe)


@pytest.mark.parametrize("forks,past,n", [(4, 576, 256), (8, 2048, 16), (16, 8192, 16)])
def test_forks_need_no_more_than_their_blocks(forks, past, n):
    blocks = past // 16 + forks * -(-n // 16)
    pool = B.oxy_pool_create(B.make_config(1, blocks, flags=B.POOL_HOST_ONLY, max_q_tokens=forks * n))
    parent = B.oxy_prefix_create(pool)
    B.oxy_prefix_append(pool, parent, 0, 0, 0, past, 0, 0)
    pids = [B.oxy_prefix_fork(pool, parent, past) for _ in range(forks)]
    batch = B.oxy_prefix_batch_build(pool, [(pid, n, past + n) for pid in pids], 0, 0)
    assert B.oxy_batch_info(batch)[:2] == (forks, forks * n) and B.oxy_free_blocks(pool) == []
    B.oxy_batch_destroy(batch)
    B.oxy_pool_destroy(pool)
