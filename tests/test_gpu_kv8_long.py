"""Launches of a pool in 8 bits in which some tokens have many split results and most have few."""
import numpy as np
import pytest

from paper_2603_14371_amd.synth import ACTION, DECODE, _TraceBuilder, _workload
from test_gpu_kv8 import _only, run_both8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("chunk", [1, 50, 300])
def test_long_tokens_anywhere_among_short_ones(chunk):
    """First, last and in the middle; several of one request; more tokens than the other merges take one way or another."""
    b = _TraceBuilder()
    pid = b.prefix(300)
    act, s0, s1 = b.stream(pid, ACTION), b.stream(pid, DECODE), b.stream(-1, DECODE)
    l0, l1, l2 = (b.stream(p, DECODE) for p in (pid, -1, pid))
    b.step([(l0, 4200), (l1, 1500), (l2, 2100), (s0, 100), (s1, 900)], attend=False)
    b.step([(l0, 1), (act, chunk), (s0, 2), (l1, 3), (s1, 1), (l2, 1)])
    b.step([(s1, 1), (l1, 1), (act, chunk)])
    b.step([(l1, 2), (l0, 1)])                    # none but long ones
    w = _workload("mixed", 11, 1, 1200, b.trace)
    gw, _ = run_both8(w, poison=True, max_partials=16384, stream_split_tokens=32)
    gw.close()


def test_a_long_token_gives_the_same_bits_alone_and_among_others():
    me = (0, 20000, 2, 7)
    alone = _only([900], [], [me], 7)
    few = _only([900], [(0, 13, 1)], [(0, 40, 1, 2), me], 7)
    many = _only([900, 300], [(i % 2, 50, 10 + i) for i in range(6)],
                 [(0, 9000, 1, 90), me] + [(i % 2, 20 * i, 1, 20 + i) for i in range(20)], 7)
    for other in (few, many):
        assert np.array_equal(alone[0], other[0]) and np.array_equal(alone[1], other[1])
