"""Keys of a prefill that an infinite negative logit takes out: a weight of 0, and NaN where a row has no other key."""
import numpy as np
import pytest

from oracle import prefill
from oracle.attention import widen_bf16
from prefill_util import bits, check, held
from test_gpu_prefill_weights import attend

pytestmark = pytest.mark.gpu
SCALE = 1.0 / 16
MINUS_INF, ONE = 0xff80, 0x3f80


def _without(got, lse, q, k, v, past, gone, in8):
    """Every row is that of its keys without those in `gone`; without any, it is NaN."""
    kk, vv = held(k, in8), held(v, in8)
    for i, seen in enumerate(prefill.sees(past, len(q), 0)):
        left = [j for j in range(seen) if j not in gone]
        if not left:
            assert np.all(np.isnan(widen_bf16(got[i]))) and np.all(lse[i] == -np.inf)
        else:
            check(got[i:i + 1], lse[i:i + 1], q[i:i + 1], kk[left], vv[left], len(left) - 1, 0, SCALE, "row %d" % i)


@pytest.mark.parametrize("way", ["rows", "pages"])
@pytest.mark.parametrize("gone", [[0], [35], [71], [0, 1, 2], list(range(32)), list(range(5, 70))])
def test_keys_with_a_logit_of_minus_infinity(gone, way):
    """A causal prompt; rows before such a key are as without it, and so are those that see it, where another is left."""
    rng = np.random.default_rng(len(gone))
    n, dim = 72, 130
    q, k, v = bits(rng, n, 8, 256), bits(rng, n, 256), bits(rng, n, 256)
    q[:, :, dim] = ONE
    k[gone, dim] = MINUS_INF
    got, lse, _ = attend(way, q, k, v)
    _without(got, lse, q, k, v, 0, set(gone), False)


@pytest.mark.parametrize("gone", [range(0, 400), range(900, 910), range(64, 905), range(0, 902)])
def test_split_results_without_a_key(gone):
    """Whole split results, or all of a token's, in which no key is left."""
    rng = np.random.default_rng(gone[-1])
    past, n, dim = 900, 5, 7
    q, k, v = bits(rng, n, 8, 256), bits(rng, past + n, 256), bits(rng, past + n, 256)
    q[:, :, dim] = ONE
    gone = [j for j in gone if j < past + n]
    k[gone, dim] = MINUS_INF
    got, lse, split = attend("pages", q, k, v, past)
    assert split > n
    _without(got, lse, q, k, v, past, set(gone), False)
