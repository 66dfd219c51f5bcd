"""Tokens of so many split results that a wavefront of the join takes them in more than one round."""
import numpy as np
import pytest

from prefill_util import bits
from test_gpu_prefill_weights import both

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("way", ["pages", "pages8"])
@pytest.mark.parametrize("rising", [True, False, None])
@pytest.mark.parametrize("past,n", [(9000, 1), (20000, 3), (40000, 17)])
def test_more_than_128_split_results_of_a_token(past, n, rising, way):
    """Eight wavefronts take an eighth each, sixteen at a time.  Rising: the largest logits come last, so that a later round
    changes the scale of what the earlier ones summed; falling, and in no order."""
    rng = np.random.default_rng(past + n)
    q, k, v = bits(rng, n, 8, 256), bits(rng, past + n, 256), bits(rng, past + n, 256)
    if rising is not None:
        ramp = np.linspace(-60.0, 60.0, past + n, dtype=np.float32) * (1 if rising else -1)
        k[:, 0] = ramp.view(np.uint32) >> 16
        q[:, :, 0] = np.float32(3.0).view(np.uint32) >> 16      # logits of -11 to 11, and what the other dims add
    # split results of all n tokens: more than 128 of each
    assert both(way, q, k, v, past) > 128 * n
