"""Rotations of more than 2048 tokens, four tokens a workgroup, in every form: pairs, halves in whole 16-byte chunks, halves that
are not; heads that fill a half wavefront's rows in flight or do not, views, rows turned in place, the last workgroup
ragged.  The tolerance is that of test_gpu_rotary.Turn.check."""
import numpy as np
import pytest

from test_gpu_rotary import Turn, _bits, _down, _rotate, _up

pytestmark = pytest.mark.gpu
FORMS = [("pairs", 256), ("pairs", 128), ("pairs", 2), ("pairs", 90), ("halves", 256), ("halves", 128), ("halves", 16),
         ("halves", 100), ("halves", 2), ("halves", 254)]


@pytest.mark.parametrize("layout,rot", FORMS)
@pytest.mark.parametrize("n,heads", [(2049, 1), (2050, 2), (2051, 7), (2052, 9), (4097, 3)])
def test_every_form(layout, rot, n, heads):
    rng = np.random.default_rng(n)
    turn = Turn(rot, layout, amplitude=1.25)
    bits, pos = _bits(rng, n, heads, 256), rng.integers(-(1 << 20), 1 << 20, n)
    turn.check(bits, pos, _down(_rotate(turn, _up(bits), pos, n, heads)))


@pytest.mark.parametrize("layout,rot", FORMS)
@pytest.mark.parametrize("n,heads", [(2051, 9), (2050, 5), (2049, 6), (2052, 1)])
def test_views_and_rows_in_place(layout, rot, n, heads):
    """Out of wide rows into wider ones: what lies between them stays; and onto themselves: the same bits."""
    import torch
    rng = np.random.default_rng(heads)
    turn = Turn(rot, layout)
    wide, pos = _bits(rng, n, 10, 256), rng.integers(0, 9000, n)
    x = _up(wide)
    out = torch.full((n, 12, 256), 77, dtype=torch.int16, device="cuda")
    _rotate(turn, x[:, 1:], pos, n, heads, 10 * 512, out[:, 2:], 12 * 512)
    got = _down(out)
    turn.check(wide[:, 1:1 + heads], pos, got[:, 2:2 + heads])
    assert np.all(got[:, :2] == 77) and np.all(got[:, 2 + heads:] == 77) and np.array_equal(_down(x), wide)
    _rotate(turn, x[:, 1:], pos, n, heads, 10 * 512, x[:, 1:], 10 * 512)
    own = _down(x)
    assert np.array_equal(own[:, 1:1 + heads], got[:, 2:2 + heads])
    assert np.array_equal(own[:, :1], wide[:, :1]) and np.array_equal(own[:, 1 + heads:], wide[:, 1 + heads:])


@pytest.mark.parametrize("layout,rot", [("pairs", 128), ("halves", 128), ("halves", 100)])
def test_a_token_gives_the_same_bits_among_few_and_many(layout, rot):
    rng = np.random.default_rng(8)
    turn = Turn(rot, layout)
    bits, pos = _bits(rng, 3001, 5, 256), rng.integers(0, 1 << 20, 3001)
    many = _down(_rotate(turn, _up(bits), pos, 3001, 5))
    for a, b in ((0, 1), (1, 4), (700, 1500), (2990, 3001)):
        few = _down(_rotate(turn, _up(bits[a:b]), pos[a:b], b - a, 5))
        assert np.array_equal(few, many[a:b])
