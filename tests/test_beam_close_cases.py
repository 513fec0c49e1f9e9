"""The groups of close hypotheses that selection is tested with are close, and not too close."""
import numpy as np
import pytest

import beam_close
import kv4


@pytest.mark.parametrize("type", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("maker", ["ties", "peaked", "light"])
def test_offers_are_closer_than_32_bits_tell(maker, type):
    rng = np.random.default_rng(5)
    if maker == "ties":
        z, scores, done, keep = beam_close.ties_at_the_border(rng, 40, 3, 2000, type)
    elif maker == "peaked":
        z, scores, done, keep = beam_close.peaked_before_flat(rng, 40, 2000, type)
    else:
        z, scores, done, keep = beam_close.light_tokens(rng, 40, 4, 2000, type)
    assert np.array_equal(beam_close.held(z, type), z)
    kept_both_ways = set()
    for g in range(40):
        p, t, s, _ = kv4.select(z[g], scores[g], done[g], keep + 1, -1, 0)
        if maker == "ties":
            assert p[0] == p[1] != p[2] or p[0] != p[1] == p[2]
            kept_both_ways.add(bool(p[0] == p[1]))
        elif maker == "peaked":
            kept_both_ways.add(float(z[g, p[1]].max()) == 3)
        else:
            order = kv4.select(z[g], scores[g], done[g], 4, -1, 0)[0]
            assert len(set(order.tolist())) == 4  # each hypothesis' largest, in the order of their sums
            d = -np.diff(kv4.select(z[g], scores[g], done[g], 4, -1, 0)[2])
            assert (d >= beam_close.LEAST).all() and (d <= beam_close.BOUND / 2).all()
    if maker != "light":
        assert kept_both_ways == {True, False}
        d = beam_close.gaps(z, scores, done, keep)
        assert (d >= beam_close.LEAST * 0.99).all() and (d <= 2.0 ** -22).all()
