"""The plain 4-bit cache and beam selection (tests/kv4.py) against hand-worked cases and the
definitions' own statements."""
from fractions import Fraction

import numpy as np
import pytest

import kv4


@pytest.mark.parametrize("hd", [32, 64, 128])
def test_every_element_has_a_place_of_its_own(hd):
    at, pairs = kv4.maps(hd)
    places = [tuple(p) for a in at for row in a for p in row]
    assert len(set(places)) == 2 * 32 * hd and {p[1] for p in places} == {0, 4}
    assert {p[0] for p in places} == set(range(32 * hd))
    assert sorted(pairs.ravel()) == list(range(32 * hd, kv4.tile_bytes(hd), 4))
    # a byte is one token's
    for v in (0, 1):
        owner = {}
        for key in range(32):
            for b, _ in at[v][key]:
                assert owner.setdefault(b, key) == key


def test_codes_by_hand():
    # 0 .. 15 with a step of 1; halves go up
    x = np.zeros(64, np.float16)
    x[:6] = [0, 15, 7.5, 7.25, 14.5, 0.5]
    n, s, m = kv4.quantize(x)
    assert list(n[:6]) == [0, 15, 8, 7, 15, 1] and s[0] == 1 and m[0] == 0
    # the scale is rounded up: 1 / 15
    x = np.where(np.arange(32) == 3, np.float16(1), np.float16(0))
    n, s, m = kv4.quantize(x)
    assert Fraction(float(s[0])) >= Fraction(1, 15) > Fraction(float(np.nextafter(s[0], np.float16(0))))
    assert n[3] == 15 and n.sum() == 15
    # one value alone, and the type's whole range
    n, s, m = kv4.quantize(np.full(64, -3.25, np.float16))
    assert not n.any() and s[0] == 0 and m[0] == np.float16(-3.25)
    x = np.where(np.arange(64) % 2, np.float16(65504), np.float16(-65504))
    n, s, m = kv4.quantize(x)
    assert m[0] == -65504 and np.isfinite(s[0]) and set(n) == {0, 15}
    assert np.isfinite(kv4.read_back(n, s, m)).all()


@pytest.mark.parametrize("scale", [1e-7, 1e-4, 1.0, 3e4])
def test_no_element_is_further_than_half_a_step(scale):
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((200, 128)) * scale).clip(-65504, 65504).astype(np.float16)
    n, s, m = kv4.quantize(x)
    err = np.abs(kv4.values(n, s, m) - x.astype(np.float64)).reshape(200, 2, 64)
    assert (err <= s.astype(np.float64)[..., None] / 2).all()


def test_selection_by_hand():
    z = np.log(np.array([[0.5, 0.25, 0.125, 0.125], [0.7, 0.1, 0.1, 0.1]]))
    z[1, 1:] = [-np.inf] * 3  # one token alone: probability 1
    p, t, s, d = kv4.select(z, [-1.0, -1.5], [0, 0], 4, eos=1, pad=3)
    assert list(p) == [1, 0, 0, 0] and list(t) == [0, 0, 1, 2] and list(d) == [0, 0, 1, 0]
    assert np.allclose(s, [-1.5, -1 + np.log(0.5), -1 + np.log(0.25), -1 + np.log(0.125)])
    # ended hypotheses go on as themselves; an empty place offers nothing
    p, t, s, d = kv4.select(z, [-1.0, -np.inf], [1, 0], 3, eos=1, pad=3)
    assert list(p) == [0, 0, 0] and list(t) == [3, 3, 3] and list(d) == [1, 1, 1] and list(s) == [-1, -np.inf, -np.inf]
    # equal offers: the first hypothesis, then the lower token
    p, t, s, d = kv4.select(np.zeros((2, 3)), [-1.0, -1.0], [0, 0], 4, eos=-1, pad=0)
    assert list(p) == [0, 0, 0, 1] and list(t) == [0, 1, 2, 0]
