"""Groups of hypotheses whose offers lie closer together than sums of 32-bit exponentials tell apart, and
further apart than 2^-31, so that their order is a matter of the definition (include/aiq_ops.h) alone.

Each maker gives (z [n, beams, V] fp32 values that `type` holds, scores [n, beams] fp32, done [n, beams], keep)."""
import numpy as np

import kv4

LEAST = 2.0 ** -31   # of a difference that counts: selection is exact to 2^-32
BOUND = 2.0 ** -19   # a flat row's 32-bit sum is looked at again for differences up to this, at least


def held(x, type):
    """fp32 numbers as the type holds them (to the nearest)."""
    x = np.asarray(x, np.float32)
    if type == "f16":
        return x.astype(np.float16).astype(np.float32)
    if type == "bf16":
        b = x.view(np.uint32).astype(np.uint64)
        return ((b + 0x7fff + (b >> 16 & 1)) & 0xffff0000).astype(np.uint32).view(np.float32)
    return x


def log_sum(row):
    top = row.max()
    return float(top) + np.log(np.sort(np.exp(row.astype(np.float64) - top)).sum())


def _score(want, by):
    """The fp32 number next to want + by that is on by's side of `want`, by LEAST at least."""
    c = np.float32(want + by)
    while (float(c) - want) * np.sign(by) < LEAST:
        c = np.nextafter(c, np.float32(np.sign(by) * np.inf))
    return c


def _step(rng):
    return rng.choice([-1.0, 1.0]) * 2.0 ** -rng.uniform(24, 30.5)


def ties_at_the_border(rng, n, beams, V, type):
    """Kept are two: a hypothesis' largest, and another's largest, of which that has two, or the first one's
    second, which lies next to those, above or below.  How much the other tokens weigh, and with that how far a 32-bit
    sum is off, differs by row."""
    z = held(np.minimum(rng.standard_normal((n, beams, V)) - rng.uniform(0, 6, (n, beams, 1)), 4), type)
    scores = np.full((n, beams), -30, np.float32)
    for g in range(n):
        a, b = rng.permutation(beams)[:2]
        at = rng.permutation(V)[:3]
        z[g, a, at[:2]] = 5.5
        z[g, b, at[1:]] = 6, 5.5
        scores[g, a] = -2.0 ** -5 * rng.uniform(1, 2)
        scores[g, b] = _score(float(scores[g, a]) - log_sum(z[g, a]) + log_sum(z[g, b]), _step(rng))
    return z, scores, np.zeros((n, beams), np.int32), 2


def peaked_before_flat(rng, n, V, type):
    """Behind one that has ended, whichever of three is first is kept: of two, two tokens are all there is, so
    that nothing of their sums is uncertain, and the other's row is flat.  The first two are closer together than the flat
    one's sum is certain."""
    z = held(np.minimum(rng.standard_normal((n, 4, V)), 2.5), type)
    scores, done = np.zeros((n, 4), np.float32), np.zeros((n, 4), np.int32)
    # a light token's logit and the next number that the type holds: their exponentials differ by some 2e-9
    w = {"f32": (-7.0, 2.0 ** -19), "f16": (-16.0, 2.0 ** -6), "bf16": (-18.0, 0.125)}[type]
    for g in range(n):
        a, b, c, d = rng.permutation(4)
        at = rng.permutation(V)[:2]
        for i, light in ((a, w[0]), (b, w[0] + w[1])):
            z[g, i] = -np.inf
            z[g, i, at] = 0, light
        z[g, c, at[0]] = 3
        flat = 3 - log_sum(z[g, c])
        scores[g, a] = scores[g, b] = flat - 2.0 ** -6
        scores[g, c] = _score(float(scores[g, a]) - log_sum(z[g, a]) - flat, _step(rng))
        scores[g, d], done[g, d] = 1, 1
    return z, scores, done, 2


def light_tokens(rng, n, beams, V, type):
    """Alike but for one token, whose exponential is within 2^-20 of the sum of what it is in the others."""
    z = np.repeat(held(np.minimum(rng.standard_normal((n, 1, V)), 4.5), type), beams, 1)
    for g in range(n):
        at = int(rng.integers(V))
        z[g, :, at] = 0
        total = np.exp(log_sum(z[g, 0]))
        k = rng.choice(np.concatenate([np.arange(-511, 0), np.arange(1, 512)]), beams, replace=False)
        z[g, :, at] = held(np.log1p(total * 2.0 ** -30 * k), type)
        for b in range(1, beams):  # (rounded to the type two may have become close, or equal)
            while np.abs(np.diff(np.sort([log_sum(r) for r in z[g, :b + 1]]))).min() < LEAST:
                z[g, b, at] = held(np.log1p(total * 2.0 ** -30 * rng.integers(-511, 512)), type)
    return z, np.full((n, beams), -2.25, np.float32), np.zeros((n, beams), np.int32), 2 * beams


def gaps(z, scores, done, keep):
    """By group: the least difference between the last offer that is kept and any other hypothesis' first that is
    not, in 64 bits."""
    out = []
    for g in range(len(z)):
        p, _, s, _ = kv4.select(z[g], scores[g], done[g], keep, -1, 0)
        least = np.inf
        for b in set(range(len(scores[g]))) - {int(p[-1])}:
            rest = kv4.select(z[g, b:b + 1], scores[g, b:b + 1], done[g, b:b + 1], keep, -1, 0)[2][int((p == b).sum()):]
            if len(rest):
                least = min(least, s[-1] - rest[0])
        out.append(least)
    return np.array(out)
