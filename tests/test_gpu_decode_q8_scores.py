"""Attention over the 8-bit cache with scores of every size that fp16 queries and keys
reach: a key that the others lie far below has all of the weight, and no score is too
large for the running softmax."""
import numpy as np
import pytest

import kv8
from helpers import gpu_ctx
from test_gpu_kv_cache8 import Step, _d

pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = gpu_ctx()
    yield c
    c.close()


# 700 rows: a warp per task; the others: several CTAs for one
@pytest.mark.parametrize("heads,lens", [((8, 8, 64), [70] * 700), ((8, 1, 32), [40] * 2500), ((4, 1, 128), [3000, 45])],
                         ids=lambda v: str(v) if isinstance(v, tuple) else f"{len(v)}x{v[0]}")
@pytest.mark.parametrize("sign", [1, -1], ids=["positive", "negative"])
def test_scores_of_every_size(ctx, heads, lens, sign):
    Hq, Hkv, hd = heads
    s = Step(2, *heads, lens, 3, 32)
    rng, w = s.rng, 2 * Hkv * hd
    st = kv8.starts(lens)

    # key n of a head is size * f[n] along all elements; f is 1 for one key of each row and
    # at most 0.9 for the others (negative scores: 0.5, and 0.55 at least)
    def factors(n, best=None):
        f = rng.uniform(0.3, 0.9, (n, Hkv)) if sign > 0 else rng.uniform(0.55, 1.0, (n, Hkv))
        if best is not None:
            f[best] = 1.0 if sign > 0 else 0.5
        return f

    def rows(f, size):
        x = np.empty((len(f), 2, Hkv, hd))
        x[:, 0] = (size * f)[..., None]
        x[:, 1] = rng.standard_normal((len(f), Hkv, hd)) + 3
        return x.reshape(len(f), w).astype(np.float16)

    best = [int(rng.integers(0, n)) for n in lens]
    own_f = np.concatenate([factors(n, b) for n, b in zip(lens, best)])
    pre_f, new_f = factors(3), factors(s.R)
    for log_q, log_k in [(4, 4), (7, 8), (8, 8), (8, 9), (9, 9), (10, 10), (11, 11), (12, 12), (13, 13), (14, 14), (15.9, 15.9)]:
        k = 2.0 ** log_k
        own, pre = rows(own_f, k), rows(pre_f, k)
        s.own_c, s.own_s, q8, sc = kv8.build_cache(own, lens, Hkv, hd)
        s.own = q8 * sc[..., None]
        s.pre_c, s.pre_s, _, _ = kv8.build_cache(pre, [3], Hkv, hd)
        s.d[:4] = [_d(a) for a in (s.own_c, s.own_s, s.pre_c, s.pre_s)]
        qkv = np.empty((s.R, (Hq + 2 * Hkv) * hd), np.float16)
        # each row its own size, so that the scores' last places differ
        qkv[:, :Hq * hd] = (sign * 2.0 ** (log_q - rng.random((s.R, 1)))).astype(np.float16)
        qkv[:, Hq * hd:] = rows(new_f, k)
        out = s.call(ctx, qkv, 0).astype(np.float64).reshape(s.R, Hkv, Hq // Hkv, hd)
        for r in range(s.R):
            v = s.own[st[r] + best[r], 1]  # [Hkv, hd]
            # the others' weight is below 2^-100: one product with a probability and its sum, and a rounding
            assert (np.abs(out[r] - v[:, None]) <= np.abs(v[:, None]) * (2.0 ** -11 + 2.0 ** -20)).all(), (log_q, r)
