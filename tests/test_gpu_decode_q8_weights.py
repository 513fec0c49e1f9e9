"""Attention over the 8-bit cache where one key has nearly all of the weight and the
output is what the many others add: their probabilities, 2^-12 to 2^-26 of the
largest, count with their own rounding, not with the largest one's."""
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


def _bound(q, k, v):
    """(out, bound) as kv8.attend, of a kernel that keeps of a probability what its
    rounding to fp16 leaves as a second fp16 number: off by 2^-22 of itself, or by half
    of fp16's last place, 2^-25, where the largest probability is 2^11 at least: 2^-36 of it."""
    Hq, hd = q.shape
    G = Hq // k.shape[1]
    k, v = np.repeat(k, G, 1), np.repeat(v, G, 1)
    z = np.einsum("hd,nhd->hn", q, k) / np.sqrt(hd)
    S = (np.einsum("hd,nhd->hn", np.abs(q), np.abs(k)) / np.sqrt(hd)).max(1)
    p = np.exp(z - z.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    out = np.einsum("hn,nhd->hd", p, v)
    A = np.einsum("hn,nhd->hd", p, np.abs(v))
    rel = 2.0 ** -22 + 2.0 ** -18 + 2 * (hd + 8) * 2.0 ** -23 * S[:, None]
    small = 2.0 ** -36 * np.abs(v).sum(0) * p.max(1)[:, None]
    return out, A * rel + small + 2.0 ** -11 * np.abs(out) + 2.0 ** -25


def _sink(seed, heads, lens, first):
    """A key of 8 along element 0 with value 0, first of the prefix (`first`) or of the
    generated tokens; all other keys have nothing there and values about 500."""
    Hq, Hkv, hd = heads
    s = Step(seed, *heads, lens, 1, 32)
    rng, w = s.rng, 2 * Hkv * hd

    def rows(n, sink=False):
        x = np.zeros((n, 2, Hkv, hd))
        x[:, 0, :, 1:] = rng.standard_normal((n, Hkv, hd - 1)) * 0.5
        x[:, 1] = 500 * np.exp(0.3 * rng.standard_normal((n, Hkv, hd)))
        if sink:
            x[0, 0, :, 0], x[0, 0, :, 1:], x[0, 1] = 8, 0, 0
        return x.reshape(n, w).astype(np.float16)

    own, pre = rows(s.T), rows(1, first)
    s.own_c, s.own_s, q, sc = kv8.build_cache(own, lens, Hkv, hd)
    s.own = q * sc[..., None]
    s.pre_c, s.pre_s, q, sc = kv8.build_cache(pre, [1], Hkv, hd)
    s.pre = q * sc[..., None]
    s.d[:4] = [_d(a) for a in (s.own_c, s.own_s, s.pre_c, s.pre_s)]
    s.gen = [rows(3, not first) for _ in range(s.R)]
    tail = np.full((s.R, 32, w), np.float16(np.nan))
    for r in range(s.R):
        tail[r, :3] = s.gen[r]
    s.tail = _d(tail)
    qkv = np.zeros((s.R, (Hq + 2 * Hkv) * hd), np.float16)
    bits = 12 + 14 * rng.random((s.R, Hq))  # log2 of the largest probability over the others'
    x = rng.standard_normal((s.R, Hq, hd)) * 0.05
    x[:, :, 0] = bits * np.sqrt(hd) / (8 * np.log2(np.e))
    qkv[:, :Hq * hd] = x.reshape(s.R, -1)
    qkv[:, Hq * hd:] = rows(s.R)
    return s, qkv


@pytest.mark.parametrize("first", [True, False], ids=["first", "last"])
@pytest.mark.parametrize("heads,lens", [((8, 8, 32), [150] * 700), ((32, 8, 64), [150 + i % 50 for i in range(700)]),
                                        ((8, 8, 128), [120] * 700), ((8, 1, 64), [40] * 1500), ((5, 1, 128), [33] * 2500),
                                        ((8, 2, 64), [300] * 20), ((4, 1, 128), [9000, 70]), ((8, 1, 32), [20000])], ids=lambda v:
                         str(v) if isinstance(v, tuple) else f"{len(v)}x{v[0]}")
def test_keys_far_below_the_largest_count(ctx, heads, lens, first):
    Hq, Hkv, hd = heads
    s, qkv = _sink(len(lens) + hd, heads, lens, first)
    out = s.call(ctx, qkv, 3).astype(np.float64)
    s.append(qkv)
    st, worst = kv8.starts(lens), 0.0
    for r in range(s.R):
        kv = np.concatenate([s.pre, s.own[st[r]:st[r + 1]], s.generated(r)])
        ref, bound = _bound(qkv[r, :Hq * hd].astype(np.float64).reshape(Hq, hd), kv[:, 0], kv[:, 1])
        worst = max(worst, float((np.abs(out[r].reshape(Hq, hd) - ref) / bound).max()))
    assert worst <= 1, f"{worst:.2f} of the bound"
