"""The 4-bit key/value cache, its attention, beam search's selection and the reordering of
its state, plainly (numpy), from the definitions in include/aiq_ops.h."""
import numpy as np

from kv8 import BLOCK, blocks, first_block, starts

UNIT = 2.0 ** 24  # every finite fp16 number is a whole number of 2^-24


def group(hd):
    return min(hd, 64)


def tile_bytes(hd):
    return 32 * hd + 256 * (2 if hd == 128 else 1)


def quantize(x):
    """x [..., hd] finite fp16 -> codes (same shape), s and m [..., groups], in whole numbers of 2^-24."""
    x = np.asarray(x, np.float16)
    X = np.rint(x.astype(np.float64) * UNIT).astype(np.int64).reshape(*x.shape[:-1], x.shape[-1] // group(x.shape[-1]), group(x.shape[-1]))
    lo, span = X.min(-1), X.max(-1) - X.min(-1)
    s = (span / 15.0 / UNIT).astype(np.float16)  # near; the least number with 15 s >= span is it or next to it
    for _ in range(2):
        s = np.where(whole(s) * 15 < span, np.nextafter(s, np.float16(np.inf)), s)
    below = np.nextafter(s, np.float16(0))
    s = np.where((s > 0) & (whole(below) * 15 >= span), below, s)
    S = whole(s)
    assert (15 * S >= span).all()
    n = (2 * (X - lo[..., None]) + S[..., None]) // np.maximum(2 * S, 1)[..., None]
    n = np.where(S[..., None] > 0, n, 0)
    assert n.min(initial=0) >= 0 and n.max(initial=0) <= 15
    m = (lo / UNIT).astype(np.float16)
    return n.reshape(x.shape), s, m


def whole(s):
    return np.rint(s.astype(np.float64) * UNIT).astype(np.int64)


def values(n, s, m):
    """What codes [..., hd] with pairs [..., groups] stand for, in 64 bits (exactly)."""
    w = n.reshape(*s.shape, group(n.shape[-1]))
    return (m.astype(np.float64)[..., None] + s.astype(np.float64)[..., None] * w).reshape(n.shape)


def read_back(n, s, m):
    """fp16, rounded once from the exact number, at most 65504."""
    v = np.minimum(values(n, s, m), 65504.0)
    return v.astype(np.float16)


def key_at(hd, key, d):
    """(byte, shift) of element d of a tile's key."""
    k, h, g = key // 16, key // 8 % 2, key % 8
    if hd == 32:
        t, b = d // 8, d % 8 // 2
        return (g * 4 + t) * 16 + (key // 8) * 4 + b, 4 * (d % 2)
    c, t, b = d // 64, d % 64 // 16, d % 16 // 2
    return (((k * (hd // 64) + c) * 8 + g) * 4 + t) * 16 + h * 8 + b, 4 * (d % 2)


def value_at(hd, key, d):
    k, h, t, e = key // 16, key // 8 % 2, key % 8 // 2, key % 2
    if hd == 32:
        g, i = d // 4, d % 4 // 2
        return 16 * hd + (((g * 4 + t) * 2 + k) * 2 + i) * 4 + e * 2 + h, 4 * (d % 2)
    c, g, i = d // 64, d % 64 // 8, d % 8 // 2
    return 16 * hd + ((((k * (hd // 64) + c) * 8 + g) * 4 + t) * 4 + i) * 4 + e * 2 + h, 4 * (d % 2)


def pair_at(hd, key, value, c):
    return 32 * hd + 256 * c + 128 * value + ((key % 8) * 4 + key // 8) * 4


_MAPS = {}


def maps(hd):
    if hd not in _MAPS:
        at = [np.array([[f(hd, j, d) for d in range(hd)] for j in range(BLOCK)]) for f in (key_at, value_at)]
        pairs = np.array([[[pair_at(hd, j, v, c) for c in range(hd // group(hd))] for j in range(BLOCK)] for v in (0, 1)])
        _MAPS[hd] = at, pairs
    return _MAPS[hd]


def tile(n, s, m):
    """A block's codes [2, BLOCK, hd] and pairs [2, BLOCK, groups] as the cache's bytes."""
    hd = n.shape[-1]
    at, pairs = maps(hd)
    out = np.zeros(tile_bytes(hd), np.uint8)
    for v in (0, 1):
        np.bitwise_or.at(out, at[v][..., 0], (n[v] << at[v][..., 1]).astype(np.uint8))
        for i, x in enumerate((s[v], m[v])):
            b = np.ascontiguousarray(x, np.float16).view(np.uint16)
            out[pairs[v] + 2 * i] = b & 255
            out[pairs[v] + 2 * i + 1] = b >> 8
    return out


def held_bytes(hd, keys):
    """Mask of the bytes of a tile that its first `keys` keys hold."""
    at, pairs = maps(hd)
    mask = np.zeros(tile_bytes(hd), bool)
    for v in (0, 1):
        mask[at[v][:keys, :, 0]] = True
        for i in range(4):
            mask[pairs[v][:keys] + i] = True
    return mask


def build_cache(rows, lens, Hkv, hd, T=None, fill=0):
    """fp16 rows [T, 2 Hkv hd] of packed sequences -> (cache [nb, Hkv, bytes], mask of the bytes that are
    defined, and by token the codes [T, 2, Hkv, hd], s and m [T, 2, Hkv, groups])."""
    T = len(rows) if T is None else T
    st, nb = starts(lens), blocks(T, len(lens))
    x = np.asarray(rows, np.float16).reshape(len(rows), 2, Hkv, hd)
    n, s, m = quantize(x)
    cache = np.full((nb, Hkv, tile_bytes(hd)), fill, np.uint8)
    mask = np.zeros(cache.shape, bool)
    for r in range(len(lens)):
        for j in range(-(-int(lens[r]) // BLOCK)):
            a = int(st[r]) + j * BLOCK
            k = min(BLOCK, int(st[r + 1]) - a)
            b = first_block(int(st[r]), r) + j
            held = held_bytes(hd, k)
            for h in range(Hkv):
                full = [np.zeros((2, BLOCK, y.shape[-1]), y.dtype) for y in (n, s, m)]
                for f, y in zip(full, (n, s, m)):
                    f[:, :k] = y[a:a + k, :, h].swapaxes(0, 1)
                t = tile(*full)
                cache[b, h, held] = t[held]
                mask[b, h] = held
    return cache, mask, n, s, m


def attend(q, k, v, kmax, vmax):
    """q [Hq, hd], exact keys and values [n, Hkv, hd], and by key and KV head the largest of
    |m| + 15 s over its groups -> (out [Hq, hd], bound on a kernel's error).

    A score s (q . n) + m sum(q), in 32 bits, is off by (hd + 16) 2^-23 S where S = sum |q| kmax /
    sqrt(hd) bounds every term and partial sum of it (tensor cores may cut off where they add); such
    an error moves numerator and denominator.  Exponentials and 32-bit sums: 2^-18 of A = sum p vmax.
    Weights p s are held as two fp16 numbers, to 2^-22 of themselves or 2^-34 of the largest, where
    that is more.  The output is rounded to fp16: 2^-11 of it, or 2^-25."""
    Hq, hd = q.shape
    G = Hq // k.shape[1]
    k, v, kmax, vmax = (np.repeat(a, G, 1) for a in (k, v, kmax, vmax))
    z = np.einsum("hd,nhd->hn", q, k) / np.sqrt(hd)
    S = (np.abs(q).sum(1)[:, None] * kmax.T / np.sqrt(hd)).max(1)
    p = np.exp(z - z.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    out = np.einsum("hn,nhd->hd", p, v)
    A = (p * vmax.T).sum(1)[:, None]
    small = 2.0 ** -34 * (vmax.T * p.max(1, keepdims=True)).sum(1)[:, None]
    return out, A * (2.0 ** -18 + 2 * (hd + 16) * 2.0 ** -23 * S[:, None]) + small + 2.0 ** -11 * np.abs(out) + 2.0 ** -25


def select(z, scores, done, keep, eos, pad):
    """One group's step: logits [beams, V] (64-bit values of what is held), scores [beams], done [beams] ->
    (parents, tokens, scores, done)."""
    offers = []
    for b in range(len(z)):
        c = float(scores[b])
        if c == -np.inf:
            continue
        if done[b]:
            offers.append((-c, b, 0, pad))
            continue
        row = z[b].astype(np.float64)
        order = np.argsort(-row, kind="stable")[:keep]
        order = order[row[order] > -np.inf]
        if not len(order):
            continue
        top = row[order[0]]
        e = np.sort(np.exp(row - top))
        log = np.log(e.sum())  # (not added to the largest logit, in which it may be lost)
        offers += [(-(c + ((row[t] - top) - log)), b, i, int(t)) for i, t in enumerate(order)]
    offers.sort(key=lambda o: o[:3])
    out = [(b, t, -s, int(bool(done[b]) or t == eos)) for s, b, _, t in offers[:keep]]
    out += [(0, pad, -np.inf, 1)] * (keep - len(out))
    p, t, s, d = zip(*out)
    return np.array(p), np.array(t), np.array(s), np.array(d)


def logits_on_4_bits(m, prefix, text, generated):
    """Vocabulary logits [len(generated) + 1, V] of an oracle model for the steps that
    follow prefix ++ text, teacher-forced on `generated`, where a generated token attends
    the 4-bit cache, itself among it.  (Keys and values are rounded to fp16 first, as they
    are before they are quantised.)"""
    from oracle import transformer as tf
    s, n0 = m.s, len(prefix) + len(text)
    ids = np.concatenate([prefix, text, generated]).astype(np.int64)
    n, pos = len(ids), np.arange(len(ids))
    x = m.embed_rows(ids)
    for l in range(s.n_layers):
        w = {name: m.get(f"l{l}.{name}") for name in tf.LAYER_TENSORS}
        h = tf.rmsnorm(x, w["attn_norm"], s.rms_eps)
        q = tf.rope((h @ w["wq"].T).reshape(n, s.n_heads, s.head_dim), pos, s.rope_theta)
        k = tf.rope((h @ w["wk"].T).reshape(n, s.n_kv_heads, s.head_dim), pos, s.rope_theta)
        v = (h @ w["wv"].T).reshape(n, s.n_kv_heads, s.head_dim)
        a = np.zeros((n, s.n_heads, s.head_dim))
        a[:n0] = tf.causal_attention(q[:n0], k[:n0], v[:n0])
        held = values(*quantize(np.stack([k, v], 1).astype(np.float16)))
        one = np.ones(held.shape[:1] + held.shape[2:3])
        for i in range(n0, n):
            a[i], _ = attend(q[i], held[:i + 1, 0], held[:i + 1, 1], one[:i + 1], one[:i + 1])
        x = x + a.reshape(n, -1) @ w["wo"].T
        h = tf.rmsnorm(x, w["mlp_norm"], s.rms_eps)
        x = x + (tf.silu(h @ w["wg"].T) * (h @ w["wu"].T)) @ w["wd"].T
    h = tf.rmsnorm(x[n0 - 1:], m.get("final_norm"), s.rms_eps)
    return h @ tf.bf16_to_f64(m.w["lm_head"]).T + tf.bf16_to_f64(m.w["lm_bias"])
