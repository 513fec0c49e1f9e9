"""The 8-bit key/value cache, its attention and the sampling of a token, plainly
in 64 bits (numpy), from the definitions in include/aiq.h and include/aiq_ops.h."""
import numpy as np

BLOCK = 32


def first_block(start, seq):
    return start // BLOCK + seq


def blocks(T, n):
    return T // BLOCK + n


def starts(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def quantize(x):
    """x [BLOCK, hd] fp16 values -> whole numbers (halves away from zero) and the fp32 scale."""
    x = x.astype(np.float64)
    a = np.abs(x).max() if x.size else 0.0
    # 127 * x is exact; of two fp16 numbers the quotient is a half exactly, where 64 bits hold
    # it exactly too, or further from one than any rounding here
    q = np.sign(x) * np.floor(np.abs(x) * 127 / a + 0.5) if a else np.zeros_like(x)
    return q.astype(np.int64), np.float32(np.float32(a) / np.float32(127))


def tile(qk, qv):
    """A block's whole numbers, keys and values [BLOCK, hd], as the cache's bytes."""
    hd = qk.shape[1]
    out = np.zeros(2 * BLOCK * hd, np.uint8)
    for key in range(BLOCK):
        for d in range(hd):
            out[key_at(hd, key, d)] = qk[key, d] + 128
            out[value_at(hd, key, d)] = qv[key, d] + 128
    return out


def key_at(hd, key, d):
    g = key % 8
    if hd == 32:
        return ((key // 16 * 8 + g) * 4 + d // 8) * 16 + key // 8 % 2 * 8 + d % 8
    return (((key // 8 * (hd // 64) + d // 64) * 8 + g) * 4 + d % 64 // 16) * 16 + d % 16


def value_at(hd, key, d):
    k, jj, t, e = key // 16, key // 8 % 2, key % 8 // 2, key % 2
    c, gh, i, gl = d // 32, d % 32 // 8, d % 8 // 2, d % 2
    return BLOCK * hd + (((k * (hd // 32) + c) * 8 + gh * 2 + gl) * 4 + t) * 16 + i * 4 + jj * 2 + e


_MAPS = {}


def tile_maps(hd):
    """Positions of (keys, values) [BLOCK, hd] in a tile."""
    if hd not in _MAPS:
        k = np.array([[key_at(hd, j, d) for d in range(hd)] for j in range(BLOCK)])
        v = np.array([[value_at(hd, j, d) for d in range(hd)] for j in range(BLOCK)])
        _MAPS[hd] = k, v
    return _MAPS[hd]


def build_cache(rows, lens, Hkv, hd, T=None, fill=0):
    """fp16 rows [T, 2 Hkv hd] of packed sequences -> (cache, scales, whole numbers [T, 2, Hkv, hd],
    scale of every token [T, 2, Hkv])."""
    n, T = len(lens), len(rows) if T is None else T
    st, nb = starts(lens), blocks(T, n)
    cache = np.full((nb, Hkv, 2 * BLOCK * hd), fill, np.uint8)
    scales = np.full((nb, Hkv, 2), np.float32(fill), np.float32)
    x = np.asarray(rows, np.float16).reshape(len(rows), 2, Hkv, hd)
    q_all = np.zeros((len(rows), 2, Hkv, hd))
    s_all = np.zeros((len(rows), 2, Hkv))
    mk, mv = tile_maps(hd)
    for r in range(n):
        for j in range(-(-int(lens[r]) // BLOCK)):
            a = int(st[r]) + j * BLOCK
            m = min(BLOCK, int(st[r + 1]) - a)
            b = first_block(int(st[r]), r) + j
            for h in range(Hkv):
                for c, at in ((0, mk), (1, mv)):
                    blk = np.zeros((BLOCK, hd), np.float16)
                    blk[:m] = x[a:a + m, c, h]
                    q, s = quantize(blk)
                    cache[b, h, at] = q + 128
                    scales[b, h, c] = s
                    q_all[a:a + m, c, h] = q[:m]
                    s_all[a:a + m, c, h] = s
    return cache, scales, q_all, s_all


def read_back(q, s):
    """fp16 rows [T, 2 Hkv hd] of whole numbers and their scales: one product in 32 bits, rounded to fp16."""
    v = q.astype(np.float32) * s.astype(np.float32)[..., None]
    return v.astype(np.float16).reshape(len(q), int(np.prod(q.shape[1:])))


def attend(q, k, v):
    """q [Hq, hd], k / v [n, Hkv, hd] -> (out [Hq, hd], bound on a kernel's error).

    The bound counts a kernel that takes scores in 32 bits, holds a block's
    probabilities in fp16 relative to the block's largest, and rounds the output to
    fp16 once: a probability is off by 2^-11 of itself (2^-25 of the block's largest
    where that is more), so that the output moves by as much of A = sum p |v|; a score
    is off by (hd + 8) 2^-23 S, S = sum |q k| / sqrt(hd) (tensor cores may cut off
    where they add), which moves numerator and denominator; 2^-18 A for the 32-bit
    exponentials and sums; the output's own 2^-11."""
    Hq, hd = q.shape
    G = Hq // k.shape[1]
    k, v = np.repeat(k, G, 1), np.repeat(v, G, 1)
    z = np.einsum("hd,nhd->hn", q, k) / np.sqrt(hd)
    S = (np.einsum("hd,nhd->hn", np.abs(q), np.abs(k)) / np.sqrt(hd)).max(1)
    p = np.exp(z - z.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    out = np.einsum("hn,nhd->hd", p, v)
    A = np.einsum("hn,nhd->hd", p, np.abs(v))
    small = 2.0 ** -25 * np.abs(v).sum(0) * p.max(1)[:, None]
    rel = 2.0 ** -11 + 2.0 ** -18 + 2 * (hd + 8) * 2.0 ** -23 * S[:, None]
    return out, A * rel + small + 2.0 ** -11 * np.abs(out) + 2.0 ** -25


def sample(z, u, temperature, top_k, top_p, min_p):
    """(token, probability) of one row of logits (exact in 32 bits) for the uniform u."""
    z = z.astype(np.float64)
    order = np.argsort(-z, kind="stable")[:top_k]
    with np.errstate(over="ignore"):  # a difference divided by next to nothing
        e = np.exp((z[order] - z[order[0]]) / temperature)
    c = np.cumsum(e)
    n = int((e >= min_p).sum())
    if top_p < 1:
        n = min(n, 1 + int((c < top_p * c[-1]).sum()))
    i = min(n - 1, int((c[:n] <= float(np.float32(u)) * c[n - 1]).sum()))
    return int(order[i]), e[i] / c[n - 1]


def logits_on_8_bits(m, prefix, text, generated):
    """Vocabulary logits [len(generated) + 1, V] of an oracle model for the steps that
    follow prefix ++ text, teacher-forced on `generated`, where generated tokens attend
    the 8-bit cache: prefix and text quantised block by block, earlier tokens in
    whole blocks too, the open block as it is.  (Keys and values are rounded to fp16
    first, as they are stored before they are quantised.)"""
    from oracle import transformer as tf
    s, n0 = m.s, len(prefix) + len(text)
    ids = np.concatenate([prefix, text, generated]).astype(np.int64)
    n, pos = len(ids), np.arange(len(ids))
    x = m.embed_rows(ids)
    kd = s.n_kv_heads * s.head_dim

    def held(rows):  # whole sequences, as the cache holds them
        if len(rows) == 0:
            return np.zeros((0, 2, s.n_kv_heads, s.head_dim))
        _, _, q, sc = build_cache(rows.reshape(len(rows), 2 * kd).astype(np.float16), [len(rows)], s.n_kv_heads, s.head_dim)
        return q * sc[..., None]

    for l in range(s.n_layers):
        w = {name: m.get(f"l{l}.{name}") for name in tf.LAYER_TENSORS}
        h = tf.rmsnorm(x, w["attn_norm"], s.rms_eps)
        q = tf.rope((h @ w["wq"].T).reshape(n, s.n_heads, s.head_dim), pos, s.rope_theta)
        k = tf.rope((h @ w["wk"].T).reshape(n, s.n_kv_heads, s.head_dim), pos, s.rope_theta)
        v = (h @ w["wv"].T).reshape(n, s.n_kv_heads, s.head_dim)
        a = np.zeros((n, s.n_heads, s.head_dim))
        a[:n0] = tf.causal_attention(q[:n0], k[:n0], v[:n0])
        kv = np.stack([k, v], 1)
        prompt = np.concatenate([held(kv[:len(prefix)]), held(kv[len(prefix):n0])])
        for i in range(n0, n):
            whole = n0 + (i - n0) // BLOCK * BLOCK
            see = np.concatenate([prompt, held(kv[n0:whole]), kv[whole:i + 1]])
            a[i], _ = attend(q[i], see[:, 0], see[:, 1])
        x = x + a.reshape(n, -1) @ w["wo"].T
        h = tf.rmsnorm(x, w["mlp_norm"], s.rms_eps)
        x = x + (tf.silu(h @ w["wg"].T) * (h @ w["wu"].T)) @ w["wd"].T
    h = tf.rmsnorm(x[n0 - 1:], m.get("final_norm"), s.rms_eps)
    return h @ tf.bf16_to_f64(m.w["lm_head"]).T + tf.bf16_to_f64(m.w["lm_bias"])
