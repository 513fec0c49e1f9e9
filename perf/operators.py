"""Performance cases of the generation step on an 8-bit key/value cache, through the Python binding.

Each case is one pass of a step-level operator (include/aiq_ops.h), at the sizes of
the repository's own workloads (the 1B- and 8B-shaped decoders, the tiny one) or
at sizes between them:

  quantize    a layer's keys and values into the 8-bit cache (a scale for each block of
              32 tokens, KV head and keys / values) and back: aiq_op_kv_quantize, aiq_op_kv_dequantize
  readback    a cache that is at hand back to fp16 rows: aiq_op_kv_dequantize
  attend      one layer's attention of a generation step over the 8-bit cache, the step's
              key and value appended to it: aiq_op_decode_attention_q8
  sample      the next token of each row from its logits and a given uniform number
              (temperature, top-k, top-p, min-p): aiq_op_sample

Where `own` is false each runs in its plain form, in elementary torch operations.
"""
import math
import zlib

import numpy as np
import torch

own = False

BLOCK = 32      # tokens that share a scale
GEN_CAP = 96    # generated tokens that a row's cache has room for


def listed():
    return [
        # one layer's prompt keys / values of a generation chunk, 1B shape, straight out of the QKV product's rows
        dict(name="quantize_1b_chunk", op="quantize", heads=32, kv=8, hd=64, rows=3263, median=120, cap=512),
        # the tiny workload's shared prefix: one short sequence of dense rows, where latency counts
        dict(name="quantize_tiny_prefix", op="quantize", heads=0, kv=4, hd=32, rows=1, median=16, cap=16),
        # the multi-label workload's rows on the 8B shape, for a kernel that takes fp16 rows
        dict(name="readback_8b", op="readback", heads=0, kv=8, hd=128, rows=1200, median=200, cap=1024),
        # an interactive query's rows, into the K / V columns of QKV rows
        dict(name="readback_1b_24", op="readback", heads=32, kv=8, hd=64, rows=24, median=120, cap=512),
        # one generation step of a decode batch (rows per chunk of the generation benchmark)
        dict(name="attend_1b_chunk", op="attend", heads=32, kv=8, hd=64, rows=3263, median=120, cap=512, prefix=64, slot=16),
        # the same on the 8B shape, the step that completes a block of generated tokens
        dict(name="attend_8b_block", op="attend", heads=32, kv=8, hd=128, rows=700, median=200, cap=1024, prefix=128, slot=63),
        # a few long documents: few rows, many keys
        dict(name="attend_8b_long", op="attend", heads=32, kv=8, hd=128, rows=4, median=30000, cap=65536, prefix=0, slot=5),
        # an interactive query: a handful of rows
        dict(name="attend_1b_24", op="attend", heads=32, kv=8, hd=64, rows=24, median=120, cap=512, prefix=64, slot=7),
        # the tiny shape, the first generated token of one row
        dict(name="attend_tiny_1", op="attend", heads=4, kv=4, hd=32, rows=1, median=32, cap=48, prefix=16, slot=0),
        # the next token of every row of a decode batch, usual settings
        dict(name="sample_1b_chunk", op="sample", rows=3263, vocab=32000, type="f32", temperature=0.8, top_k=50,
             top_p=0.95, min_p=0.0, banned=0.0),
        # a handful of rows over the 8B shape's vocabulary, a wide candidate set, some tokens ruled out
        dict(name="sample_8b_24", op="sample", rows=24, vocab=128256, type="f16", temperature=1.3, top_k=1000, top_p=0.9,
             min_p=0.02, banned=0.01),
        # one row of the tiny vocabulary
        dict(name="sample_tiny_1", op="sample", rows=1, vocab=4096, type="f32", temperature=1.0, top_k=40, top_p=1.0,
             min_p=0.05, banned=0.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "readback", "attend", "attend", "sample", "sample"])
    if op == "sample":
        vocab = _log(rng, 1000, 128256)
        return dict(op=op, rows=_log(rng, 1, min(4096, 104_000_000 // vocab)), vocab=vocab,
                    type=rng.choice(["f32", "f16", "bf16"]), temperature=round(rng.uniform(0.3, 2.0), 3),
                    top_k=_log(rng, 1, min(1024, vocab)), top_p=rng.choice([1.0, round(rng.uniform(0.3, 0.99), 3)]),
                    min_p=rng.choice([0.0, round(rng.uniform(0.005, 0.3), 4)]), banned=rng.choice([0.0, 0.02]))
    heads, kv, hd = rng.choice([(32, 8, 64), (32, 8, 128), (8, 2, 64), (4, 4, 32), (16, 2, 128), (12, 4, 64)])
    median = _log(rng, 8, 20000)
    cap = max(64, 4 * median)
    # at most as many cached values as the largest listed cases have
    rows = _log(rng, 1, max(1, min(3263, 400_000_000 // (median * 2 * kv * hd))))
    case = dict(op=op, heads=heads, kv=kv, hd=hd, rows=rows, median=median, cap=cap)
    if op == "attend":
        return dict(case, prefix=rng.choice([0, 16, 64, 70, 128]), slot=rng.randint(0, GEN_CAP - 1))
    return dict(case, heads=rng.choice([0, heads]))


# ------------------------------------------------------------------ inputs ---

def _rng(case, seed):
    text = repr(sorted((k, v) for k, v in case.items() if k != "name"))
    return np.random.Generator(np.random.PCG64([int(seed) & 0xFFFFFFFF, zlib.crc32(text.encode())]))


def _lens(case):
    """Text lengths of the workloads: lognormal, sigma 0.5.  The same lengths for
    every seed; prepare() shuffles them."""
    if case["rows"] == 1 and case["median"] == case["cap"]:
        return np.full(1, case["cap"], np.int64)
    x = np.exp(_rng(case, 0).normal(math.log(case["median"]), 0.5, case["rows"]))
    return np.clip(np.rint(x), 1, case["cap"]).astype(np.int64)


class State:
    """What a program has in hand before a call."""


def _normal(g, shape, std=0.9):
    # keys and values of a 0.02-initialised projection of a normalised 2048-wide row: std 0.9
    out = torch.empty(shape, dtype=torch.float16, device="cuda")
    flat, step = out.view(-1), 1 << 26
    for i in range(0, flat.numel(), step):
        n = min(step, flat.numel() - i)
        flat[i:i + n] = torch.empty(n, device="cuda").normal_(0, std, generator=g)
    return out


def _slots(starts, lens):
    """Where the tokens of packed sequences lie in the cache: sequence r's blocks begin
    at block starts[r] // BLOCK + r.  (block, place in it) of every token, and the blocks."""
    n = len(lens)
    seq = torch.repeat_interleave(torch.arange(n, device="cuda"), lens)
    at = torch.arange(int(lens.sum()), device="cuda") - starts[seq]
    return starts[seq] // BLOCK + seq + at // BLOCK, at % BLOCK, int(lens.sum()) // BLOCK + n


def _quantize(blocks, dtype):
    """Blocks [nb, BLOCK, 2, KV, hd] to whole numbers -127 .. 127 (halves away from
    zero) and scales [nb, KV, 2] = the largest magnitude / 127."""
    x = blocks.to(dtype)
    a = x.abs().amax((1, 4), keepdim=True)
    q = torch.sign(x) * torch.floor(x.abs() * 127 / torch.where(a > 0, a, 1) + 0.5)
    return q, (a / 127)[:, 0, :, :, 0].transpose(1, 2)


def _tiles(q):
    """Whole numbers [nb, BLOCK, 2, KV, hd] (int8) in the cache's own order: per block
    and KV head the keys' and then the values' bytes, each + 128, as include/aiq_ops.h
    lays them out."""
    nb, _, _, kv, hd = q.shape
    u = (q.to(torch.int16) + 128).to(torch.uint8)
    k, v = u[:, :, 0], u[:, :, 1]
    if hd == 32:
        k = k.reshape(nb, 2, 2, 8, kv, 4, 8).permute(0, 4, 1, 3, 5, 2, 6)
    else:
        k = k.reshape(nb, 4, 8, kv, hd // 64, 4, 16).permute(0, 3, 1, 4, 2, 5, 6)
    v = v.reshape(nb, 2, 2, 4, 2, kv, hd // 32, 4, 4, 2).permute(0, 5, 1, 6, 7, 9, 3, 8, 2, 4)
    return torch.cat([k.reshape(nb, kv, -1), v.reshape(nb, kv, -1)], 2).contiguous()


def _cache(kv_rows, block, place, nb, KV, hd):
    """The quantised cache of fp16 rows: whole numbers by token, scales, tiles."""
    x = torch.zeros((nb, BLOCK, 2, KV, hd), dtype=torch.float16, device="cuda")
    x[block, place] = kv_rows.view(-1, 2, KV, hd)
    q, s = _quantize(x, torch.float32)
    q = q.to(torch.int8)
    return q[block, place].contiguous(), s.contiguous(), _tiles(q)


def prepare(case, seed):
    rng, st = _rng(case, seed), State()
    g = torch.Generator(device="cuda")
    g.manual_seed(int(rng.integers(0, 2 ** 62)))
    st.case = dict(case)
    if case["op"] == "sample":
        R, V = case["rows"], case["vocab"]
        t = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[case["type"]]
        # rows from almost flat to peaked
        std = torch.empty(R, 1, device="cuda").uniform_(0.7, 4.0, generator=g)
        z = torch.empty(R, V, device="cuda").normal_(0, 1, generator=g) * std
        if case["banned"]:
            z[torch.empty(R, V, device="cuda").uniform_(0, 1, generator=g) < case["banned"]] = -math.inf
        st.logits = z.to(t)
        st.u = torch.empty(R, device="cuda").uniform_(0, 1, generator=g).clamp_(max=1 - 2.0 ** -24)
        st.tokens = torch.zeros(R, dtype=torch.int32, device="cuda")
        st.probs = torch.zeros(R, device="cuda")
        torch.cuda.synchronize()
        return st
    H, KV, hd, R = case["heads"], case["kv"], case["hd"], case["rows"]
    kd = KV * hd
    st.lens = torch.from_numpy(rng.permutation(_lens(case))).cuda()
    st.T = int(st.lens.sum())
    st.starts = torch.zeros(R + 1, dtype=torch.int64, device="cuda")
    st.starts[1:] = st.lens.cumsum(0)
    st.seq = st.starts.int()
    st.block, st.place, st.nb = _slots(st.starts[:-1], st.lens)
    st.kv = _normal(g, (st.T, (H + 2 * KV) * hd if case["op"] == "quantize" else 2 * kd))
    if case["op"] == "quantize":
        st.cache = torch.full((st.nb, KV, BLOCK * 2 * hd), 128, dtype=torch.uint8, device="cuda")
        st.scales = torch.zeros((st.nb, KV, 2), device="cuda")
        st.back = torch.zeros((st.T, 2 * kd), dtype=torch.float16, device="cuda")
    elif case["op"] == "readback":
        st.q, st.scales, st.cache = _cache(st.kv, st.block, st.place, st.nb, KV, hd)
        st.kv = None
        st.back = torch.zeros((st.T, (H + 2 * KV) * hd), dtype=torch.float16, device="cuda")
    else:
        P, one = case["prefix"], torch.tensor([0], device="cuda")
        st.q, st.scales, st.cache = _cache(st.kv, st.block, st.place, st.nb, KV, hd)
        st.kv = None
        b, p, n = _slots(one, one + max(P, 1))
        st.pq, st.pscales, st.pcache = _cache(_normal(g, (max(P, 1), 2 * kd)), b, p, n, KV, hd)
        st.pblock = b
        G = GEN_CAP // BLOCK
        x = _normal(g, (R * G, BLOCK, 2, KV, hd))
        q, s = _quantize(x, torch.float32)
        st.gcache = _tiles(q.to(torch.int8))
        st.gq, st.gscales = q.to(torch.int8).view(R, GEN_CAP, 2, KV, hd), s.contiguous()
        st.gseq = torch.tensor([0, R * GEN_CAP], dtype=torch.int32, device="cuda")
        st.tail = _normal(g, (R, BLOCK, 2 * kd))
        st.qkv = _normal(g, (R, (H + 2 * KV) * hd))
        st.out = torch.zeros((R, H * hd), dtype=torch.float16, device="cuda")
        st.back = torch.zeros((R * GEN_CAP, 2 * kd), dtype=torch.float16, device="cuda")
    torch.cuda.synchronize()
    return st


# ------------------------------------------------------------- plain forms ---

def _plain_quantize(st):
    c = st.case
    KV, hd = c["kv"], c["hd"]
    x = torch.zeros((st.nb, BLOCK, 2, KV, hd), device="cuda")
    x[st.block, st.place] = st.kv[:, c["heads"] * hd:].reshape(-1, 2, KV, hd).float()
    q, s = _quantize(x, torch.float32)
    values = q[st.block, st.place] * s[st.block].transpose(1, 2)[..., None]
    return {"values": values.half().view(st.T, -1), "scales": s}


def _plain_readback(st):
    c = st.case
    values = st.q.float() * st.scales[st.block].transpose(1, 2)[..., None]
    st.back[:, c["heads"] * c["hd"]:] = values.half().view(st.T, -1)
    return {"rows": st.back}


def _plain_attend(st):
    c = st.case
    H, KV, hd, R, P, slot = c["heads"], c["kv"], c["hd"], c["rows"], c["prefix"], c["slot"]
    kd, open_, full = KV * hd, slot % BLOCK, slot // BLOCK * BLOCK
    st.tail[:, open_] = st.qkv[:, H * hd:]
    q = st.qkv[:, :H * hd].float().view(R, KV, H // KV, hd) / math.sqrt(hd)
    # the shared prefix
    pk, pv = (st.pq.float() * st.pscales[st.pblock].transpose(1, 2)[..., None])[:P].unbind(1)
    # every row's own tokens, padded to the longest
    j = torch.arange(int(st.lens.max()), device="cuda")
    at = (st.starts[:-1, None] + j).clamp(max=st.T - 1)
    ok, ov = (st.q[at].float() * st.scales[st.block[at]].transpose(2, 3)[..., None]).unbind(2)
    # generated tokens: whole blocks of 8 bits, then the open block's
    gs = st.gscales.view(R, -1, 1, KV, 2).transpose(3, 4).expand(R, -1, BLOCK, 2, KV).reshape(R, GEN_CAP, 2, KV, 1)
    gk, gv = (st.gq[:, :full].float() * gs[:, :full]).unbind(2)
    tk, tv = st.tail[:, :open_ + 1].float().view(R, -1, 2, KV, hd).unbind(2)
    z = torch.cat([torch.einsum("rhgd,lhd->rhgl", q, pk),
                   torch.einsum("rhgd,rlhd->rhgl", q, ok).masked_fill((j >= st.lens[:, None])[:, None, None], -math.inf),
                   torch.einsum("rhgd,rlhd->rhgl", q, gk), torch.einsum("rhgd,rlhd->rhgl", q, tk)], -1)
    p = (z - z.amax(-1, keepdim=True)).exp()
    p = p / p.sum(-1, keepdim=True)
    a, b, d = P, P + len(j), P + len(j) + full
    o = (torch.einsum("rhgl,lhd->rhgd", p[..., :a], pv) + torch.einsum("rhgl,rlhd->rhgd", p[..., a:b], ov)
         + torch.einsum("rhgl,rlhd->rhgd", p[..., b:d], gv) + torch.einsum("rhgl,rlhd->rhgd", p[..., d:], tv))
    out = {"out": o.reshape(R, H * hd).half(), "appended": st.tail[:, open_]}
    if open_ == BLOCK - 1:
        w, s = _quantize(st.tail.view(R, BLOCK, 2, KV, hd), torch.float32)
        out["block"] = (w * s.transpose(1, 2)[:, None, ..., None]).half().view(R, BLOCK, 2 * kd)
        out["block_scales"] = s
    return out


def _plain_sample(st):
    c = st.case
    z, order = st.logits.float().sort(dim=1, descending=True, stable=True)
    z, order = z[:, :c["top_k"]].double(), order[:, :c["top_k"]]
    e = ((z - z[:, :1]) / c["temperature"]).exp()
    total = e.cumsum(1)
    n = (e >= c["min_p"]).sum(1)
    if c["top_p"] < 1:
        n = torch.minimum(n, 1 + (total < c["top_p"] * total[:, -1:]).sum(1))
    kept = total.gather(1, n[:, None] - 1)
    i = (total <= st.u.double()[:, None] * kept).sum(1, keepdim=True)
    return {"tokens": order.gather(1, i)[:, 0].int(), "probs": (e.gather(1, i) / kept)[:, 0].float()}


# ---------------------------------------------------------------- own calls ---

_kept = {}  # the context that a program keeps for its whole life


def _aiq():
    if not _kept:
        from paper_2608_10139_gb300 import aiq
        _kept.update(aiq=aiq, ctx=aiq.Context(0))
    return _kept["aiq"], _kept["ctx"]


def _own(st):
    aiq, ctx = _aiq()
    c = st.case
    if c["op"] == "sample":
        t = {"f32": aiq.LOGITS_F32, "f16": aiq.LOGITS_F16, "bf16": aiq.LOGITS_BF16}[c["type"]]
        ctx.op_sample(st.logits.data_ptr(), t, c["vocab"], c["rows"], c["vocab"], st.u.data_ptr(), st.tokens.data_ptr(),
                      temperature=c["temperature"], top_k=c["top_k"], top_p=c["top_p"], min_p=c["min_p"],
                      probs=st.probs.data_ptr())
        return {"tokens": st.tokens, "probs": st.probs}
    H, KV, hd, R = c["heads"], c["kv"], c["hd"], c["rows"]
    kd = KV * hd
    if c["op"] == "quantize":
        ctx.op_kv_quantize(st.kv.data_ptr() + 2 * H * hd, st.kv.shape[1], st.T, st.seq.data_ptr(), R, KV, hd,
                           st.cache.data_ptr(), st.scales.data_ptr())
        ctx.op_kv_dequantize(st.cache.data_ptr(), st.scales.data_ptr(), st.T, st.seq.data_ptr(), R, KV, hd,
                             st.back.data_ptr(), 2 * kd)
        return {"values": st.back, "scales": st.scales}
    if c["op"] == "readback":
        ctx.op_kv_dequantize(st.cache.data_ptr(), st.scales.data_ptr(), st.T, st.seq.data_ptr(), R, KV, hd,
                             st.back.data_ptr() + 2 * H * hd, st.back.shape[1])
        return {"rows": st.back}
    P, slot = c["prefix"], c["slot"]
    ctx.op_decode_attention_q8(st.qkv.data_ptr(), R, H, KV, hd, st.cache.data_ptr(), st.scales.data_ptr(), st.T,
                               st.seq.data_ptr(), st.gcache.data_ptr(), st.gscales.data_ptr(), st.tail.data_ptr(),
                               GEN_CAP, slot, st.out.data_ptr(), prefix=st.pcache.data_ptr() if P else 0,
                               prefix_scales=st.pscales.data_ptr() if P else 0, P=P)
    out = {"out": st.out, "appended": st.tail[:, slot % BLOCK]}
    if slot % BLOCK == BLOCK - 1:
        # the generated tokens' cache is one sequence of whole blocks
        ctx.op_kv_dequantize(st.gcache.data_ptr(), st.gscales.data_ptr(), R * GEN_CAP, st.gseq.data_ptr(), 1, KV, hd,
                             st.back.data_ptr(), 2 * kd)
        b = slot // BLOCK
        out["block"] = st.back.view(R, GEN_CAP, 2 * kd)[:, b * BLOCK:(b + 1) * BLOCK]
        out["block_scales"] = st.gscales.view(R, -1, KV, 2)[:, b]
    return out


def run(state):
    if own:
        return _own(state)
    return {"quantize": _plain_quantize, "readback": _plain_readback, "attend": _plain_attend,
            "sample": _plain_sample}[state.case["op"]](state)


# -------------------------------------------------------------------- work ---

def work(case):
    if case["op"] == "sample":
        size = 4 if case["type"] == "f32" else 2
        return {"bytes": case["rows"] * (case["vocab"] * size + 12), "flops": 0}
    width = 2 * case["kv"] * case["hd"]  # values of a token
    lens = _lens(case).astype(np.float64)
    T, R = float(lens.sum()), case["rows"]
    scales = width / case["hd"] * 4 / BLOCK  # bytes a token
    if case["op"] == "quantize":  # fp16 in, the cache and the values that it stands for out
        return {"bytes": T * (width * 5 + scales), "flops": 0}
    if case["op"] == "readback":
        return {"bytes": T * (width * 3 + scales), "flops": 0}
    H, hd, P, slot = case["heads"], case["hd"], case["prefix"], case["slot"]
    open_, full = slot % BLOCK, slot // BLOCK * BLOCK
    keys = T + P + R * full
    flops = 4.0 * H * hd * (T + R * (P + slot + 1))
    n = keys * (width + scales) + R * (open_ * width * 2 + H * hd * 4 + width * 4)
    if open_ == BLOCK - 1:  # the block, and the values that the generated cache stands for
        n += R * (BLOCK * (width + scales) + GEN_CAP * (width * 3 + scales))
    return {"bytes": n, "flops": flops}


# ------------------------------------------------------- the same in 64 bits ---

def _exact_blocks(rows, lens, KV, hd):
    """By sequence and block: [nb_used] lists of (values, scales) in 64 bits."""
    out, scales, at = [], [], 0
    for n in lens:
        x = rows[at:at + n].double().view(n, 2, KV, hd)
        x = torch.nn.functional.pad(x, (0, 0, 0, 0, 0, 0, 0, -n % BLOCK)).view(-1, BLOCK, 2, KV, hd)
        s = x.abs().amax((1, 4)) / 127
        w = x / s.clamp(min=1e-300)[:, None, :, :, None]
        # w + 1/2 away from zero, where it is a half to within its own rounding
        w = w.sign() * (w.abs() + (0.5 + 1e-9)).floor()
        out.append((w * s[:, None, :, :, None]).view(-1, 2 * KV * hd)[:n])
        scales.append(s.transpose(1, 2))
        at += n
    return out, scales


def _exact_attend(st):
    c = st.case
    H, KV, hd, P, slot = c["heads"], c["kv"], c["hd"], c["prefix"], c["slot"]
    G, open_, full = H // KV, slot % BLOCK, slot // BLOCK * BLOCK

    def values(q, s, block):
        return q.double() * s.double()[block].transpose(-1, -2)[..., None]

    gen_block = torch.arange(full, device="cuda") // BLOCK
    gs, starts = st.gscales.view(c["rows"], -1, KV, 2), st.starts.tolist()
    prefix, out = values(st.pq, st.pscales, st.pblock)[:P], []
    for r in range(c["rows"]):
        a, b = starts[r], starts[r + 1]
        new = st.qkv[r].double()
        rows = torch.cat([prefix, values(st.q[a:b], st.scales, st.block[a:b]), values(st.gq[r, :full], gs[r], gen_block),
                          st.tail[r, :open_].double().view(-1, 2, KV, hd), new[H * hd:].view(1, 2, KV, hd)])
        k, v = rows.unbind(1)
        z = torch.matmul(new[:H * hd].view(KV, G, hd), k.permute(1, 2, 0)) * hd ** -0.5
        out.append(torch.matmul(torch.softmax(z, -1), v.transpose(0, 1)).reshape(-1))
    res = {"out": torch.stack(out), "appended": None}
    if open_ == BLOCK - 1:
        rows = torch.cat([st.tail[:, :open_], st.qkv[:, None, H * hd:]], 1)
        w, s = _exact_blocks(rows.reshape(-1, 2 * KV * hd), [rows.shape[0] * BLOCK], KV, hd)
        res.update(block=w[0].view(rows.shape), block_scales=s[0])
    return res


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "sample":
        z, _ = st.logits.double().topk(case["top_k"], dim=1)
        p = torch.softmax(z / case["temperature"], 1)
        below = p.cumsum(1) - p
        keep = p >= case["min_p"] * p[:, :1]
        if case["top_p"] < 1:
            keep &= below < case["top_p"]
        p = torch.where(keep, p, 0)
        p = p / p.sum(1, keepdim=True)
        # the draw's place among the kept ones does not depend on how equal logits are ordered
        i = (p.cumsum(1) <= st.u.double()[:, None]).sum(1, keepdim=True).clamp(max=case["top_k"] - 1)
        return {"tokens": None, "probs": p.gather(1, i)[:, 0]}
    KV, hd = case["kv"], case["hd"]
    if case["op"] == "quantize":
        w, s = _exact_blocks(st.kv[:, case["heads"] * hd:], st.lens.tolist(), KV, hd)
        scales = torch.zeros((st.nb, KV, 2), dtype=torch.float64, device="cuda")
        first = (st.starts[:-1] // BLOCK).tolist()
        for r, x in enumerate(s):
            scales[first[r] + r:first[r] + r + len(x)] = x
        return {"values": torch.cat(w), "scales": scales}
    if case["op"] == "readback":
        rows = torch.zeros(st.back.shape, dtype=torch.float64, device="cuda")
        rows[:, case["heads"] * hd:] = (st.q.double() * st.scales.double()[st.block].transpose(1, 2)[..., None]).flatten(1)
        return {"rows": rows}
    return _exact_attend(st)
