"""Performance cases of generation on a 4-bit key/value cache and of beam search, through the Python binding.

Each case is one pass of a step-level operator (include/aiq_ops.h), at the sizes of
the repository's own workloads (the 1B- and 8B-shaped decoders, the tiny one) or
at sizes between them:

  quantize    a layer's keys and values into the 4-bit cache (a scale and a smallest value for each
              token, KV head, keys / values and at most 64 elements) and back: aiq_op_kv_quantize4, aiq_op_kv_dequantize4
  readback    a cache that is at hand back to fp16 rows: aiq_op_kv_dequantize4
  attend      one layer's attention of a generation step over the 4-bit cache, which takes the
              step's key and value; a sequence's beams share its prompt: aiq_op_decode_attention_q4
  select      the next beams of each sequence from its beams' logits and scores: aiq_op_beam_select
  reorder     the beams' state by their parents, every layer's rows at once: aiq_op_beam_reorder

Where `own` is false each runs in its plain form, in elementary torch operations.
"""
import math
import zlib

import numpy as np
import torch

own = False

BLOCK = 32      # tokens of a tile
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
        dict(name="attend_1b_chunk", op="attend", heads=32, kv=8, hd=64, rows=3263, beams=1, median=120, cap=512,
             prefix=64, slot=16),
        # beam search on the 8B shape, four beams a text, into the third block of generated tokens
        dict(name="attend_8b_beams", op="attend", heads=32, kv=8, hd=128, rows=175, beams=4, median=200, cap=1024,
             prefix=128, slot=64),
        # a few long documents: few rows, many keys
        dict(name="attend_8b_long", op="attend", heads=32, kv=8, hd=128, rows=4, beams=1, median=30000, cap=65536,
             prefix=0, slot=5),
        # the tiny shape, the first generated token of one row
        dict(name="attend_tiny_1", op="attend", heads=4, kv=4, hd=32, rows=1, beams=1, median=32, cap=48, prefix=16,
             slot=0),
        # the next beams of a decode batch's texts, 1B shape
        dict(name="select_1b_chunk", op="select", rows=800, beams=4, keep=4, vocab=32000, type="f32", banned=0.0),
        # one text over the 8B shape's vocabulary, twice as many continuations as beams, some tokens ruled out
        dict(name="select_8b_1", op="select", rows=1, beams=8, keep=16, vocab=128256, type="f16", banned=0.01),
        # 37 generated tokens of every layer of the 1B shape's 4-bit cache: two blocks of the three that a row has room for
        dict(name="reorder_1b_chunk", op="reorder", layers=16, rows=300, beams=4, bytes=36864, pitch=55296, inplace=True),
        # the tokens so far of one text's beams
        dict(name="reorder_tokens_8", op="reorder", layers=1, rows=1, beams=8, bytes=148, pitch=384, inplace=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "readback", "attend", "attend", "attend", "select", "select", "reorder"])
    if op == "select":
        vocab, beams = _log(rng, 1000, 128256), rng.choice([1, 2, 3, 4, 5, 8, 16])
        return dict(op=op, rows=_log(rng, 1, min(1024, max(1, 100_000_000 // (vocab * beams)))), beams=beams,
                    keep=rng.choice([beams, 2 * beams]), vocab=vocab, type=rng.choice(["f32", "f16", "bf16"]),
                    banned=rng.choice([0.0, 0.02]))
    if op == "reorder":
        beams, layers = rng.choice([2, 3, 4, 5, 8, 16]), rng.choice([1, 2, 16, 32])
        unit = rng.choice([1, 4, 16, 16])  # bytes that rows, pitch and size are multiples of
        size = unit * _log(rng, 8, 4096)
        rows = _log(rng, 1, max(1, min(1000, 900_000_000 // (layers * beams * size))))
        return dict(op=op, layers=layers, rows=rows, beams=beams, bytes=size,
                    pitch=size + unit * rng.choice([0, 1, 7, 16]), inplace=rng.random() < 0.5)
    heads, kv, hd = rng.choice([(32, 8, 64), (32, 8, 128), (8, 2, 64), (4, 4, 32), (16, 2, 128), (12, 4, 64)])
    median = _log(rng, 8, 20000)
    cap = max(64, 4 * median)
    # at most as many cached values as the largest listed cases have
    rows = _log(rng, 1, max(1, min(3263, 400_000_000 // (median * 2 * kv * hd))))
    case = dict(op=op, heads=heads, kv=kv, hd=hd, rows=rows, median=median, cap=cap)
    if op == "attend":
        beams = rng.choice([1, 1, 2, 3, 4, 5, 8])
        return dict(case, rows=max(1, rows // beams), beams=beams, prefix=rng.choice([0, 16, 64, 70, 128]),
                    slot=rng.randint(0, GEN_CAP - 1))
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


def _parents(case):
    """The beams' parents [rows, beams], the same for every seed; prepare() shuffles the rows.
    Few hypotheses survive a step, the better ones with more descendants.  In place, those that
    survive keep their places and the others take copies of them."""
    rng, n, b = _rng(case, 0), case["rows"], case["beams"]
    w = np.exp(rng.normal(0, 1, (n, b)))
    p = (rng.random((n, b, 1)) > (w / w.sum(1, keepdims=True)).cumsum(1)[:, None]).sum(2)
    p = np.minimum(p, b - 1)
    if case["inplace"]:
        lives = np.zeros((n, b), bool)
        lives[np.arange(n)[:, None], p] = True
        p = np.where(lives, np.arange(b), p)
    return p.astype(np.int32)


def _hypotheses(case):
    """Which of the beams [rows, beams] have ended, and which places hold none (score -infinity): the
    same for every seed; prepare() shuffles the rows."""
    rng, shape = _rng(case, 0), (case["rows"], case["beams"])
    done, none = rng.random(shape) < 0.05, rng.random(shape) < 0.02
    none[:, 0] = done[:, 0] = False
    return done, none


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


def _quantize(x):
    """fp16 values [.., hd] to whole numbers 0 .. 15 (uint8) and, per at most 64 of them, the
    scale (their range / 15, rounded up to fp16) and the smallest.  In 64 bits: a value may lie
    next to the border between two whole numbers."""
    hd = x.shape[-1]
    w = x.double().view(*x.shape[:-1], max(1, hd // 64), min(hd, 64))
    m = w.amin(-1)
    y = (w.amax(-1) - m) / 15
    s = y.half()
    s = torch.where(s.double() < y, (s.view(torch.int16) + 1).view(torch.float16), s)
    d = torch.where(s > 0, s.double(), 1.0)[..., None]
    q = torch.floor((w - m[..., None]) / d + 0.5)
    return q.to(torch.uint8).view(x.shape), s, m.half()


def _values(q, s, m):
    """What whole numbers, scales and smallest values stand for, in 32 bits."""
    hd = q.shape[-1]
    w = q.view(*q.shape[:-1], max(1, hd // 64), min(hd, 64)).float()
    return (w * s.float()[..., None] + m.float()[..., None]).view(q.shape)


def _tiles(q, s, m):
    """Whole numbers [nb, BLOCK, 2, KV, hd] and their scales and smallest values [nb, BLOCK, 2, KV, C]
    in the cache's own order, as include/aiq_ops.h lays them out: [nb, KV, bytes]."""
    nb, _, _, kv, hd = q.shape
    p = q[..., 0::2] | q[..., 1::2] << 4
    k, v = p[:, :, 0], p[:, :, 1]
    if hd == 32:
        k = k.reshape(nb, 4, 8, kv, 4, 4).permute(0, 3, 2, 4, 1, 5)
        v = v.reshape(nb, 2, 2, 4, 2, kv, 8, 2).permute(0, 5, 6, 3, 1, 7, 4, 2)
    else:
        c = hd // 64
        k = k.reshape(nb, 2, 2, 8, kv, c, 4, 8).permute(0, 4, 1, 5, 3, 6, 2, 7)
        v = v.reshape(nb, 2, 2, 4, 2, kv, c, 8, 4).permute(0, 5, 1, 6, 7, 3, 8, 4, 2)
    sm = torch.stack([s, m], -1).view(nb, 4, 8, 2, kv, -1, 2).permute(0, 4, 5, 3, 2, 1, 6).contiguous()
    return torch.cat([k.reshape(nb, kv, -1), v.reshape(nb, kv, -1), sm.view(nb, kv, -1).view(torch.uint8)], 2).contiguous()


def _cache(rows, block, place, nb, KV, hd):
    """The quantised cache of fp16 rows [T, 2 KV hd]: whole numbers, scales and smallest values by token, tiles."""
    q, s, m = _quantize(rows.view(-1, 2, KV, hd))
    out = []
    for x in (q, s, m):
        y = torch.zeros((nb, BLOCK, *x.shape[1:]), dtype=x.dtype, device="cuda")
        y[block, place] = x
        out.append(y)
    return q, s, m, _tiles(*out)


def prepare(case, seed):
    rng, st = _rng(case, seed), State()
    g = torch.Generator(device="cuda")
    g.manual_seed(int(rng.integers(0, 2 ** 62)))
    st.case = dict(case)
    if case["op"] == "select":
        n, b, V, keep = case["rows"], case["beams"], case["vocab"], case["keep"]
        t = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[case["type"]]
        # rows from almost flat to peaked
        std = torch.empty(n * b, 1, device="cuda").uniform_(0.7, 4.0, generator=g)
        z = torch.empty(n * b, V, device="cuda").normal_(0, 1, generator=g) * std
        if case["banned"]:
            z[torch.empty(n * b, V, device="cuda").uniform_(0, 1, generator=g) < case["banned"]] = -math.inf
        st.logits = z.to(t)
        # scores of hypotheses some tokens long, best first; a few have ended, a few places hold none
        scores = -np.sort(rng.uniform(5, 12, (n, b)), 1).astype(np.float32)
        at = rng.permutation(n)
        done, none = (x[at] for x in _hypotheses(case))
        scores[none] = -np.inf
        st.scores = torch.from_numpy(scores).cuda()
        st.done = torch.from_numpy(done.astype(np.int32)).cuda()
        st.parents, st.tokens, st.out_done = (torch.zeros((n, keep), dtype=torch.int32, device="cuda") for _ in range(3))
        st.out = torch.zeros((n, keep), device="cuda")
        st.eos, st.pad = 2, 0
        torch.cuda.synchronize()
        return st
    if case["op"] == "reorder":
        n, b = case["rows"], case["beams"]
        unit = 4 if case["bytes"] % 4 == 0 and case["pitch"] % 4 == 0 else 1
        st.width = case["bytes"] // unit
        t = torch.int32 if unit == 4 else torch.uint8
        st.rows = torch.randint(0, 2 ** 31 - 1 if unit == 4 else 256, (case["layers"], n * b, case["pitch"] // unit),
                                dtype=t, device="cuda", generator=g)
        st.to = st.rows if case["inplace"] else torch.zeros_like(st.rows)
        st.parents = torch.from_numpy(rng.permutation(_parents(case))).cuda()
        torch.cuda.synchronize()
        return st
    H, KV, hd, S = case["heads"], case["kv"], case["hd"], case["rows"]
    kd = KV * hd
    st.lens = torch.from_numpy(rng.permutation(_lens(case))).cuda()
    st.T = int(st.lens.sum())
    st.starts = torch.zeros(S + 1, dtype=torch.int64, device="cuda")
    st.starts[1:] = st.lens.cumsum(0)
    st.seq = st.starts.int()
    st.block, st.place, st.nb = _slots(st.starts[:-1], st.lens)
    st.kv = _normal(g, (st.T, (H + 2 * KV) * hd if case["op"] == "quantize" else 2 * kd))
    tile = BLOCK * hd + 256 * max(1, hd // 64)
    if case["op"] == "quantize":
        st.cache = torch.zeros((st.nb, KV, tile), dtype=torch.uint8, device="cuda")
        st.back = torch.zeros((st.T, 2 * kd), dtype=torch.float16, device="cuda")
    elif case["op"] == "readback":
        st.q, st.s, st.m, st.cache = _cache(st.kv, st.block, st.place, st.nb, KV, hd)
        st.kv = None
        st.back = torch.zeros((st.T, (H + 2 * KV) * hd), dtype=torch.float16, device="cuda")
    else:
        P, one, R = case["prefix"], torch.tensor([0], device="cuda"), S * case["beams"]
        st.q, st.s, st.m, st.cache = _cache(st.kv, st.block, st.place, st.nb, KV, hd)
        st.kv = None
        b, p, n = _slots(one, one + max(P, 1))
        st.pq, st.ps, st.pm, st.pcache = _cache(_normal(g, (max(P, 1), 2 * kd)), b, p, n, KV, hd)
        G = GEN_CAP // BLOCK
        q, s, m = _quantize(_normal(g, (R * G, BLOCK, 2, KV, hd)))
        st.gcache = _tiles(q, s, m)
        st.gq, st.gs, st.gm = (x.view(R, GEN_CAP, 2, KV, -1) for x in (q, s, m))
        st.qkv = _normal(g, (R, (H + 2 * KV) * hd))
        st.out = torch.zeros((R, H * hd), dtype=torch.float16, device="cuda")
        st.held = torch.zeros((R, 2 * kd), dtype=torch.float16, device="cuda")
    torch.cuda.synchronize()
    return st


# ------------------------------------------------------------- plain forms ---

def _plain_quantize(st):
    c = st.case
    q, s, m = _quantize(st.kv[:, c["heads"] * c["hd"]:].reshape(-1, 2, c["kv"], c["hd"]))
    return {"values": _values(q, s, m).clamp(max=65504).half().view(st.T, -1)}


def _plain_readback(st):
    c = st.case
    st.back[:, c["heads"] * c["hd"]:] = _values(st.q, st.s, st.m).clamp(max=65504).half().view(st.T, -1)
    return {"rows": st.back}


def _plain_attend(st):
    c = st.case
    H, KV, hd, S, B, P, slot = c["heads"], c["kv"], c["hd"], c["rows"], c["beams"], c["prefix"], c["slot"]
    R = S * B
    new = _quantize(st.qkv[:, H * hd:].reshape(R, 2, KV, hd))
    for state, x in zip((st.gq, st.gs, st.gm), new):
        state[:, slot] = x
    q = st.qkv[:, :H * hd].float().view(S, B, KV, H // KV, hd) / math.sqrt(hd)
    # the shared prefix
    pk, pv = _values(st.pq, st.ps, st.pm)[:P].unbind(1)
    # every sequence's own tokens, padded to the longest
    j = torch.arange(int(st.lens.max()), device="cuda")
    at = (st.starts[:-1, None] + j).clamp(max=st.T - 1)
    ok, ov = _values(st.q[at], st.s[at], st.m[at]).unbind(2)
    # every row's generated tokens
    gk, gv = (x.reshape(S, B, slot + 1, KV, hd)
              for x in _values(st.gq[:, :slot + 1], st.gs[:, :slot + 1], st.gm[:, :slot + 1]).unbind(2))
    out = (j >= st.lens[:, None])[:, None, None, None]
    z = torch.cat([torch.einsum("sbhgd,lhd->sbhgl", q, pk),
                   torch.einsum("sbhgd,slhd->sbhgl", q, ok).masked_fill(out, -math.inf),
                   torch.einsum("sbhgd,sblhd->sbhgl", q, gk)], -1)
    p = (z - z.amax(-1, keepdim=True)).exp()
    p = p / p.sum(-1, keepdim=True)
    a, b = P, P + len(j)
    o = (torch.einsum("sbhgl,lhd->sbhgd", p[..., :a], pv) + torch.einsum("sbhgl,slhd->sbhgd", p[..., a:b], ov)
         + torch.einsum("sbhgl,sblhd->sbhgd", p[..., b:], gv))
    return {"out": o.reshape(R, H * hd).half(), "held": _values(*new).clamp(max=65504).half().view(R, -1)}


def _plain_select(st):
    c = st.case
    n, B, V, keep = c["rows"], c["beams"], c["vocab"], c["keep"]
    k = min(keep, V)
    z, order = st.logits.float().sort(dim=1, descending=True, stable=True)
    # scores of different beams may lie next to one another
    top = z[:, :1].double()
    lse = top + torch.cat([(x.double() - t).exp().sum(1, keepdim=True).log()
                           for x, t in zip(z.split(512), top.split(512))])
    live = (st.scores > -math.inf).view(n * B, 1)
    s = torch.where(live & (z[:, :k] > -math.inf), st.scores.double().view(n * B, 1) + (z[:, :k].double() - lse), -math.inf)
    tokens = order[:, :k].int()
    # a hypothesis that has ended goes on as itself
    ended = (st.done != 0).view(n * B, 1)
    first = torch.arange(k, device="cuda") == 0
    s = torch.where(ended, torch.where(first, st.scores.double().view(n * B, 1), -math.inf), s)
    tokens = torch.where(ended, st.pad, tokens)
    s, at = s.view(n, B * k).sort(dim=1, descending=True, stable=True)
    s, at = s[:, :keep], at[:, :keep]
    none = s == -math.inf
    parents = torch.where(none, 0, at // k).int()
    tokens = torch.where(none, st.pad, tokens.view(n, B * k).gather(1, at)).int()
    done = (none | (st.done.gather(1, parents.long()) != 0) | (tokens == st.eos)).int()
    if s.shape[1] < keep:
        more = keep - s.shape[1]
        s = torch.nn.functional.pad(s, (0, more), value=-math.inf)
        parents, tokens, done = (torch.nn.functional.pad(x, (0, more), value=v) for x, v in
                                 ((parents, 0), (tokens, st.pad), (done, 1)))
    return {"parents": parents, "tokens": tokens, "scores": s.float(), "done": done}


def _plain_reorder(st):
    b = st.case["beams"]
    n = len(st.parents)
    rows = (st.parents.long() + b * torch.arange(n, device="cuda")[:, None]).view(-1)
    st.to[:, :, :st.width] = st.rows[:, rows, :st.width]
    return {"rows": st.to}


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
    if c["op"] == "select":
        t = {"f32": aiq.LOGITS_F32, "f16": aiq.LOGITS_F16, "bf16": aiq.LOGITS_BF16}[c["type"]]
        ctx.op_beam_select(st.logits.data_ptr(), t, c["vocab"], c["rows"], c["beams"], c["vocab"], st.scores.data_ptr(),
                           c["keep"], st.parents.data_ptr(), st.tokens.data_ptr(), st.out.data_ptr(),
                           done=st.done.data_ptr(), done_out=st.out_done.data_ptr(), eos=st.eos, pad=st.pad)
        return {"parents": st.parents, "tokens": st.tokens, "scores": st.out, "done": st.out_done}
    if c["op"] == "reorder":
        ctx.op_beam_reorder(st.rows.data_ptr(), st.to.data_ptr(), c["bytes"], c["pitch"], c["rows"], c["beams"],
                            st.parents.data_ptr(), layers=c["layers"], layer_pitch=c["rows"] * c["beams"] * c["pitch"])
        return {"rows": st.to}
    H, KV, hd, S = c["heads"], c["kv"], c["hd"], c["rows"]
    kd = KV * hd
    if c["op"] == "quantize":
        ctx.op_kv_quantize4(st.kv.data_ptr() + 2 * H * hd, st.kv.shape[1], st.T, st.seq.data_ptr(), S, KV, hd,
                            st.cache.data_ptr())
        ctx.op_kv_dequantize4(st.cache.data_ptr(), st.T, st.seq.data_ptr(), S, KV, hd, st.back.data_ptr(), 2 * kd)
        return {"values": st.back}
    if c["op"] == "readback":
        ctx.op_kv_dequantize4(st.cache.data_ptr(), st.T, st.seq.data_ptr(), S, KV, hd, st.back.data_ptr() + 2 * H * hd,
                              st.back.shape[1])
        return {"rows": st.back}
    P = c["prefix"]
    ctx.op_decode_attention_q4(st.qkv.data_ptr(), S * c["beams"], H, KV, hd, st.cache.data_ptr(), st.T,
                               st.seq.data_ptr(), st.gcache.data_ptr(), GEN_CAP, c["slot"], st.out.data_ptr(),
                               beams=c["beams"], prefix=st.pcache.data_ptr() if P else 0, P=P, held=st.held.data_ptr())
    return {"out": st.out, "held": st.held}


def run(state):
    if own:
        return _own(state)
    return {"quantize": _plain_quantize, "readback": _plain_readback, "attend": _plain_attend, "select": _plain_select,
            "reorder": _plain_reorder}[state.case["op"]](state)


# -------------------------------------------------------------------- work ---

def work(case):
    if case["op"] == "select":
        done, none = _hypotheses(case)
        size = 4 if case["type"] == "f32" else 2
        # rows that have ended or hold no hypothesis need not be read
        return {"bytes": int((~(done | none)).sum()) * case["vocab"] * size + done.size * 8 + case["rows"] * case["keep"] * 16,
                "flops": 0}
    if case["op"] == "reorder":
        p = _parents(case)
        moved = p != np.arange(case["beams"]) if case["inplace"] else np.ones(p.shape, bool)
        read = sum(len(set(r[m])) for r, m in zip(p, moved))
        return {"bytes": case["layers"] * case["bytes"] * float(read + moved.sum()) + 4.0 * p.size, "flops": 0}
    width = 2 * case["kv"] * case["hd"]  # values of a token
    held = width / 2 + width / min(case["hd"], 64) * 4  # a token's bytes in the cache
    lens = _lens(case).astype(np.float64)
    T = float(lens.sum())
    if case["op"] == "quantize":  # fp16 in, the cache and the values that it stands for out
        return {"bytes": T * (width * 4 + held), "flops": 0}
    if case["op"] == "readback":
        return {"bytes": T * (width * 2 + held), "flops": 0}
    H, hd, P, slot, B = case["heads"], case["hd"], case["prefix"], case["slot"], case["beams"]
    R = case["rows"] * B
    flops = 4.0 * H * hd * (B * T + R * (P + slot + 1))
    return {"bytes": (T + P + R * (slot + 1)) * held + R * (H * hd * 4 + width * 4), "flops": flops}


# ------------------------------------------------------- the same in 64 bits ---

def _exact_held(x):
    """fp16 rows [n, KV, hd] as the cache holds them, in 64 bits: a group of at most 64 elements a row."""
    g = x.double().reshape(-1, min(x.shape[-1], 64))
    low, high = g.aminmax(dim=1, keepdim=True)
    step = (high - low) / 15
    # up to the next number of fp16: of 11 significant bits, and a multiple of 2^-24
    _, e = torch.frexp(step)
    last = torch.tensor([2.0 ** i for i in range(-24, 5)], dtype=torch.float64, device=x.device)[e.long().clamp(min=-13) + 13]
    step = torch.ceil(step / last) * last
    n = torch.ceil(((g - low) * 2 - step) / (step * 2).clamp(min=1e-300))
    # halves go up
    n = torch.where(n * 2 * step + step == (g - low) * 2, n + 1, n)
    return (low + n.clamp(min=0) * step).view(x.shape)


def _exact_attend(st):
    c = st.case
    H, KV, hd, P, slot, B = c["heads"], c["kv"], c["hd"], c["prefix"], c["slot"], c["beams"]
    new = _exact_held(st.qkv[:, H * hd:].reshape(-1, KV, hd)).view(-1, 2, KV, hd)

    def values(q, s, m):
        w = q.double().unflatten(-1, (s.shape[-1], -1))
        return (m.double()[..., None] + s.double()[..., None] * w).flatten(-2)

    starts, out = st.starts.tolist(), []
    prefix = values(st.pq, st.ps, st.pm)[:P]
    for r in range(len(st.qkv)):
        a, b = starts[r // B], starts[r // B + 1]
        rows = torch.cat([prefix, values(st.q[a:b], st.s[a:b], st.m[a:b]),
                          values(st.gq[r, :slot], st.gs[r, :slot], st.gm[r, :slot]), new[r:r + 1]])
        k, v = rows.unbind(1)
        z = torch.matmul(st.qkv[r, :H * hd].double().view(KV, H // KV, hd), k.permute(1, 2, 0)) * hd ** -0.5
        out.append(torch.matmul(torch.softmax(z, -1), v.transpose(0, 1)).reshape(-1))
    return {"out": torch.stack(out), "held": new.clamp(max=65504).flatten(1)}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "select":
        n, B, keep = case["rows"], case["beams"], case["keep"]
        best = []
        for r in range(n):
            z = st.logits[r * B:(r + 1) * B].double()
            s = st.scores[r].double()[:, None] + torch.log_softmax(z, 1)
            s = torch.where(st.done[r, :, None] != 0, -math.inf, s)
            s[:, 0] = torch.where(st.done[r] != 0, st.scores[r].double(), s[:, 0])
            s = s.nan_to_num(nan=-math.inf, neginf=-math.inf).flatten()
            s = torch.cat([s, s.new_full((keep,), -math.inf)])
            best.append(s.topk(keep).values)
        # which tokens these are is decided by comparisons alone
        return {"parents": None, "tokens": None, "scores": torch.stack(best), "done": None}
    if case["op"] == "reorder":
        at = torch.arange(len(st.parents), device="cuda")
        old, to = (x.view(case["layers"], len(at), case["beams"], -1) for x in (st.rows.clone(), st.to))
        for i in range(case["beams"]):
            to[:, :, i, :st.width] = old[:, at, st.parents[:, i].long(), :st.width]
        return {"rows": st.to}
    KV, hd, H = case["kv"], case["hd"], case["heads"]
    if case["op"] == "quantize":
        rows = torch.cat([_exact_held(x.reshape(-1, KV, hd)).view(len(x), -1)
                          for x in st.kv[:, H * hd:].split(1 << 15)])
        return {"values": rows.clamp(max=65504)}
    if case["op"] == "readback":
        rows = torch.zeros(st.back.shape, dtype=torch.float64, device="cuda")
        w = st.q.double().unflatten(-1, (st.s.shape[-1], -1)) * st.s.double()[..., None] + st.m.double()[..., None]
        rows[:, H * hd:] = w.flatten(1)
        return {"rows": rows}
    return _exact_attend(st)
