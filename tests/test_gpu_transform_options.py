"""AI_TRANSFORM on the 8-bit key/value cache (option kv_bits) and with sampled tokens
(AIQ_GEN_SAMPLE), against the oracle."""
import ctypes as C
from dataclasses import replace

import numpy as np
import pytest

import kv8
import synth
from helpers import MARGIN_RTOL, gpu_ctx, weights_list
from oracle import relational as rel
from oracle import transformer as tf
from paper_2608_10139_gb300 import aiq

pytestmark = pytest.mark.gpu

SHAPES = {
    "mha_hd32": synth.TINY,
    "gqa4_hd64": replace(synth.TINY, d_model=256, n_heads=8, n_kv_heads=2, head_dim=64, d_ffn=512),
    "gqa3_hd64": replace(synth.TINY, d_model=256, n_heads=6, n_kv_heads=2, head_dim=64, d_ffn=384),
    "gqa8_hd128": replace(synth.TINY, d_model=256, n_heads=8, n_kv_heads=1, head_dim=128, d_ffn=384),
}


@pytest.fixture(scope="module")
def ctx():
    c = gpu_ctx()
    yield c
    c.close()


def _inputs(shape, n_rows, seed, empty_every=0, prefix_len=16, lens=None):
    rng = np.random.default_rng(seed)
    lens = rng.integers(1, 70, n_rows) if lens is None else np.asarray(lens)
    if empty_every:
        lens[::empty_every] = 0
    off = np.zeros(n_rows + 1, np.int64)
    np.cumsum(lens, out=off[1:])
    toks = rng.integers(0, shape.vocab, int(off[-1])).astype(np.int32)
    cols = {"r": rng.integers(0, 10, n_rows).astype(np.int32)}
    return synth.Table(n_rows, cols, off, toks), rng.integers(0, shape.vocab, prefix_len).astype(np.int32)


def _run(ctx, shape, W, table, prefix, preds, max_new, bits=16, rows=4096, **kw):
    m = ctx.load_model(shape, weights_list(shape, W))
    t = ctx.load_table(table.cols, (table.offsets, table.tokens))
    ctx.set_option("kv_bits", bits)
    ctx.set_option("decode_rows", rows)
    try:
        return ctx.run_transform(t, m, preds, prefix, max_new, **kw)
    finally:
        ctx.set_option("kv_bits", 16)
        ctx.set_option("decode_rows", 4096)
        ctx.free_table(t)
        ctx.free_model(m)


def _zero_model(vocab=500, scale=1.5):
    """Every position's logits are the LM-head bias, exactly."""
    shape = replace(synth.TINY, vocab=vocab)
    W = synth.make_weights(shape, 0, zero=True)
    W["lm_bias"] = synth.f32_to_bf16_bits((np.random.default_rng(3).standard_normal(vocab) * scale).astype(np.float32))
    return shape, W, tf.bf16_to_f64(W["lm_bias"])


@pytest.mark.parametrize("name", list(SHAPES))
def test_8_bit_cache_matches_the_oracle_on_8_bits(ctx, name):
    """Every greedy token is an argmax, to the parity tolerance, of the oracle's logits
    with the same keys and values rounded the same way; 36 tokens, so that a
    generated block is completed and attended."""
    shape = SHAPES[name]
    W = synth.make_weights(shape, 3100)
    table, prefix = _inputs(shape, 14, 21, empty_every=6, prefix_len=33)
    preds = [("r", rel.GE, 3)]
    r = _run(ctx, shape, W, table, prefix, preds, 36, bits=8, rows=5)
    cand = rel.compact(rel.predicate_mask(table.cols, preds, table.n_rows))
    assert np.array_equal(r.gen_row_ids, cand) and r.gen_tokens.shape == (len(cand), 36)
    model = tf.Model(shape, W, True)
    for i, row in enumerate(cand[:5]):
        z = kv8.logits_on_8_bits(model, prefix, table.text(int(row)), r.gen_tokens[i, :-1])
        for t in range(36):
            top = z[t].max()
            gap = top - z[t][r.gen_tokens[i, t]]
            assert gap <= MARGIN_RTOL * max(1.0, abs(top)), f"row {row} step {t}: {gap:.4g} below the largest"


def test_8_bit_cache_without_a_prefix_and_in_few_tokens(ctx):
    shape = SHAPES["gqa4_hd64"]
    W = synth.make_weights(shape, 3101)
    table, prefix = _inputs(shape, 9, 4, prefix_len=0)
    model = tf.Model(shape, W, True)
    for new in (1, 2, 3):
        r = _run(ctx, shape, W, table, prefix, [], new, bits=8)
        for i in range(3):
            z = kv8.logits_on_8_bits(model, prefix, table.text(i), r.gen_tokens[i, :-1])
            for t in range(new):
                assert z[t].max() - z[t][r.gen_tokens[i, t]] <= MARGIN_RTOL * max(1.0, abs(z[t].max()))


def test_options_leave_greedy_fp16_results_as_they_were(ctx):
    shape = SHAPES["gqa4_hd64"]
    W = synth.make_weights(shape, 3102)
    table, prefix = _inputs(shape, 40, 5)
    first = _run(ctx, shape, W, table, prefix, [], 12)
    _run(ctx, shape, W, table, prefix, [], 12, bits=8)
    again = _run(ctx, shape, W, table, prefix, [], 12)
    assert np.array_equal(first.gen_tokens, again.gen_tokens)


@pytest.mark.parametrize("bits", [16, 8])
def test_top_k_1_gives_the_greedy_tokens(ctx, bits):
    shape = SHAPES["gqa4_hd64"]
    W = synth.make_weights(shape, 3103)
    table, prefix = _inputs(shape, 60, 6, empty_every=13)
    u = np.random.default_rng(1).random((60, 10)).astype(np.float32) * np.float32(0.999)
    preds = [("r", rel.GE, 4)]
    greedy = _run(ctx, shape, W, table, prefix, preds, 10, bits=bits)
    drawn = _run(ctx, shape, W, table, prefix, preds, 10, bits=bits, sampling=dict(temperature=0.7, top_k=1), uniforms=u)
    assert np.array_equal(greedy.gen_tokens, drawn.gen_tokens)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("rows", [7, 4096])
@pytest.mark.parametrize("sampling", [dict(temperature=0.9, top_k=40), dict(temperature=1.4, top_k=500, top_p=0.8),
                                      dict(temperature=1.0, top_k=300, top_p=0.97, min_p=0.02)], ids=str)
def test_draws_are_exact_where_the_logits_are(ctx, bits, rows, sampling):
    """Step t of a row takes its own uniform number, whichever rows run together."""
    shape, W, bias = _zero_model()
    table, prefix = _inputs(shape, 50, 8, empty_every=9)
    u = np.minimum(np.random.default_rng(2).random((50, 9)).astype(np.float32), np.float32(1 - 2.0 ** -24))
    preds = [("r", rel.GE, 5)]
    r = _run(ctx, shape, W, table, prefix, preds, 9, bits=bits, rows=rows, sampling=sampling, uniforms=u)
    kw = {**dict(temperature=1.0, top_k=50, top_p=1.0, min_p=0.0), **sampling}
    for i, row in enumerate(r.gen_row_ids):
        want = [kv8.sample(bias, u[row, t], **kw)[0] for t in range(9)]
        assert r.gen_tokens[i].tolist() == want, row


def test_eos_pad_and_like_with_draws(ctx):
    shape, W, bias = _zero_model(vocab=40, scale=0.5)
    table, prefix = _inputs(shape, 30, 9)
    u = np.random.default_rng(4).random((30, 12)).astype(np.float32) * np.float32(0.999)
    sp = dict(temperature=1.0, top_k=40)
    toks = np.array([[kv8.sample(bias, u[i, t], 1.0, 40, 1.0, 0.0)[0] for t in range(12)] for i in range(30)])
    eos = int(np.bincount(toks.ravel()).argmax())
    r = _run(ctx, shape, W, table, prefix, [], 12, eos=eos, pad=7, sampling=sp, uniforms=u)
    for i in range(30):
        at = np.flatnonzero(toks[i] == eos)
        n = int(at[0]) if len(at) else 12
        want = np.where(np.arange(12) <= n, toks[i], 7)
        assert r.gen_text_len[i] == n and np.array_equal(r.gen_tokens[i], want)
    pat = toks[3, :2].tolist()
    r = _run(ctx, shape, W, table, prefix, [], 12, eos=-1, sampling=sp, uniforms=u, like=pat)
    want = [i for i in range(30) if rel.like_contains(toks[i], np.array(pat))]
    assert r.row_ids.tolist() == want and r.count == len(want)


def test_draws_stay_among_the_oracles_largest(ctx):
    shape = SHAPES["gqa4_hd64"]
    W = synth.make_weights(shape, 3104)
    table, prefix = _inputs(shape, 12, 10)
    u = np.random.default_rng(5).random((12, 8)).astype(np.float32) * np.float32(0.999)
    r = _run(ctx, shape, W, table, prefix, [], 8, bits=8, sampling=dict(temperature=1.0, top_k=20), uniforms=u)
    model = tf.Model(shape, W, True)
    distinct = 0
    for i in range(4):
        z = kv8.logits_on_8_bits(model, prefix, table.text(i), r.gen_tokens[i, :-1])
        for t in range(8):
            kth = np.sort(z[t])[-20]
            assert z[t][r.gen_tokens[i, t]] >= kth - MARGIN_RTOL * max(1.0, abs(z[t].max()))
            distinct += r.gen_tokens[i, t] != tf.first_argmax(z[t])
    assert distinct > 8  # they are draws, not the largest


def test_refusals(ctx):
    shape, W, _ = _zero_model()
    table, prefix = _inputs(shape, 6, 11)
    u = np.full((6, 3), 0.5, np.float32)
    for sp in (dict(temperature=0.0), dict(top_k=0), dict(top_k=501), dict(top_p=0.0), dict(min_p=2.0)):
        with pytest.raises(aiq.AiqError) as e:
            _run(ctx, shape, W, table, prefix, [], 3, sampling=sp, uniforms=u)
        assert e.value.status == aiq.ERR_INVALID_ARG, sp
    with pytest.raises(ValueError):
        _run(ctx, shape, W, table, prefix, [], 4, sampling=dict(top_k=5), uniforms=u)
    with pytest.raises(aiq.AiqError):
        ctx.set_option("kv_bits", 4)
    # a number outside [0, 1) is reported where a candidate row takes it, and only there
    bad = u.copy()
    row = int(np.flatnonzero(table.cols["r"] == table.cols["r"].max())[0])
    bad[row, 1] = 1.0
    with pytest.raises(aiq.AiqError) as e:
        _run(ctx, shape, W, table, prefix, [], 3, sampling=dict(top_k=5), uniforms=bad)
    assert e.value.status == aiq.ERR_DEVICE_CHECK
    _run(ctx, shape, W, table, prefix, [("r", rel.LT, int(table.cols["r"][row]))], 3, sampling=dict(top_k=5), uniforms=bad)
    # more than 8 query heads per KV head
    wide = replace(synth.TINY, d_model=512, n_heads=16, n_kv_heads=1, head_dim=32, d_ffn=512)
    with pytest.raises(aiq.AiqError) as e:
        _run(ctx, wide, synth.make_weights(wide, 1), table, prefix, [], 3, bits=8)
    assert e.value.status == aiq.ERR_UNSUPPORTED


def test_uniforms_alone_are_refused(ctx):
    shape, W, _ = _zero_model()
    table, prefix = _inputs(shape, 3, 12)
    with pytest.raises(ValueError):
        _run(ctx, shape, W, table, prefix, [], 3, uniforms=np.zeros((3, 3), np.float32))


def test_the_flag_needs_its_arguments(ctx):
    shape, W, _ = _zero_model()
    table, prefix = _inputs(shape, 3, 12)
    m = ctx.load_model(shape, weights_list(shape, W))
    t = ctx.load_table(table.cols, (table.offsets, table.tokens))
    sel, keep = ctx._select(t, [], prefix, [], aiq.AGG_COUNT, 0, "text")
    g = aiq._Generate(2, -1, 0, None, 0, aiq.GEN_SAMPLE)
    h = C.c_int64()
    assert ctx.lib.aiq_run_transform(ctx.h, t.handle, m, C.byref(sel), C.byref(g), C.byref(h)) == aiq.ERR_INVALID_ARG
    ctx.free_table(t)
    ctx.free_model(m)


def test_short_memory_is_refused_and_the_context_works_on(ctx):
    shape, W, bias = _zero_model()
    table, prefix = _inputs(shape, 40, 13)
    u = np.full((40, 4), 0.25, np.float32)
    m = ctx.load_model(shape, weights_list(shape, W))
    t = ctx.load_table(table.cols, (table.offsets, table.tokens))
    ctx.set_option("kv_bits", 8)
    try:
        ctx.set_option("device_bytes_max", 1 << 20)
        with pytest.raises(aiq.AiqError) as e:
            ctx.run_transform(t, m, [], prefix, 4, sampling=dict(top_k=30), uniforms=u)
        assert e.value.status == aiq.ERR_OOM
        ctx.set_option("device_bytes_max", 0)
        r = ctx.run_transform(t, m, [], prefix, 4, sampling=dict(top_k=30), uniforms=u)
        assert (r.gen_tokens == kv8.sample(bias, 0.25, 1.0, 30, 1.0, 0.0)[0]).all()
    finally:
        ctx.set_option("device_bytes_max", 0)
        ctx.set_option("kv_bits", 16)
        ctx.free_table(t)
        ctx.free_model(m)
