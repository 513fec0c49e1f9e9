"""AI_TRANSFORM on the 4-bit key/value cache (option kv4), against the oracle."""
from dataclasses import replace

import numpy as np
import pytest

import kv4
import synth
from helpers import MARGIN_RTOL, gpu_ctx, weights_list
from oracle import relational as rel
from oracle import transformer as tf
from paper_2608_10139_gb300 import aiq
from test_gpu_transform_options import SHAPES, _inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = gpu_ctx()
    yield c
    c.close()


def _run(ctx, shape, W, table, prefix, preds, max_new, on=1, rows=4096, **kw):
    m = ctx.load_model(shape, weights_list(shape, W))
    t = ctx.load_table(table.cols, (table.offsets, table.tokens))
    ctx.set_option("kv4", on)
    ctx.set_option("decode_rows", rows)
    try:
        return ctx.run_transform(t, m, preds, prefix, max_new, **kw)
    finally:
        ctx.set_option("kv4", 0)
        ctx.set_option("decode_rows", 4096)
        ctx.free_table(t)
        ctx.free_model(m)


@pytest.mark.parametrize("name", list(SHAPES))
def test_matches_the_oracle_on_4_bits(ctx, name):
    """Every greedy token is an argmax, to the parity tolerance, of the oracle's logits
    with the same keys and values rounded the same way; 36 tokens, past a block's end."""
    shape = SHAPES[name]
    W = synth.make_weights(shape, 3100)
    table, prefix = _inputs(shape, 14, 21, empty_every=6, prefix_len=33)
    preds = [("r", rel.GE, 3)]
    r = _run(ctx, shape, W, table, prefix, preds, 36, rows=5)
    cand = rel.compact(rel.predicate_mask(table.cols, preds, table.n_rows))
    assert np.array_equal(r.gen_row_ids, cand) and r.gen_tokens.shape == (len(cand), 36)
    model = tf.Model(shape, W, True)
    for i, row in enumerate(cand[:5]):
        z = kv4.logits_on_4_bits(model, prefix, table.text(int(row)), r.gen_tokens[i, :-1])
        for t in range(36):
            top = z[t].max()
            gap = top - z[t][r.gen_tokens[i, t]]
            assert gap <= MARGIN_RTOL * max(1.0, abs(top)), f"row {row} step {t}: {gap:.4g} below the largest"


def test_without_a_prefix_and_in_few_tokens(ctx):
    shape = SHAPES["gqa4_hd64"]
    W = synth.make_weights(shape, 3101)
    table, prefix = _inputs(shape, 9, 4, prefix_len=0)
    model = tf.Model(shape, W, True)
    for new in (1, 2, 3):
        r = _run(ctx, shape, W, table, prefix, [], new)
        for i in range(3):
            z = kv4.logits_on_4_bits(model, prefix, table.text(i), r.gen_tokens[i, :-1])
            for t in range(new):
                assert z[t].max() - z[t][r.gen_tokens[i, t]] <= MARGIN_RTOL * max(1.0, abs(z[t].max()))


def test_the_option_leaves_the_others_as_they_were(ctx):
    shape = SHAPES["gqa4_hd64"]
    W = synth.make_weights(shape, 3102)
    table, prefix = _inputs(shape, 40, 5)
    first = _run(ctx, shape, W, table, prefix, [], 12, on=0)
    on = _run(ctx, shape, W, table, prefix, [], 12)
    ctx.set_option("kv_bits", 8)
    try:
        both = _run(ctx, shape, W, table, prefix, [], 12)
    finally:
        ctx.set_option("kv_bits", 16)
    again = _run(ctx, shape, W, table, prefix, [], 12, on=0)
    assert np.array_equal(first.gen_tokens, again.gen_tokens) and np.array_equal(on.gen_tokens, both.gen_tokens)


@pytest.mark.parametrize("rows", [7, 4096])
def test_chunks_and_top_k_1_give_the_greedy_tokens(ctx, rows):
    shape = SHAPES["gqa8_hd128"]
    W = synth.make_weights(shape, 3103)
    table, prefix = _inputs(shape, 60, 6, empty_every=13)
    u = np.random.default_rng(1).random((60, 10)).astype(np.float32) * np.float32(0.999)
    preds = [("r", rel.GE, 4)]
    greedy = _run(ctx, shape, W, table, prefix, preds, 10)
    drawn = _run(ctx, shape, W, table, prefix, preds, 10, rows=rows, sampling=dict(temperature=0.7, top_k=1), uniforms=u)
    assert np.array_equal(greedy.gen_tokens, drawn.gen_tokens)


def test_it_takes_less_memory(ctx):
    """A query that the fp16 cache does not fit into the device bytes allowed runs on the 4-bit one."""
    shape = SHAPES["gqa8_hd128"]
    W = synth.make_weights(shape, 3104)
    table, prefix = _inputs(shape, 60, 7, lens=np.full(60, 1500))

    def tokens(on, cap):
        """In a context of its own, whose buffers no earlier query has made; None: no room."""
        with gpu_ctx() as c:
            m = c.load_model(shape, weights_list(shape, W))
            t = c.load_table(table.cols, (table.offsets, table.tokens))
            c.set_option("kv4", on)
            c.set_option("device_bytes_max", cap)
            try:
                return c.run_transform(t, m, [], prefix, 4).gen_tokens
            except aiq.AiqError as e:
                assert e.status == aiq.ERR_OOM
                return None

    def least(on):
        lo, hi = 1, 1 << 32
        want = tokens(on, hi)
        while hi - lo > 4 << 20:
            mid = (lo + hi) // 2
            got = tokens(on, mid)
            assert got is None or np.array_equal(got, want)
            lo, hi = (mid, hi) if got is None else (lo, mid)
        return hi
    # 90,000 tokens of two layers: 92 MB of fp16 keys and values, 26 MB in 4 bits
    assert least(0) - least(1) > 50 << 20


def test_refusals(ctx):
    for value in (2, -1, 4):
        with pytest.raises(aiq.AiqError) as e:
            ctx.set_option("kv4", value)
        assert e.value.status == aiq.ERR_INVALID_ARG
    shape = replace(SHAPES["gqa4_hd64"], n_heads=18, n_kv_heads=1, head_dim=64)
    W = synth.make_weights(shape, 1)
    table, prefix = _inputs(shape, 4, 1)
    with pytest.raises(aiq.AiqError) as e:
        _run(ctx, shape, W, table, prefix, [], 2)
    assert e.value.status == aiq.ERR_UNSUPPORTED


@pytest.mark.parametrize("option,value,cache", [("kv4", 1, "4-bit"), ("kv_bits", 8, "8-bit")])
def test_a_refusal_names_the_cache_in_use(ctx, option, value, cache):
    shape = replace(SHAPES["gqa4_hd64"], n_heads=18, n_kv_heads=1, head_dim=64)
    W = synth.make_weights(shape, 1)
    table, prefix = _inputs(shape, 4, 1)
    before = {"kv4": 0, "kv_bits": 16}[option]
    ctx.set_option(option, value)
    try:
        with pytest.raises(aiq.AiqError, match=f"the {cache} cache takes up to 8 query heads per KV head") as e:
            _run(ctx, shape, W, table, prefix, [], 2, on=int(option == "kv4"))
    finally:
        ctx.set_option(option, before)
    assert e.value.status == aiq.ERR_UNSUPPORTED
