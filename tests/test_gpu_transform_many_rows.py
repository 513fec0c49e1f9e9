"""AI_TRANSFORM of batches of many rows: on the 8-bit cache by the attention's warp per
task, with the rows' order made once a chunk, and drawn tokens whose logits are made a
part of the rows at a time."""
import numpy as np
import pytest

import kv8
import synth
from helpers import MARGIN_RTOL, gpu_ctx, weights_list
from oracle import transformer as tf
from paper_2608_10139_gb300 import aiq
from test_gpu_transform_options import SHAPES, _inputs, _run, _zero_model

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = gpu_ctx()
    yield c
    c.close()


@pytest.mark.parametrize("name,rows,new", [("mha_hd32", 1400, 36), ("gqa4_hd64", 2600, 4), ("gqa3_hd64", 2600, 4),
                                           ("gqa8_hd128", 4000, 4)])
def test_many_rows_on_the_8_bit_cache(ctx, name, rows, new):
    shape = SHAPES[name]
    W = synth.make_weights(shape, 3110)
    table, prefix = _inputs(shape, rows, 31, empty_every=50, prefix_len=20)
    r = _run(ctx, shape, W, table, prefix, [], new, bits=8)
    assert np.array_equal(r.gen_row_ids, np.arange(rows)) and r.n_chunks == 1
    lens = np.diff(table.offsets)
    model = tf.Model(shape, W, True)
    for row in {0, 1, rows - 1, int(lens.argmax()), rows // 2 + 7}:
        z = kv8.logits_on_8_bits(model, prefix, table.text(row), r.gen_tokens[row, :-1])
        for t in range(new):
            gap = z[t].max() - z[t][r.gen_tokens[row, t]]
            assert gap <= MARGIN_RTOL * max(1.0, abs(z[t].max())), f"row {row} step {t}: {gap:.4g} below the largest"


@pytest.mark.parametrize("bits", [16, 8])
def test_draws_in_little_memory(bits):
    """115 MB of logits a step under a cap that leaves 40 MB beside the greedy query's least."""
    shape, W, bias = _zero_model(vocab=32000)
    rows = 900
    table, prefix = _inputs(shape, rows, 14, lens=np.full(rows, 3))
    u = np.random.default_rng(3).random((rows, 2)).astype(np.float32) * np.float32(0.999)
    c = gpu_ctx()
    try:
        m = c.load_model(shape, weights_list(shape, W))
        t = c.load_table(table.cols, (table.offsets, table.tokens))
        c.set_option("kv_bits", bits)
        loaded = sum(v.nbytes for v in weights_list(shape, W))
        for cap in range(loaded, loaded + (1 << 29), 4 << 20):
            c.set_option("device_bytes_max", cap)
            try:
                c.run_transform(t, m, [], prefix, 2)
                break
            except aiq.AiqError as e:
                assert e.status == aiq.ERR_OOM
        assert cap < loaded + (1 << 28)
        sampling = dict(temperature=0.9, top_k=40, top_p=0.9)
        c.set_option("device_bytes_max", cap + (40 << 20))
        r = c.run_transform(t, m, [], prefix, 2, sampling=sampling, uniforms=u)
        want = [[kv8.sample(bias, u[i, s], 0.9, 40, 0.9, 0.0)[0] for s in range(2)] for i in range(rows)]
        assert np.array_equal(r.gen_tokens, want)
    finally:
        c.close()


def test_numbers_of_64_bits_below_1_stay_below_1(ctx):
    """The largest 64-bit numbers below 1 are in [0, 1), though their nearest 32-bit number is 1."""
    shape, W, bias = _zero_model()
    table, prefix = _inputs(shape, 5, 15)
    u = np.full((5, 3), 1 - 2.0 ** -53)
    u[1] = 1 - 2.0 ** -25
    r = _run(ctx, shape, W, table, prefix, [], 3, sampling=dict(temperature=1.3, top_k=400), uniforms=u)
    want = kv8.sample(bias, np.float32(1 - 2.0 ** -24), 1.3, 400, 1.0, 0.0)[0]
    assert (r.gen_tokens == want).all()
    for bad in (1.0, -1e-9, float("nan")):  # these are not
        u[2, 1] = bad
        with pytest.raises(aiq.AiqError) as e:
            _run(ctx, shape, W, table, prefix, [], 3, sampling=dict(top_k=5), uniforms=u)
        assert e.value.status == aiq.ERR_DEVICE_CHECK


def test_sampling_without_numbers_is_refused(ctx):
    shape, W, _ = _zero_model()
    table, prefix = _inputs(shape, 5, 15)
    with pytest.raises(ValueError):
        _run(ctx, shape, W, table, prefix, [], 3, sampling=dict(top_k=5))
