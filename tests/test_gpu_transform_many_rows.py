"""AI_TRANSFORM of batches of many rows: on the 8-bit cache by the attention's warp per
task, with the rows' order made once a chunk, and drawn tokens whose logits are made a
part of the rows at a time."""
import numpy as np
import pytest

import kv8
import synth
from helpers import MARGIN_RTOL, gpu_ctx, weights_list
from oracle import transformer as tf
from test_gpu_transform_options import SHAPES, _inputs, _run

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
