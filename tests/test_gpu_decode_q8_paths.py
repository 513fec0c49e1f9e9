"""The variants of the attention over the 8-bit cache that its rules choose between:
5 to 8 query heads per KV head, for which a product takes the probabilities' two parts
one after the other, by a warp per task and by several CTAs for one; and rows in
another order."""
import numpy as np
import pytest

import kv8
from helpers import gpu_ctx
from test_gpu_kv_cache8 import Step, _d, _rows

pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = gpu_ctx()
    yield c
    c.close()


def _step(ctx, seed, heads, lens, P, slot, cap=96):
    s = Step(seed, *heads, lens, P, cap)
    s.fill_generated(slot)
    qkv = s.qkv()
    out = s.call(ctx, qkv, slot)
    s.append(qkv)
    s.check(out, qkv)


@pytest.mark.parametrize("heads", [(8, 1, 32), (6, 1, 32), (10, 2, 32), (5, 1, 64), (14, 2, 128)], ids=str)
@pytest.mark.parametrize("P,slot", [(0, 0), (33, 31), (40, 63)])
def test_five_to_eight_heads(ctx, heads, P, slot):
    _step(ctx, P + slot, heads, [0, 1, 31, 32, 33, 200, 17, 16], P, slot)


@pytest.mark.parametrize("heads", [(8, 1, 32), (8, 1, 64), (7, 1, 64), (6, 1, 128)], ids=str)
@pytest.mark.parametrize("slot", [0, 31, 40])
def test_five_to_eight_heads_in_many_rows(ctx, heads, slot):
    """A warp takes whole tasks."""
    _step(ctx, slot, heads, [i % 41 for i in range(2500)], 5 if slot else 0, slot, cap=64)


@pytest.mark.parametrize("heads", [(8, 1, 32), (7, 1, 32), (8, 1, 64), (7, 1, 64), (8, 1, 128), (7, 1, 128), (16, 2, 64)], ids=str)
@pytest.mark.parametrize("lens", [[6000], [5000, 2100]], ids=str)
def test_five_to_eight_heads_of_several_ranges(ctx, heads, lens):
    """Several CTAs for a task: its last one merges, a warp two heads one after the other."""
    _step(ctx, sum(lens), heads, lens, 20, 9)


@pytest.mark.parametrize("heads", [(8, 8, 32), (16, 8, 64), (8, 1, 64), (8, 8, 128)], ids=str)
@pytest.mark.parametrize("longest", [90, 250])
def test_rows_in_another_order_have_the_same_bits(ctx, heads, longest):
    """Where a warp takes whole tasks, nothing of a row depends on the rows beside it."""
    Hq, Hkv, hd = heads
    R = 700 if Hkv == 8 else 2500
    s = Step(11, *heads, [(i * 37) % longest for i in range(R)], 9, 32)
    own = _rows(s.rng, s.T, 2 * Hkv * hd)
    st = kv8.starts(s.lens)

    def load(order):
        lens = [s.lens[r] for r in order]
        rows = np.concatenate([own[st[r]:st[r + 1]] for r in order])
        c, sc, _, _ = kv8.build_cache(rows, lens, Hkv, hd)
        s.d[0], s.d[1], s.d[4] = _d(c), _d(sc), _d(kv8.starts(lens))

    qkv = s.qkv()
    load(range(R))
    first = s.call(ctx, qkv, 0)
    order = np.random.default_rng(1).permutation(R)
    load(order)
    assert np.array_equal(s.call(ctx, qkv[order], 0), first[order])
    # and beside other rows: the first half, twice
    order = np.concatenate([np.arange(R // 2), np.arange(R - R // 2) % (R // 2)])
    s.T = int(sum(s.lens[r] for r in order))
    load(order)
    assert np.array_equal(s.call(ctx, qkv[order], 0), first[order])
