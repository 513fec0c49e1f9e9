"""Beam search's selection where offers lie closer together than its 32-bit sums tell apart: what is kept and its
order are those of the definition (aiq_ops.h), and scores are as exact as it says."""
import numpy as np
import pytest

import beam_close
import kv4
from helpers import gpu_ctx
from paper_2608_10139_gb300 import aiq
from test_gpu_beam import TYPES, _select

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = gpu_ctx()
    yield c
    c.close()


def _compare(ctx, groups, type, ld=None, offset=0):
    z, scores, done, keep = groups
    held, out = _select(ctx, z, scores, done, keep, type, ld=ld, offset=offset)
    assert np.array_equal(held, z)
    wrong = []
    for g in range(len(z)):
        p, t, s, d = kv4.select(z[g], scores[g], done[g], keep, -1, 0)
        if not (np.array_equal(out[0][g], p) and np.array_equal(out[1][g], t) and np.array_equal(out[3][g], d)):
            wrong.append(g)
        else:  # a log is right to 2^-17, and a score is rounded once
            assert (np.abs(out[2][g] - s) <= np.abs(s) * 2.0 ** -24 + 2.0 ** -17).all()
    assert not wrong, f"{len(wrong)} of {len(z)} groups, the first {wrong[:5]}"


# Rows that a group's last block merges (of two and of four), that are cut into parts, and that are merged by a launch.
@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("n,beams,V", [(200, 2, 4000), (200, 4, 4001), (9, 2, 40000), (700, 2, 3001), (90, 16, 1003)])
def test_a_tie_at_the_border_beside_another_offer(ctx, n, beams, V, type):
    rng = np.random.default_rng(n + beams)
    _compare(ctx, beam_close.ties_at_the_border(rng, n, beams, V, type), type)


@pytest.mark.parametrize("type", list(TYPES))
def test_ties_in_rows_that_begin_anywhere(ctx, type):
    rng = np.random.default_rng(77)
    _compare(ctx, beam_close.ties_at_the_border(rng, 100, 3, 2999, type), type, ld=3001, offset=5)


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("n,V", [(200, 4000), (9, 40000), (400, 3001)])
def test_a_flat_row_behind_peaked_ones(ctx, n, V, type):
    rng = np.random.default_rng(n)
    _compare(ctx, beam_close.peaked_before_flat(rng, n, V, type), type)


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("n,beams,V", [(200, 4, 4000), (2, 4, 128256), (3, 16, 20001), (700, 2, 1500)])
def test_hypotheses_that_one_light_token_tells_apart(ctx, n, beams, V, type):
    """Every group's rows are close to one another by any bound on a 32-bit sum."""
    rng = np.random.default_rng(n + beams)
    _compare(ctx, beam_close.light_tokens(rng, n, beams, V, type), type)


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("keep", [1, 4])
def test_more_ties_than_are_kept(ctx, type, keep):
    """Rows whose keep + 1 largest logits are equal, of equal scores: the hypothesis of the smaller sum comes first,
    and all that is kept is its."""
    rng = np.random.default_rng(keep)
    z, scores, done, _ = beam_close.light_tokens(rng, 150, 2, 4001, type)
    for g in range(150):
        free = np.flatnonzero(z[g, 0] == z[g, 1])
        z[g][:, rng.permutation(free)[:keep + 1]] = 4.5
    _compare(ctx, (z, scores, done, keep), type)


def test_rows_that_ascend_little_by_little(ctx):
    """Each chunk of a row is above what was read before, so that its list is cut back, and the sum of the others
    brought to another number, hundreds of times.  Beside it the same row backwards, whose score alone tells them apart."""
    V, n = 3_000_000, 310
    up = (np.arange(V) / V * 0.01).astype(np.float32)
    z = torch.as_tensor(np.stack([up, up[::-1]])).cuda().expand(n, 2, V).contiguous()
    scores = np.full((n, 2), -1, np.float32)
    scores[:, 1] += np.float32(2.0) ** -np.arange(18, 23)[np.arange(n) % 5] * np.where(np.arange(n) % 2, 1, -1)
    sc = torch.as_tensor(scores).cuda()
    p, t = (torch.zeros((n, 2), dtype=torch.int32, device="cuda") for _ in range(2))
    so = torch.zeros((n, 2), device="cuda")
    torch.cuda.synchronize()
    ctx.op_beam_select(z.data_ptr(), aiq.LOGITS_F32, V, n, 2, V, sc.data_ptr(), 2, p.data_ptr(), t.data_ptr(), so.data_ptr())
    p, t, so = (x.cpu().numpy() for x in (p, t, so))
    first = (scores[:, 1] > scores[:, 0]).astype(np.int32)  # (by 2^-22 at least, the row's two largest by 2^-27)
    want = scores.max(1)[:, None] + (up[::-1][:2].astype(np.float64) - beam_close.log_sum(up))
    assert (np.abs(so - want) <= np.abs(want) * 2.0 ** -24 + 2.0 ** -17).all(), np.abs(so - want).max()
    assert np.array_equal(p, np.repeat(first[:, None], 2, 1)), (p != first[:, None]).any(1).sum()
    assert np.array_equal(t, np.where(first[:, None], [0, 1], [V - 1, V - 2]))
