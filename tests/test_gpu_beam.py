"""Beam search's selection and the reordering of its state against their definitions, and
both with the 4-bit cache as a search uses them, through the C-ABI (aiq_ops.h)."""
import numpy as np
import pytest

import kv4
from helpers import gpu_ctx
from paper_2608_10139_gb300 import aiq

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": (aiq.LOGITS_F32, torch.float32), "f16": (aiq.LOGITS_F16, torch.float16),
         "bf16": (aiq.LOGITS_BF16, torch.bfloat16)}


@pytest.fixture(scope="module")
def ctx():
    c = gpu_ctx()
    yield c
    c.close()


def _select(ctx, z, scores, done, keep, type="f32", eos=-1, pad=0, ld=None, offset=0, fails=False):
    """z [n, beams, V] fp32 values, stored as `type` at a pitch of ld elements, `offset` elements into their buffer."""
    code, dt = TYPES[type]
    n, beams, V = z.shape
    ld = ld or V
    buf = torch.full((n * beams * ld + offset + 8,), float("nan"), dtype=dt, device="cuda")
    view = buf[offset:offset + n * beams * ld].view(n * beams, ld)
    view[:, :V] = torch.as_tensor(z.reshape(n * beams, V)).cuda().to(dt)
    held = view[:, :V].float().cpu().numpy().reshape(n, beams, V)
    sc = torch.as_tensor(np.ascontiguousarray(scores, np.float32)).cuda()
    dn = torch.as_tensor(np.ascontiguousarray(done, np.int32)).cuda() if done is not None else None
    p, t, d = (torch.full((n * keep + 1,), -9, dtype=torch.int32, device="cuda") for _ in range(3))
    s = torch.full((n * keep + 1,), -9.0, device="cuda")
    torch.cuda.synchronize()

    def call():
        ctx.op_beam_select(view.data_ptr(), code, ld, n, beams, V, sc.data_ptr(), keep, p.data_ptr(), t.data_ptr(),
                           s.data_ptr(), done=dn.data_ptr() if dn is not None else 0, done_out=d.data_ptr(), eos=eos, pad=pad)
    if fails:
        with pytest.raises(aiq.AiqError) as e:
            call()
        assert e.value.status == aiq.ERR_DEVICE_CHECK
    else:
        call()
    out = [x.cpu().numpy() for x in (p, t, s, d)]
    assert all(x[-1] == -9 for x in out)
    return held, [x[:-1].reshape(n, keep) for x in out]


def _check(held, out, scores, done, keep, eos=-1, pad=0, groups=None):
    done = np.zeros(np.shape(scores)) if done is None else done
    for g in range(len(held)) if groups is None else groups:
        p, t, s, d = kv4.select(held[g], np.asarray(scores, np.float32)[g], done[g], keep, eos, pad)
        assert np.array_equal(out[0][g], p) and np.array_equal(out[1][g], t), f"group {g}: {out[0][g]} {out[1][g]}, not {p} {t}"
        assert np.array_equal(out[3][g], d)
        # the sum of a row's exponentials: tokens that are kept in 64 bits, the others' to 2^-18 of theirs; one rounding
        fin = s > -np.inf
        assert (np.isinf(out[2][g]) == ~fin).all()
        assert (np.abs(out[2][g][fin] - s[fin]) <= np.abs(s[fin]) * 2.0 ** -24 * 1.01 + 2.0 ** -18).all()


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("n,beams,V,keep", [(1, 1, 1, 1), (1, 1, 5, 1), (2, 2, 3, 4), (3, 4, 31, 8), (5, 3, 33, 3), (40, 4, 1000, 4),
                                            (2, 16, 1000, 32), (1, 16, 32000, 16), (7, 5, 4097, 10), (1, 8, 128256, 16),
                                            (2, 4, 128257, 4), (300, 2, 1500, 4), (1, 1, 300001, 2), (600, 4, 2500, 8)])
def test_selection(ctx, type, n, beams, V, keep):
    rng = np.random.default_rng(n * V + keep)
    z = (rng.standard_normal((n, beams, V)) * np.exp(rng.normal(0.3, 0.7, (n, beams, 1)))).astype(np.float32)
    scores = -rng.uniform(0, 6, (n, beams))
    done = rng.random((n, beams)) < 0.15
    scores[rng.random((n, beams)) < 0.1] = -np.inf
    eos, pad = int(rng.integers(0, V)), V - 1
    held, out = _select(ctx, z, scores, done, keep, type, eos, pad)
    _check(held, out, scores, done, keep, eos, pad, groups=range(0, n, max(1, n // 40)))


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("ld,offset", [(1003, 0), (1003, 1), (1008, 3), (1001, 7), (2048, 5)])
def test_pitch_and_alignment(ctx, type, ld, offset):
    """Rows that begin anywhere; what lies between them (NaN) is not read."""
    rng = np.random.default_rng(ld + offset)
    z = rng.standard_normal((4, 3, 1001)).astype(np.float32) * 2
    scores = -rng.uniform(0, 3, (4, 3))
    held, out = _select(ctx, z, scores, None, 6, type, ld=ld, offset=offset)
    _check(held, out, scores, None, 6)


def test_the_first_step_has_one_hypothesis(ctx):
    rng = np.random.default_rng(1)
    z = np.repeat(rng.standard_normal((3, 1, 5000)), 6, 1).astype(np.float32)
    scores = np.full((3, 6), -np.inf)
    scores[:, 0] = 0
    held, out = _select(ctx, z, scores, None, 6)
    _check(held, out, scores, None, 6)
    assert not out[0].any()


@pytest.mark.parametrize("V", [1, 7, 1025, 5000, 70000])
@pytest.mark.parametrize("levels", [1, 2, 3])
def test_equal_offers_go_by_hypothesis_and_token(ctx, V, levels):
    rng = np.random.default_rng(V + levels)
    row = rng.integers(0, levels, (2, 1, V)).astype(np.float32) - 1
    z = np.repeat(row, 4, 1)  # the hypotheses are alike, and their scores equal
    z[0][z[0] == 0] = -0.0
    for keep in (1, 4, 8):
        held, out = _select(ctx, z, np.full((2, 4), -1.5), None, keep, "f16")
        _check(held, out, np.full((2, 4), -1.5), None, keep)


def test_offers_that_32_bits_do_not_tell_apart(ctx):
    """Hypotheses whose offers differ by less than 2^-24 of them: the sums of the exponentials decide."""
    rng = np.random.default_rng(8)
    n, V = 64, 30000
    base = rng.standard_normal((n, 1, V)).astype(np.float32)
    z = np.repeat(base, 4, 1)
    for b in range(1, 4):  # one of the light tokens a little more or less
        for g in range(n):
            at = rng.integers(0, V, 5)
            z[g, b, at] = np.float32(-6) + np.float32(1e-3) * rng.standard_normal(5).astype(np.float32)
    scores = np.full((n, 4), -2.25)
    held, out = _select(ctx, z, scores, None, 8)
    _check(held, out, scores, None, 8)


def test_rows_that_offer_little_or_nothing(ctx):
    rng = np.random.default_rng(2)
    z = rng.standard_normal((6, 4, 3000)).astype(np.float32)
    z[0] = -np.inf                                   # nothing at all
    z[1, :3] = -np.inf                               # one hypothesis alone
    z[2] = -np.inf
    z[2, 1, 2999] = -7                               # one token alone
    z[3, 2] = np.float32(-3.4e38)                    # the type's lowest, everywhere but in one place
    z[3, 2, 17] = np.float32(-3.3e38)
    z[4, :] = np.where(rng.random((4, 3000)) < 0.999, -np.inf, z[4])
    z[5, 0] = np.float32(-3.4e38)                    # the type's lowest, everywhere
    scores = -rng.uniform(0, 3, (6, 4))
    scores[5, 1:] = -np.inf
    held, out = _select(ctx, z, scores, None, 8, pad=5)
    _check(held, out, scores, None, 8, pad=5)
    scores[:] = -np.inf                              # no hypothesis
    held, out = _select(ctx, z, scores, None, 4, pad=5)
    _check(held, out, scores, None, 4, pad=5)


def test_rows_in_order_and_peaked(ctx):
    n = 40000
    z = np.stack([np.arange(n), np.arange(n)[::-1], np.where(np.arange(n) == 31999, 80, 0),
                  np.where(np.arange(n) % 1000 == 3, 5, -5), 1e4 * np.sin(np.arange(n)), np.where(np.arange(n) < 6000, -1e5, 1e5)])
    z = z[:, None].astype(np.float32) / np.array([16, 16, 1, 1, 1, 1])[:, None, None]
    for keep in (1, 2, 32):
        held, out = _select(ctx, z, np.zeros((6, 1)), None, keep)
        _check(held, out, np.zeros((6, 1)), None, keep)


def test_small_differences_count(ctx):
    """A token of probability close to 1: its log is small, and exact to its own rounding."""
    z = np.full((2, 2, 2000), -12.0, np.float32)
    z[0, 0, 3], z[0, 1, 9], z[1, 0, 3], z[1, 1, 1999] = 10, 12, 30, 5
    scores = np.zeros((2, 2))
    held, out = _select(ctx, z, scores, None, 2)
    for g in range(2):
        p, t, s, d = kv4.select(held[g], scores[g], np.zeros(2), 2, -1, 0)
        assert np.array_equal(out[0][g], p) and np.array_equal(out[1][g], t)
        assert (np.abs(out[2][g] - s) <= np.abs(s) * 2.0 ** -17 + 1e-12).all()


def test_ended_hypotheses_are_not_read(ctx):
    rng = np.random.default_rng(3)
    z = rng.standard_normal((5, 4, 700)).astype(np.float32)
    done = rng.random((5, 4)) < 0.5
    z[done] = np.nan
    scores = -rng.uniform(0, 9, (5, 4))
    scores[2, 1], z[2, 1] = -np.inf, np.nan
    held, out = _select(ctx, z, scores, done, 4, eos=3, pad=699)
    _check(held, out, scores, done, 4, 3, 699)


@pytest.mark.parametrize("V", [50, 5000, 100000])
@pytest.mark.parametrize("what", ["logit nan", "logit inf", "score nan", "score inf"])
def test_what_allows_no_choice_is_reported(ctx, V, what):
    rng = np.random.default_rng(4)
    z = rng.standard_normal((3, 4, V)).astype(np.float32)
    scores = -rng.uniform(0, 3, (3, 4))
    bad = np.nan if "nan" in what else np.inf
    if "logit" in what:
        z[1, 2, V - 1] = bad
    else:
        scores[1, 2] = bad
    held, out = _select(ctx, z, scores, None, 4, fails=True, pad=7)
    _check(held, out, scores, None, 4, pad=7, groups=[0, 2])
    assert (out[0][1] == 0).all() and (out[1][1] == 7).all() and (out[2][1] == -np.inf).all() and (out[3][1] == 1).all()
    z[1, 2], scores[1, 2] = 0, -1
    held, out = _select(ctx, z, scores, None, 4)
    _check(held, out, scores, None, 4)


# -------------------------------------------------------------- reordering ---

@pytest.mark.parametrize("beams", [1, 2, 3, 4, 5, 8, 11, 16])
@pytest.mark.parametrize("bytes,pitch,offset", [(16, 16, 0), (4096, 4112, 0), (36, 40, 4), (4, 4, 0), (33, 35, 1), (1, 1, 3), (20000, 20000, 0),
                                                (6, 8, 2)])
@pytest.mark.parametrize("in_place", [True, False])
def test_reorder(ctx, beams, bytes, pitch, offset, in_place):
    rng = np.random.default_rng(beams + bytes)
    n, layers = 5, 3
    lp = n * beams * pitch + (16 if pitch % 16 == 0 else 3)
    size = layers * lp + 64
    src = rng.integers(0, 256, size, dtype=np.uint8)
    dst = src if in_place else rng.integers(0, 256, size, dtype=np.uint8)
    p = rng.integers(0, beams, (n, beams)).astype(np.int32)
    p[0] = np.arange(beams)
    p[1] = np.arange(beams)[::-1]
    ref = dst.copy()
    for l in range(layers):
        for g in range(n):
            for i in range(beams):
                a, b = (offset + l * lp + (g * beams + k) * pitch for k in (i, p[g, i]))
                ref[a:a + bytes] = src[b:b + bytes]
    ds = torch.as_tensor(src).cuda()
    dd = ds if in_place else torch.as_tensor(dst).cuda()
    dp = torch.as_tensor(p).cuda()
    torch.cuda.synchronize()
    ctx.op_beam_reorder(ds.data_ptr() + offset, dd.data_ptr() + offset, bytes, pitch, n, beams, dp.data_ptr(), layers=layers,
                        layer_pitch=lp)
    assert np.array_equal(dd.cpu().numpy(), ref)


def test_reorder_of_layers_within_rows(ctx):
    """[row][layer]: the layers' pitch is less than the rows'."""
    rng = np.random.default_rng(1)
    x = rng.integers(0, 2 ** 31, (6, 4, 24), dtype=np.int32)
    d, p = torch.as_tensor(x).cuda(), torch.as_tensor(np.array([[1, 1, 0], [2, 0, 2]], np.int32)).cuda()
    torch.cuda.synchronize()
    ctx.op_beam_reorder(d.data_ptr(), d.data_ptr(), 80, 384, 2, 3, p.data_ptr(), layers=4, layer_pitch=96)
    ref = x.copy()
    ref[:, :, :20] = x[[1, 1, 0, 5, 3, 5], :, :20]
    assert np.array_equal(d.cpu().numpy(), ref)


@pytest.mark.parametrize("bad", [-1, 3, 2 ** 31 - 1])
def test_a_parent_outside_the_group_is_reported(ctx, bad):
    x = np.arange(9 * 8, dtype=np.int32).reshape(9, 8)
    d = torch.as_tensor(x).cuda()
    p = torch.as_tensor(np.array([[1, 0, 2], [0, bad, 1], [2, 2, 0]], np.int32)).cuda()
    torch.cuda.synchronize()
    with pytest.raises(aiq.AiqError) as e:
        ctx.op_beam_reorder(d.data_ptr(), d.data_ptr(), 32, 32, 3, 3, p.data_ptr())
    assert e.value.status == aiq.ERR_DEVICE_CHECK
    assert np.array_equal(d.cpu().numpy(), x[[1, 0, 2, 3, 4, 5, 8, 8, 6]])


# ---------------------------------------------------------------- together ---

@pytest.mark.parametrize("beams", [2, 4])
def test_a_search_on_the_4_bit_cache(ctx, beams):
    """Steps of a search of two layers' attention, selection and reordering: every beam's
    cache and history is its ancestors', and its score the sum of their steps'."""
    rng = np.random.default_rng(beams)
    S, L, Hq, Hkv, hd, cap, V, steps = 3, 2, 4, 2, 64, 40, 300, 37
    R, w, gb = S * beams, 2 * Hkv * hd, 2
    lens = [5, 40, 0]
    rows = (rng.standard_normal((sum(lens), w)) * 0.9).astype(np.float16)
    cache, mask, *own4 = kv4.build_cache(rows, lens, Hkv, hd)
    from kv8 import starts
    own, st = torch.as_tensor(cache).cuda(), torch.as_tensor(starts(lens)).cuda()
    tb = kv4.tile_bytes(hd)
    gen = torch.zeros((L, R, gb, Hkv, tb), dtype=torch.uint8, device="cuda")
    out = torch.zeros((R, Hq * hd), dtype=torch.float16, device="cuda")
    W = torch.as_tensor((rng.standard_normal((Hq * hd, V)) * 0.2).astype(np.float32)).cuda()
    emb = torch.as_tensor((rng.standard_normal((L, V, (Hq + 2 * Hkv) * hd)) * 0.9).astype(np.float16)).cuda()
    scores = torch.full((S, beams), -np.inf, device="cuda")
    scores[:, 0] = 0
    token = torch.ones((S, beams), dtype=torch.int32, device="cuda")
    done = torch.zeros_like(token)
    history = torch.zeros((R, cap), dtype=torch.int32, device="cuda")
    parents, tokens, done_out = (torch.zeros_like(token) for _ in range(3))
    scores_out = torch.zeros_like(scores)
    paths = [[[] for _ in range(beams)] for _ in range(S)]  # the tokens fed so far, by hypothesis
    for step in range(steps):
        fed = token.view(-1).long()
        history[:, step] = token.view(-1)
        for g in range(S):
            for i in range(beams):
                paths[g][i] = paths[g][i] + [int(token[g, i])]
        x = torch.zeros((R, Hq * hd), device="cuda")
        for l in range(L):
            qkv = emb[l, fed].contiguous()
            torch.cuda.synchronize()
            ctx.op_decode_attention_q4(qkv.data_ptr(), R, Hq, Hkv, hd, own.data_ptr(), sum(lens), st.data_ptr(),
                                       gen[l].data_ptr(), cap, step, out.data_ptr(), beams=beams)
            x += out.float()
        z = (x @ W).contiguous()
        torch.cuda.synchronize()
        ctx.op_beam_select(z.data_ptr(), aiq.LOGITS_F32, V, S, beams, V, scores.data_ptr(), beams, parents.data_ptr(),
                           tokens.data_ptr(), scores_out.data_ptr(), done=done.data_ptr(), done_out=done_out.data_ptr(), eos=7, pad=0)
        zn, sn, dn = z.cpu().numpy().reshape(S, beams, V), scores.cpu().numpy(), done.cpu().numpy()
        for g in range(S):
            p, t, s, d = kv4.select(zn[g], sn[g], dn[g], beams, 7, 0)
            assert np.array_equal(parents[g].cpu().numpy(), p) and np.array_equal(tokens[g].cpu().numpy(), t)
            assert np.array_equal(done_out[g].cpu().numpy(), d)
            paths[g] = [list(paths[g][i]) for i in p]
        used = step // 32 + 1
        ctx.op_beam_reorder(gen.data_ptr(), gen.data_ptr(), used * Hkv * tb, gb * Hkv * tb, S, beams, parents.data_ptr(),
                            layers=L, layer_pitch=R * gb * Hkv * tb)
        ctx.op_beam_reorder(history.data_ptr(), history.data_ptr(), 4 * (step + 1), 4 * cap, S, beams, parents.data_ptr())
        scores.copy_(scores_out), token.copy_(tokens), done.copy_(done_out)
        torch.cuda.synchronize()
    h = history.cpu().numpy()
    keys = emb.cpu().numpy()
    for g in range(S):
        for i in range(beams):
            r = g * beams + i
            assert list(h[r, :steps]) == paths[g][i]
            for l in range(L):
                ref, mask, *_ = kv4.build_cache(keys[l, paths[g][i], Hq * hd:], [steps], Hkv, hd)
                got = gen[l, r].cpu().numpy()
                assert np.array_equal(got[mask[:gb]], ref[:gb][mask[:gb]])
