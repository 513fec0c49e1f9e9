"""Calls on the 4-bit cache and of beam search that meet each other or that no single batch reaches:
two contexts at once, many groups, few rows of close hypotheses, many rows with starts that do not
ascend."""
import threading

import numpy as np
import pytest

import kv4
from helpers import gpu_ctx
from paper_2608_10139_gb300 import aiq
from test_gpu_beam import _check, _select
from test_gpu_kv_cache4 import Batch, _d, _rows

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = gpu_ctx()
    yield c
    c.close()


def test_more_groups_than_counters(ctx):
    rng = np.random.default_rng(1)
    z = rng.standard_normal((5000, 2, 60)).astype(np.float32)
    scores = -rng.uniform(0, 4, (5000, 2))
    held, out = _select(ctx, z, scores, None, 4, "f16", eos=7)
    _check(held, out, scores, None, 4, eos=7, groups=range(0, 5000, 97))


@pytest.mark.parametrize("n,beams,V", [(1, 4, 128256), (2, 16, 40000), (5000, 2, 300)])
def test_close_hypotheses_of_few_and_of_many_rows(ctx, n, beams, V):
    """Alike but for some light tokens, which decide: rows in several parts, and more groups than are merged by the
    row kernel."""
    rng = np.random.default_rng(n + beams)
    z = np.repeat(rng.standard_normal((n, 1, V)).astype(np.float32), beams, 1)
    for b in range(1, beams):
        at = rng.integers(0, V, (n, 5))
        for g in range(n):
            z[g, b, at[g]] = np.float32(-6) + np.float32(1e-3) * rng.standard_normal(5).astype(np.float32)
    scores = np.full((n, beams), -2.25)
    held, out = _select(ctx, z, scores, None, 2 * beams)
    _check(held, out, scores, None, 2 * beams, groups=range(0, n, max(1, n // 30)))


@pytest.mark.parametrize("rows,beams,low,high", [(1200, 1, 250, 550), (3000, 1, 0, 60), (60, 4, 100, 400), (3, 1, 100, 400)])
def test_starts_that_do_not_ascend_and_the_call_behind_them(ctx, rows, beams, low, high):
    """Reported, with nothing written outside; the next call is not disturbed.  1,200 long rows are cut into
    ranges, 3,000 short ones drawn, the others split."""
    rng = np.random.default_rng(rows)
    lens = [int(x) for x in rng.integers(low, high, rows)]
    b = Batch(ctx, rng, 64, 8, 2, beams, lens, 40, 33)
    good = b.st.clone()
    qkv = _rows(rng, b.R, 12 * 64)
    for at, value in ((rows // 2, 3), (rows, 2 ** 31 - 1), (0, -5), (rows // 3, 2 ** 31 - 1)):
        b.st.copy_(good)
        b.st[at] = value
        torch.cuda.synchronize()
        with pytest.raises(aiq.AiqError) as e:
            b.step(qkv, 0)
        assert e.value.status == aiq.ERR_DEVICE_CHECK
        assert (b.out[b.R] == 9).all() and (b.guard[-1] == 77).all()
    b.st.copy_(good)
    torch.cuda.synchronize()
    b.check(rng, [0], rows=rng.choice(b.R, min(b.R, 20), replace=False).tolist())


def test_two_contexts_at_once():
    """Each has its own stream, workspace and counters."""
    rng = np.random.default_rng(9)
    work = []
    for k in range(2):
        c = gpu_ctx()
        b = Batch(c, rng, 64, 8, 2, 1, [int(x) for x in rng.integers(100, 700, 900 if k else 12)], 40, 33)
        z = torch.as_tensor(rng.standard_normal((40, 4, 5000)).astype(np.float32)).cuda()
        s = torch.as_tensor(-rng.uniform(0, 4, (40, 4)).astype(np.float32)).cuda()
        p, t = (torch.zeros(40 * 4, dtype=torch.int32, device="cuda") for _ in range(2))
        work.append((c, b, _rows(rng, b.R, 12 * 64), z, s, p, t, torch.zeros(160, device="cuda")))
    torch.cuda.synchronize()

    def run(w, outs, times):
        c, b, qkv, z, s, p, t, so = w
        for _ in range(times):
            out, _ = b.step(qkv, 0)
            c.op_beam_select(z.data_ptr(), aiq.LOGITS_F32, 5000, 40, 4, 5000, s.data_ptr(), 4, p.data_ptr(), t.data_ptr(), so.data_ptr())
            outs.append((out.copy(), p.cpu().numpy(), t.cpu().numpy(), so.cpu().numpy()))

    alone = [[], []]
    for w, o in zip(work, alone):
        run(w, o, 1)
    both = [[], []]
    threads = [threading.Thread(target=run, args=(w, o, 15)) for w, o in zip(work, both)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    for o, ref in zip(both, alone):
        assert len(o) == 15
        for got in o:
            assert [np.array_equal(x, y) for x, y in zip(got, ref[0])] == [True] * 4
    for w in work:
        w[0].close()


@pytest.mark.parametrize("hd,beams,rows", [(64, 3, 300), (64, 1, 250), (128, 1, 200), (32, 1, 250)])
def test_texts_cut_anywhere(ctx, hd, beams, rows):
    """A text's tiles over the ranges of one to many warps: lengths 0 to 500, two much longer."""
    rng = np.random.default_rng(hd + beams)
    lens = [int(x) for x in rng.integers(0, 500, rows) * (rng.random(rows) < 0.9)]
    lens[rows // 3] = 9000
    lens[-1] = 5000
    b = Batch(ctx, rng, hd, 16, 8, beams, lens, 70, 40)
    b.check(rng, [0], rows=rng.choice(b.R, 40, replace=False).tolist() + [rows // 3 * beams, b.R - 1, 0])


@pytest.mark.parametrize("n,beams,V,keep,type", [(900, 4, 3000, 4, "f16"), (2, 8, 70000, 16, "f32"), (200, 1, 30000, 32, "bf16")])
def test_equal_selections_give_equal_bits(ctx, n, beams, V, keep, type):
    """Rows in ascending order too, whose lists are cut many times: the order in which entries arrive must not show."""
    rng = np.random.default_rng(V)
    z = rng.standard_normal((n, beams, V)).astype(np.float32)
    z[::3] = np.sort(z[::3], -1)
    scores = -rng.uniform(0, 4, (n, beams))
    _, first = _select(ctx, z, scores, None, keep, type)
    for _ in range(12):
        _, out = _select(ctx, z, scores, None, keep, type)
        assert [np.array_equal(x, y) for x, y in zip(first, out)] == [True] * 4


def test_a_cache_beyond_32_bits(ctx):
    """Tokens, tiles and generated blocks whose offsets pass 2^32 bytes: as the same ones near the start."""
    rng = np.random.default_rng(12)
    Hq, Hkv, hd, n = 8, 8, 128, 100
    w, tb, T = 2 * Hkv * hd, kv4.tile_bytes(hd), 3_800_001
    rows = _d(_rows(rng, n, w))
    kv = torch.empty((T, w), dtype=torch.float16, device="cuda")
    kv[T - n:] = rows
    far, near = (torch.full((nb, Hkv, tb), 7, dtype=torch.uint8, device="cuda") for nb in (T // 32 + 1, n // 32 + 1))
    assert far.numel() > 2 ** 32
    st_far, st_near = _d(np.array([T - n, T], np.int32)), _d(np.array([0, n], np.int32))
    ctx.op_kv_quantize4(kv.data_ptr(), w, T, st_far.data_ptr(), 1, Hkv, hd, far.data_ptr())
    ctx.op_kv_quantize4(rows.data_ptr(), w, n, st_near.data_ptr(), 1, Hkv, hd, near.data_ptr())
    assert torch.equal(far[(T - n) // 32:][:4], near) and (far[:(T - n) // 32] == 7).all()
    kv[T - n:] = 0
    ctx.op_kv_dequantize4(far.data_ptr(), T, st_far.data_ptr(), 1, Hkv, hd, kv.data_ptr(), w)
    back = torch.zeros_like(rows)
    torch.cuda.synchronize()
    ctx.op_kv_dequantize4(near.data_ptr(), n, st_near.data_ptr(), 1, Hkv, hd, back.data_ptr(), w)
    assert torch.equal(kv[T - n:], back)
    del kv
    # two rows of the sequence, as beams, whose generated tokens have room for a million more
    qkv = _d(_rows(rng, 2, (Hq + 2 * Hkv) * hd))
    outs = []
    for own, st, t, cap in ((far, st_far, T, 4_000_000), (near, st_near, n, 40)):
        gen = torch.full((2, -(-cap // 32), Hkv, tb), 9, dtype=torch.uint8, device="cuda")
        out = torch.zeros((2, Hq * hd), dtype=torch.float16, device="cuda")
        torch.cuda.synchronize()
        ctx.op_decode_attention_q4(qkv.data_ptr(), 2, Hq, Hkv, hd, own.data_ptr(), t, st.data_ptr(), gen.data_ptr(), cap, 0,
                                   out.data_ptr(), beams=2)
        outs.append((out.cpu().numpy(), gen[:, 0].clone(), bool((gen[:, 1] == 9).all())))
        del gen
    assert torch.equal(outs[0][1], outs[1][1]) and outs[0][2] and outs[1][2]
    q = qkv.cpu().numpy()
    held = kv4.quantize(rows.cpu().numpy().reshape(n, 2, Hkv, hd))
    for r in range(2):
        new = kv4.quantize(q[r, Hq * hd:].reshape(1, 2, Hkv, hd))
        c, sc, m = (np.concatenate(x) for x in zip(held, new))
        x, big = kv4.values(c, sc, m), (np.abs(m.astype(np.float64)) + 15 * sc.astype(np.float64)).max(-1)
        ref, tol = kv4.attend(q[r, :Hq * hd].astype(np.float64).reshape(Hq, hd), x[:, 0], x[:, 1], big[:, 0], big[:, 1])
        for out, _, _ in outs:
            assert (np.abs(out[r].astype(np.float64).reshape(Hq, hd) - ref) <= tol).all()


def test_rows_beyond_32_bits_of_selection_and_reordering(ctx):
    rng = np.random.default_rng(13)
    ld = 2 ** 30 + 24
    big = torch.zeros(2 * ld + 5000, dtype=torch.float16, device="cuda")
    z = rng.standard_normal((1, 3, 5000)).astype(np.float16)
    for b in range(3):
        big[b * ld:b * ld + 5000] = torch.as_tensor(z[0, b]).cuda()
    s = torch.as_tensor(np.array([[-1.0, -2.0, -0.5]], np.float32)).cuda()
    p, t = (torch.zeros(6, dtype=torch.int32, device="cuda") for _ in range(2))
    so = torch.zeros(6, device="cuda")
    torch.cuda.synchronize()
    ctx.op_beam_select(big.data_ptr(), aiq.LOGITS_F16, ld, 1, 3, 5000, s.data_ptr(), 6, p.data_ptr(), t.data_ptr(), so.data_ptr())
    rp, rt, rs, _ = kv4.select(z[0].astype(np.float32), s.cpu().numpy()[0], np.zeros(3), 6, -1, 0)
    assert np.array_equal(p.cpu().numpy(), rp) and np.array_equal(t.cpu().numpy(), rt)
    assert np.abs(so.cpu().numpy() - rs).max() <= 2.0 ** -18 + np.abs(rs).max() * 2.0 ** -24
    # and the rows themselves, 2 GB apart, moved in place
    parents = torch.as_tensor(np.array([[2, 0, 0]], np.int32)).cuda()
    torch.cuda.synchronize()
    ctx.op_beam_reorder(big.data_ptr(), big.data_ptr(), 9998, 2 * ld, 1, 3, parents.data_ptr())
    for b, a in enumerate((2, 0, 0)):
        got = big[b * ld:b * ld + 5000].cpu().numpy()
        assert np.array_equal(got[:4999], z[0, a, :4999]) and got[4999] == z[0, b, 4999]


@pytest.mark.parametrize("beams,bytes,pitch,offset", [(3, 9000, 9013, 5), (4, 1024, 1027, 0), (4, 1025, 1027, 3), (16, 257, 260, 1),
                                                      (16, 4099, 4100, 15), (2, 2047, 2048, 8), (1, 8193, 8200, 2), (7, 15, 17, 9),
                                                      (8, 513, 520, 4), (5, 4004, 4012, 12)])
@pytest.mark.parametrize("in_place", [True, False])
def test_reorder_of_rows_that_begin_anywhere(ctx, beams, bytes, pitch, offset, in_place):
    """Pieces of rows that source and destination cut at different bytes, their ends, and what lies beside them."""
    rng = np.random.default_rng(bytes + beams)
    n, layers, other = 9, 2, offset if in_place else (offset * 7 + 3) % 16
    lp = n * beams * pitch + 1
    src = rng.integers(0, 256, layers * lp + 64, dtype=np.uint8)
    dst = src if in_place else rng.integers(0, 256, len(src), dtype=np.uint8)
    p = rng.integers(0, beams, (n, beams)).astype(np.int32)
    ref = dst.copy()
    for l in range(layers):
        for g in range(n):
            for i in range(beams):
                a, b = (l * lp + (g * beams + k) * pitch for k in (i, p[g, i]))
                ref[other + a:other + a + bytes] = src[offset + b:offset + b + bytes]
    ds = torch.as_tensor(src).cuda()
    dd = ds if in_place else torch.as_tensor(dst).cuda()
    dp = torch.as_tensor(p).cuda()
    torch.cuda.synchronize()
    ctx.op_beam_reorder(ds.data_ptr() + offset, dd.data_ptr() + other, bytes, pitch, n, beams, dp.data_ptr(), layers=layers, layer_pitch=lp)
    assert np.array_equal(dd.cpu().numpy(), ref)


@pytest.mark.parametrize("type", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,beams,V,keep", [(400, 4, 9000, 8), (3, 3, 9001, 6), (700, 2, 12289, 4)])
def test_rows_whose_largest_logits_come_late(ctx, type, n, beams, V, keep):
    """More than a list holds lie above the bound of the first chunks: ascending rows, and a few among others."""
    rng = np.random.default_rng(V)
    z = (rng.standard_normal((n, beams, V)) * 2).astype(np.float32)
    late = rng.random((n, beams)) < 0.3
    z[late] = np.sort(z[late], -1)
    z[0, 0, 4096:] += 30  # nearly all of the row
    scores = -rng.uniform(0, 3, (n, beams))
    held, out = _select(ctx, z, scores, None, keep, type, ld=V + 3, offset=1)
    _check(held, out, scores, None, keep, groups=range(0, n, max(1, n // 40)))


@pytest.mark.parametrize("bytes,pitch", [(33, 35), (5001, 5003), (600000, 600004)])
def test_a_parent_outside_leaves_its_group(ctx, bytes, pitch):
    """Rows that begin anywhere, and 4-byte words: the group stays as it was, the others are moved."""
    rng = np.random.default_rng(bytes)
    x = rng.integers(0, 256, 9 * pitch, dtype=np.uint8)
    d = torch.as_tensor(x).cuda()
    p = torch.as_tensor(np.array([[1, 0, 2], [0, 3, 1], [2, 2, 0]], np.int32)).cuda()
    torch.cuda.synchronize()
    with pytest.raises(aiq.AiqError) as e:
        ctx.op_beam_reorder(d.data_ptr(), d.data_ptr(), bytes, pitch, 3, 3, p.data_ptr())
    assert e.value.status == aiq.ERR_DEVICE_CHECK
    ref = x.reshape(9, pitch).copy()
    ref[:, :bytes] = ref[[1, 0, 2, 3, 4, 5, 8, 8, 6], :bytes]
    assert np.array_equal(d.cpu().numpy().reshape(9, pitch), ref)
