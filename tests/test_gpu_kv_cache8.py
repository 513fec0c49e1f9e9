"""The 8-bit key/value cache (quantised as it is written, read back, attended and
appended to by a generation step) against its definition in 64 bits, through the
C-ABI (aiq_ops.h)."""
import numpy as np
import pytest

import kv8
from helpers import gpu_ctx
from paper_2608_10139_gb300 import aiq

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

LENGTHS = [
    [1], [31], [32], [33], [64, 1], [0, 0, 5], [100, 0, 32, 31, 33, 0, 1], [7] * 45 + [200], [0, 0],
]
# a sequence boundary in every place of a block, many short sequences, more than 32 * 32 of them
MANY = [[i % 40 for i in range(1500)], [1] * 40, [i for i in range(70)]]


@pytest.fixture(scope="module")
def ctx():
    c = gpu_ctx()
    yield c
    c.close()


def _d(a):
    t = torch.as_tensor(np.ascontiguousarray(a)).cuda()
    torch.cuda.synchronize()
    return t


def _rows(rng, n, width, std=0.9):
    # a scale of its own for every 16 rows, so that blocks differ
    s = np.repeat(np.exp(rng.normal(0, 1, -(-n // 16) if n else 0)), 16)[:n]
    return (rng.standard_normal((n, width)) * std * s[:, None]).astype(np.float16)


def _quantize(ctx, rows, lens, Hkv, hd, T=None, pad=0, fill=7):
    """rows at a pitch of their width + pad, the keys `pad` elements in."""
    T = len(rows) if T is None else T
    width = 2 * Hkv * hd
    buf = np.full((max(T, 1), width + pad), np.float16(np.nan))
    buf[:T, pad:] = rows[:T]
    kv, st = _d(buf), _d(kv8.starts(lens))
    nb = kv8.blocks(T, len(lens))
    cache = torch.full((max(nb, 1), Hkv, 64 * hd), fill, dtype=torch.uint8, device="cuda")
    scales = torch.full((max(nb, 1), Hkv, 2), float(fill), device="cuda")
    torch.cuda.synchronize()
    ctx.op_kv_quantize(kv.data_ptr() + 2 * pad, width + pad, T, st.data_ptr(), len(lens), Hkv, hd, cache.data_ptr(),
                       scales.data_ptr())
    return cache, scales, st


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("Hkv", [1, 3, 8])
@pytest.mark.parametrize("lens", LENGTHS, ids=lambda v: f"{len(v)}x{sum(v)}")
def test_quantize_is_exact(ctx, hd, Hkv, lens):
    rng = np.random.default_rng(hd * 10 + Hkv)
    T = sum(lens) + 3  # rows behind the last sequence
    rows = _rows(rng, T, 2 * Hkv * hd)
    rows[sum(lens):] = np.nan  # are not read
    ref, ref_s, q, s = kv8.build_cache(rows[:sum(lens)], lens, Hkv, hd, T=T, fill=7)
    cache, scales, st = _quantize(ctx, rows, lens, Hkv, hd, T=T, pad=8 * Hkv)
    got, nb = cache.cpu().numpy(), kv8.blocks(T, len(lens))
    for b in range(nb):
        assert np.array_equal(got[b], ref[b]), f"block {b}"
    assert np.array_equal(scales.cpu().numpy()[:nb], ref_s)
    # and back, into rows with a pitch; what lies beside and behind them stays
    back = torch.full((T, 2 * Hkv * hd + 16), 3.0, dtype=torch.float16, device="cuda")
    torch.cuda.synchronize()
    ctx.op_kv_dequantize(cache.data_ptr(), scales.data_ptr(), T, st.data_ptr(), len(lens), Hkv, hd,
                         back.data_ptr() + 16, 2 * Hkv * hd + 16)
    b = back.cpu().numpy()
    n = sum(lens)
    assert np.array_equal(b[:n, 8:-8], kv8.read_back(q, s))
    assert (b[n:] == 3).all() and (b[:, :8] == 3).all() and (b[:, -8:] == 3).all()
    # a value is off by at most half a step of its scale and its own rounding
    if n:
        x = rows[:n].astype(np.float64).reshape(n, 2, Hkv, hd)
        v = b[:n, 8:-8].astype(np.float64).reshape(x.shape)
        assert (np.abs(v - x) <= s[..., None] / 2 * (1 + 2.0 ** -20) + np.abs(v) * 2.0 ** -11 + 2.0 ** -25).all()


@pytest.mark.parametrize("lens", MANY, ids=lambda v: f"{len(v)}x{sum(v)}")
def test_many_sequences(ctx, lens):
    rng = np.random.default_rng(len(lens))
    rows = _rows(rng, sum(lens), 2 * 32)
    ref, ref_s, q, s = kv8.build_cache(rows, lens, 1, 32, fill=7)
    cache, scales, _ = _quantize(ctx, rows, lens, 1, 32)
    assert np.array_equal(cache.cpu().numpy()[:len(ref)], ref)
    assert np.array_equal(scales.cpu().numpy()[:len(ref)], ref_s)


@pytest.mark.parametrize("top", [65504.0, 1.0, 0.3333, 127.0, 254.0, 6.1e-5, 2.0 ** -24, 3 * 2.0 ** -24, 1023 * 2.0 ** -24])
def test_rounding_of_halves_and_extremes(ctx, top):
    """Every fp16 number from 0 to the block's largest that is a half step, its
    neighbours, and all multiples of top / 254."""
    top = np.float16(top)
    half = np.arange(0, 255) * np.float64(top) / 254
    x = np.concatenate([half.astype(np.float16), np.nextafter(half.astype(np.float16), np.float16(0)),
                        np.nextafter(half.astype(np.float16), np.float16(np.inf))])
    x = x[np.abs(x) <= top]
    x = np.concatenate([x, -x])
    per = BLK = 32 * 64 - 1
    n = -(-len(x) // per)
    rows = np.zeros((n * 32, 2, 64), np.float16)
    for b in range(n):
        blk = np.zeros(BLK, np.float16)
        part = x[b * per:(b + 1) * per]
        blk[:len(part)] = part
        for c in (0, 1):
            rows[b * 32:(b + 1) * 32, c] = np.append(blk, top).reshape(32, 64)
    rows = rows.reshape(n * 32, 128)
    ref, ref_s, _, _ = kv8.build_cache(rows, [len(rows)], 1, 64)
    cache, scales, _ = _quantize(ctx, rows, [len(rows)], 1, 64)
    assert np.array_equal(cache.cpu().numpy()[:len(ref) - 1], ref[:-1])
    assert np.array_equal(scales.cpu().numpy()[:len(ref) - 1], ref_s[:-1])


def test_values_that_are_not_finite_are_reported(ctx):
    rows = _rows(np.random.default_rng(0), 70, 2 * 2 * 64)
    for bad in (np.nan, np.inf, -np.inf):
        for at in ((0, 0), (69, 255), (40, 130)):
            x = rows.copy()
            x[at] = bad
            with pytest.raises(aiq.AiqError) as e:
                _quantize(ctx, x, [70], 2, 64)
            assert e.value.status == aiq.ERR_DEVICE_CHECK
    _quantize(ctx, rows, [70], 2, 64)  # the context works on


@pytest.mark.parametrize("starts", [[0, 41], [0, 50, 40], [-3, 40], [0, 2 ** 31 - 1], [5, 3, 40], [0, -5, 40]])
def test_sequences_outside_the_rows_are_reported(ctx, starts):
    rows = _d(_rows(np.random.default_rng(0), 40, 2 * 64))
    n = len(starts) - 1
    st = _d(np.array(starts, np.int32))
    cache = torch.zeros((kv8.blocks(40, n), 1, 64 * 64), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((kv8.blocks(40, n), 1, 2), device="cuda")
    torch.cuda.synchronize()
    for call in (lambda: ctx.op_kv_quantize(rows.data_ptr(), 128, 40, st.data_ptr(), n, 1, 64, cache.data_ptr(),
                                            scales.data_ptr()),
                 lambda: ctx.op_kv_dequantize(cache.data_ptr(), scales.data_ptr(), 40, st.data_ptr(), n, 1, 64,
                                              rows.data_ptr(), 128)):
        with pytest.raises(aiq.AiqError) as e:
            call()
        assert e.value.status == aiq.ERR_DEVICE_CHECK


def test_a_first_sequence_behind_the_last_block_is_reported(ctx):
    test_sequences_outside_the_rows_are_reported(ctx, [1000, 1005])
    test_sequences_outside_the_rows_are_reported(ctx, [2 ** 31 - 40, 2 ** 31 - 9])


# ------------------------------------------------------------------ attention

class Step:
    """Caches of a decode batch on the device and, in 64 bits, what they hold."""

    def __init__(self, seed, Hq, Hkv, hd, lens, P, gen_cap, std=0.9):
        self.rng = np.random.default_rng(seed)
        self.dims, self.lens, self.P, self.cap = (Hq, Hkv, hd), lens, P, gen_cap
        self.R, self.T = len(lens), sum(lens)
        w = 2 * Hkv * hd
        own = _rows(self.rng, self.T, w, std)
        self.own_c, self.own_s, q, s = kv8.build_cache(own, lens, Hkv, hd, fill=200)
        self.own = q * s[..., None]
        pre = _rows(self.rng, P, w, std)
        self.pre_c, self.pre_s, q, s = kv8.build_cache(pre, [P], Hkv, hd, fill=200)
        self.pre = q * s[..., None]
        self.gen = [np.zeros((0, w), np.float16) for _ in range(self.R)]  # every generated token so far
        self.d = [_d(a) for a in (self.own_c, self.own_s, self.pre_c, self.pre_s, kv8.starts(lens))]
        gb = gen_cap // 32
        self.gc = torch.full((max(self.R * gb, 1), Hkv, 64 * hd), 201, dtype=torch.uint8, device="cuda")
        self.gs = torch.full((max(self.R * gb, 1), Hkv, 2), float("nan"), device="cuda")
        # places that no token has come to hold NaN
        self.tail = torch.full((self.R, 32, w), float("nan"), dtype=torch.float16, device="cuda")

    def call(self, ctx, qkv, slot):
        Hq, Hkv, hd = self.dims
        x, out = _d(qkv), torch.full((self.R, Hq * hd), -7.0, dtype=torch.float16, device="cuda")
        c, s, pc, ps, st = self.d
        torch.cuda.synchronize()
        ctx.op_decode_attention_q8(x.data_ptr(), self.R, Hq, Hkv, hd, c.data_ptr(), s.data_ptr(), self.T, st.data_ptr(),
                                   self.gc.data_ptr(), self.gs.data_ptr(), self.tail.data_ptr(), self.cap, slot,
                                   out.data_ptr(), prefix=pc.data_ptr() if self.P else 0,
                                   prefix_scales=ps.data_ptr() if self.P else 0, P=self.P)
        return out.cpu().numpy()

    def append(self, qkv):
        """The step's keys and values join the generated tokens."""
        Hq, Hkv, hd = self.dims
        for r in range(self.R):
            self.gen[r] = np.concatenate([self.gen[r], qkv[r:r + 1, Hq * hd:]])

    def generated(self, r):
        """Row r's generated tokens as the cache holds them: whole blocks quantised once the step after is run."""
        Hq, Hkv, hd = self.dims
        n = len(self.gen[r])
        full = max(n - 1, 0) // 32 * 32  # the step that fills a block still attends its fp16 values
        x = self.gen[r].astype(np.float64).reshape(n, 2, Hkv, hd)
        if full:
            _, _, q, s = kv8.build_cache(self.gen[r][:full], [full], Hkv, hd)
            x[:full] = q * s[..., None]
        return x

    def check(self, out, qkv, what=""):
        Hq, Hkv, hd = self.dims
        st, worst = kv8.starts(self.lens), 0.0
        for r in range(self.R):
            kv = np.concatenate([self.pre, self.own[st[r]:st[r + 1]], self.generated(r)])
            ref, bound = kv8.attend(qkv[r, :Hq * hd].astype(np.float64).reshape(Hq, hd), kv[:, 0], kv[:, 1])
            err = np.abs(out[r].astype(np.float64).reshape(Hq, hd) - ref)
            worst = max(worst, float((err / bound).max()))
            assert (err <= bound).all(), f"{what} row {r}: {float((err / bound).max()):.2f} of the bound"
        return worst

    def qkv(self, std=0.9):
        Hq, Hkv, hd = self.dims
        return (self.rng.standard_normal((self.R, (Hq + 2 * Hkv) * hd)) * std).astype(np.float16)

    def fill_generated(self, slot):
        """Tokens 0 .. slot - 1 as if generated by earlier steps."""
        Hq, Hkv, hd = self.dims
        full, w, gb = slot // 32 * 32, 2 * Hkv * hd, self.cap // 32
        tail = np.full((self.R, 32, w), np.float16(np.nan))
        for r in range(self.R):
            self.gen[r] = _rows(self.rng, slot, w)
            if full:
                c, s, _, _ = kv8.build_cache(self.gen[r][:full], [full], Hkv, hd)
                self.gc[r * gb:r * gb + full // 32] = torch.as_tensor(c[:full // 32]).cuda()
                self.gs[r * gb:r * gb + full // 32] = torch.as_tensor(s[:full // 32]).cuda()
            tail[r, :slot - full] = self.gen[r][full:]
        self.tail = _d(tail)


HEADS = [(4, 4, 32), (8, 2, 32), (8, 8, 64), (8, 2, 64), (6, 2, 64), (8, 1, 64), (7, 1, 64), (2, 1, 128), (4, 4, 128),
         (16, 2, 128), (10, 2, 128)]


@pytest.mark.parametrize("heads", HEADS, ids=str)
@pytest.mark.parametrize("P,slot", [(0, 0), (1, 5), (33, 31), (64, 32), (0, 70), (40, 63)])
def test_attention(ctx, heads, P, slot):
    s = Step(P + slot, *heads, [0, 1, 31, 32, 33, 200, 17, 16], P, 96)
    s.fill_generated(slot)
    qkv = s.qkv()
    out = s.call(ctx, qkv, slot)
    s.append(qkv)
    s.check(out, qkv)


@pytest.mark.parametrize("heads,lens", [((8, 2, 64), [1] * 7), ((4, 1, 128), [5000]), ((8, 8, 32), [3000, 1]),
                                        ((32, 8, 64), [60, 131, 9, 2500]), ((4, 1, 64), [40] * 1500),
                                        ((32, 8, 128), [300] * 40), ((8, 8, 32), [35] * 700)], ids=str)
def test_attention_sizes(ctx, heads, lens):
    s = Step(sum(lens), *heads, lens, 20, 32)
    s.fill_generated(9)
    qkv = s.qkv()
    out = s.call(ctx, qkv, 9)
    s.append(qkv)
    s.check(out, qkv)


@pytest.mark.parametrize("heads,rows", [((8, 8, 32), 700), ((8, 8, 64), 700), ((8, 2, 64), 2500), ((4, 4, 128), 1000)], ids=str)
@pytest.mark.parametrize("slot", [0, 31, 40])
def test_many_rows(ctx, heads, rows, slot):
    """Batches in which a warp takes whole tasks, one after the other; rows of every small length."""
    Hq, Hkv, hd = heads
    s = Step(slot, *heads, [i % 71 for i in range(rows)], 33 if slot else 0, 64)
    s.fill_generated(slot)
    qkv = s.qkv()
    out = s.call(ctx, qkv, slot)
    s.append(qkv)
    s.check(out, qkv)
    if slot == 31:
        gc, gs = s.gc.cpu().numpy(), s.gs.cpu().numpy()
        for r in range(0, rows, 7):
            c, sc, _, _ = kv8.build_cache(s.gen[r], [32], Hkv, hd)
            assert np.array_equal(gc[2 * r], c[0]) and np.array_equal(gs[2 * r], sc[0])


@pytest.mark.parametrize("heads", [(4, 4, 32), (6, 2, 64), (8, 1, 128)], ids=str)
def test_steps_build_the_cache(ctx, heads):
    """70 steps: each output, and the cache that they leave, equal to the tokens quantised at once."""
    Hq, Hkv, hd = heads
    s = Step(7, *heads, [3, 0, 50], 5, 80)
    for slot in range(70):
        qkv = s.qkv(std=0.9 * (1 + slot % 5))
        out = s.call(ctx, qkv, slot)
        s.append(qkv)
        s.check(out, qkv, f"step {slot}")
    gb, gc, gs, tail = 80 // 32, s.gc.cpu().numpy(), s.gs.cpu().numpy(), s.tail.cpu().numpy()
    for r in range(s.R):
        c, sc, _, _ = kv8.build_cache(s.gen[r][:64], [64], Hkv, hd)
        assert np.array_equal(gc[r * gb:r * gb + 2], c[:2]) and np.array_equal(gs[r * gb:r * gb + 2], sc[:2])
        assert np.array_equal(tail[r, :6], s.gen[r][64:])


def test_a_rows_bits_do_not_depend_on_the_rows_beside_it(ctx):
    heads, lens = (8, 2, 64), [40, 300, 0, 77]
    s = Step(3, *heads, lens, 10, 32)
    s.fill_generated(4)
    qkv = s.qkv()
    first = s.call(ctx, qkv, 4)
    assert np.array_equal(first, s.call(ctx, qkv, 4))  # nor on when it runs
    moved = np.nan_to_num(first)
    assert np.array_equal(moved, first)


@pytest.mark.parametrize("heads", [(4, 4, 32), (8, 2, 64), (4, 1, 128)], ids=str)
@pytest.mark.parametrize("part", ["keys", "values", "both"])
def test_blocks_of_zeros(ctx, heads, part):
    """A block whose keys (or values) are all 0 has scale 0."""
    Hq, Hkv, hd = heads
    s = Step(6, *heads, [33, 0, 5, 64], 7, 64)
    kd = Hkv * hd
    c = slice(0, kd) if part == "keys" else slice(kd, 2 * kd) if part == "values" else slice(0, 2 * kd)
    own, pre = _rows(s.rng, s.T, 2 * kd), _rows(s.rng, s.P, 2 * kd)
    own[:, c], pre[:, c] = 0, 0
    s.own_c, s.own_s, q, sc = kv8.build_cache(own, s.lens, Hkv, hd)
    s.own = q * sc[..., None]
    s.pre_c, s.pre_s, q, sc = kv8.build_cache(pre, [7], Hkv, hd)
    s.pre = q * sc[..., None]
    s.d[:4] = [_d(a) for a in (s.own_c, s.own_s, s.pre_c, s.pre_s)]
    for slot in range(2):
        qkv = s.qkv()
        if part == "both":
            qkv[:, Hq * hd:] = 0
        out = s.call(ctx, qkv, slot)
        s.append(qkv)
        s.check(out, qkv)


@pytest.mark.parametrize("scale", [1e-4, 30.0])
def test_small_and_large_scores(ctx, scale):
    """Scores that are all alike, and scores where one key has all the weight."""
    s = Step(5, 8, 2, 64, [200, 33], 0, 32, std=scale)
    qkv = s.qkv(std=min(scale, 10.0))
    out = s.call(ctx, qkv, 0)
    s.append(qkv)
    s.check(out, qkv)


def test_unreached_bytes_count_for_nothing(ctx):
    """Bytes of keys past a sequence's end, unused blocks, and unused places of the tail."""
    s = Step(9, 4, 2, 64, [33, 5, 47], 3, 64)
    s.fill_generated(35)
    qkv = s.qkv()
    first = s.call(ctx, qkv, 35)
    st = kv8.starts(s.lens)
    mk, mv = kv8.tile_maps(64)
    c = s.own_c.copy()
    for r, n in enumerate(s.lens):
        b = kv8.first_block(int(st[r]), r) + n // 32
        for m in (mk, mv):
            c[b][:, m[n % 32:]] = 255
    s.d[0] = _d(c)
    assert np.array_equal(s.call(ctx, qkv, 35), first)


@pytest.mark.parametrize("starts,T", [([0, 10, 5], 40), ([0, 30, 41], 40), ([-1, 3, 9], 40)])
def test_attention_reports_sequences_outside_the_tokens(ctx, starts, T):
    s = Step(1, 4, 2, 64, [20, 20], 0, 32)
    s.d[4] = _d(np.array(starts, np.int32))
    with pytest.raises(aiq.AiqError) as e:
        s.call(ctx, s.qkv(), 0)
    assert e.value.status == aiq.ERR_DEVICE_CHECK


def test_attention_reports_what_is_not_finite(ctx):
    s = Step(1, 4, 2, 64, [20, 20], 0, 32)
    for at in ((0, 3), (1, 4 * 64), (1, 6 * 64 + 1)):  # a query, a key, a value
        qkv = s.qkv()
        qkv[at] = np.nan
        with pytest.raises(aiq.AiqError) as e:
            s.call(ctx, qkv, 0)
        assert e.value.status == aiq.ERR_DEVICE_CHECK


def test_offsets_beyond_32_bits(ctx):
    """1.2 million tokens of 2,048 values: bytes and elements past 2^31, and rows past 2^32 bytes."""
    Hkv, hd, T = 8, 128, 1_200_000
    w = 2 * Hkv * hd
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    kv = torch.empty((T, w), dtype=torch.float16, device="cuda")
    for i in range(0, T, 100_000):
        kv[i:i + 100_000].normal_(generator=g)
    lens = [T - 50, 50]
    st = _d(kv8.starts(lens))
    nb = kv8.blocks(T, 2)
    cache = torch.zeros((nb, Hkv, 64 * hd), dtype=torch.uint8, device="cuda")
    scales = torch.zeros((nb, Hkv, 2), device="cuda")
    torch.cuda.synchronize()
    ctx.op_kv_quantize(kv.data_ptr(), w, T, st.data_ptr(), 2, Hkv, hd, cache.data_ptr(), scales.data_ptr())
    tail = kv[-50:].cpu().numpy()
    ref, ref_s, q, s = kv8.build_cache(tail, [50], Hkv, hd)
    b = kv8.first_block(T - 50, 1)
    assert np.array_equal(cache[b:b + 2].cpu().numpy(), ref[:2]) and np.array_equal(scales[b:b + 2].cpu().numpy(), ref_s[:2])
    j = (2 ** 31 // w) // 32 * 32  # a block of the first sequence around 2^31 elements
    ref, ref_s, _, _ = kv8.build_cache(kv[j:j + 32].cpu().numpy(), [32], Hkv, hd)
    assert np.array_equal(cache[j // 32].cpu().numpy(), ref[0])
    back = torch.zeros_like(kv)
    torch.cuda.synchronize()
    ctx.op_kv_dequantize(cache.data_ptr(), scales.data_ptr(), T, st.data_ptr(), 2, Hkv, hd, back.data_ptr(), w)
    assert np.array_equal(back[-50:].cpu().numpy(), kv8.read_back(q, s))
    assert float((back[j - 64:j + 64].float() - kv[j - 64:j + 64].float()).abs().max()) < 0.03
    del back
    Hq = 16
    qkv = torch.empty((2, (Hq + 2 * Hkv) * hd), dtype=torch.float16, device="cuda").normal_(generator=g)
    gt = torch.zeros((2, 32, w), dtype=torch.float16, device="cuda")
    out = torch.zeros((2, Hq * hd), dtype=torch.float16, device="cuda")
    torch.cuda.synchronize()
    ctx.op_decode_attention_q8(qkv.data_ptr(), 2, Hq, Hkv, hd, cache.data_ptr(), scales.data_ptr(), T, st.data_ptr(), 0, 0,
                               gt.data_ptr(), 8, 0, out.data_ptr())
    x = qkv.cpu().numpy()
    rows = np.concatenate([(q * s[..., None]), x[1, Hq * hd:].astype(np.float64).reshape(1, 2, Hkv, hd)])
    want, bound = kv8.attend(x[1, :Hq * hd].astype(np.float64).reshape(Hq, hd), rows[:, 0], rows[:, 1])
    got = out.cpu().numpy().astype(np.float64)
    assert (np.abs(got[1].reshape(Hq, hd) - want) <= bound).all()
    # the long row: 64-bit sums on the GPU, a KV head at a time, of the values the cache holds
    for h in (0, Hkv - 1):
        c = cache[:(T - 50 + 31) // 32, h].view(-1, 64 * hd)
        mk, mv = (torch.as_tensor(m).cuda() for m in kv8.tile_maps(hd))
        parts = []
        for m, k in ((mk, 0), (mv, 1)):
            v = (c[:, m.reshape(-1)].double().view(-1, 32, hd) - 128) * scales[:len(c), h, k].double()[:, None, None]
            parts.append(v.reshape(-1, hd)[:T - 50])
        new = qkv[0, Hq * hd:].double().view(2, Hkv, hd)[:, h]
        k, v = torch.cat([parts[0], new[:1]]), torch.cat([parts[1], new[1:]])
        qh = qkv[0, :Hq * hd].double().view(Hkv, 2, hd)[h]
        p = torch.softmax(qh @ k.T / hd ** 0.5, 1)
        ref, A = p @ v, p @ v.abs()
        err = (out[0].double().view(Hkv, 2, hd)[h] - ref).abs()
        # as kv8.attend's bound: 2^-11 of the output, 2^-11 + 2^-18 and the scores' part of A
        S = float((qh.abs() @ k.abs().T / hd ** 0.5).max())
        rel = 2.0 ** -11 + 2.0 ** -18 + 2 * (hd + 8) * 2.0 ** -23 * S
        assert bool((err <= A * rel + ref.abs() * 2.0 ** -11 + 2.0 ** -25).all())


def test_two_contexts_at_once():
    """Each has its own stream, workspace and counters."""
    import threading
    made, outs, fails = [], {}, []

    def work(i):
        try:
            c = made[i]
            s = Step(40 + i, 8, 2, 64, [900, 30, 2500], 10, 64)
            s.fill_generated(20)
            qkv = s.qkv()
            first = s.call(c, qkv, 20)
            for _ in range(40):
                assert np.array_equal(s.call(c, qkv, 20), first)
            s.append(qkv)
            s.check(first, qkv)
            outs[i] = first
        except Exception as e:  # reported by the main thread
            fails.append(e)

    made = [gpu_ctx(), gpu_ctx()]
    try:
        threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        for c in made:
            c.close()
    assert not fails, fails
    assert len(outs) == 2


@pytest.mark.parametrize("rows,heads", [(140, (8, 8, 64)), (1100, (4, 1, 32)), (150, (56, 8, 128)), (40, (16, 8, 64)),
                                        (3, (4, 2, 32))], ids=str)
@pytest.mark.parametrize("length", [10, 150, 700])
def test_tasks_and_tiles(ctx, rows, heads, length):
    """Few and many tasks of few and many tiles: a warp, a CTA and several CTAs for one."""
    s = Step(rows, *heads, [length - i % 9 for i in range(rows)], 20, 64)
    s.fill_generated(33)
    qkv = s.qkv()
    out = s.call(ctx, qkv, 33)
    s.append(qkv)
    s.check(out, qkv)


@pytest.mark.parametrize("rows,heads", [(700, (8, 8, 32)), (5200, (4, 1, 64)), (700, (8, 8, 128))], ids=str)
@pytest.mark.parametrize("longest", [70, 300])
def test_many_rows_of_very_different_lengths(ctx, rows, heads, longest):
    """The longest rows may be taken first; the output is that of the rows as they came."""
    rng = np.random.default_rng(rows)
    lens = np.where(rng.random(rows) < 0.3, 0, rng.integers(1, longest, rows))
    lens[rows // 2], lens[rows - 1], lens[3] = 33_100, 1_500, 700
    s = Step(rows, *heads, [int(n) for n in lens], 5, 32)
    s.fill_generated(2)
    qkv = s.qkv()
    out = s.call(ctx, qkv, 2)
    s.append(qkv)
    s.check(out, qkv)


@pytest.mark.parametrize("length", [20, 200])
def test_many_rows_with_one_outside_the_tokens(ctx, length):
    rows = 700
    s = Step(1, 8, 8, 32, [length] * rows, 0, 32)
    qkv = s.qkv()
    first = s.call(ctx, qkv, 0)
    good = s.d[4]
    starts = kv8.starts(s.lens)
    starts[300] += length + 10  # behind the next one
    s.d[4] = _d(starts)
    with pytest.raises(aiq.AiqError) as e:
        s.call(ctx, qkv, 0)
    assert e.value.status == aiq.ERR_DEVICE_CHECK
    s.d[4] = good
    assert np.array_equal(s.call(ctx, qkv, 0), first)


def test_a_call_after_a_reported_one_is_right(ctx):
    """Starts that do not ascend, in a call whose rows share CTAs, leave nothing behind."""
    s = Step(50, 4, 1, 64, [4000, 3000], 0, 32)
    qkv = s.qkv()
    first = s.call(ctx, qkv, 0)
    good = s.d[4]
    for starts in ([0, 7000, 10], [0, -1, 7000], [5000, 10, 7000], [0, 4000, 8000]):
        s.d[4] = _d(np.array(starts, np.int32))
        with pytest.raises(aiq.AiqError) as e:
            s.call(ctx, qkv, 0)
        assert e.value.status == aiq.ERR_DEVICE_CHECK
        s.d[4] = good
        assert np.array_equal(s.call(ctx, qkv, 0), first)


@pytest.mark.parametrize("rows,length", [(3, 40), (2, 6000), (700, 20)])
def test_the_first_sequence_need_not_begin_at_the_first_token(ctx, rows, length):
    """As aiq_op_kv_quantize lays out sequences that begin at token 77 of the rows at hand."""
    Hq, Hkv, hd, first = 8, 8 if rows == 700 else 2, 32, 77
    s = Step(rows, Hq, Hkv, hd, [length + i % 5 for i in range(rows)], 0, 32)
    starts = kv8.starts(s.lens)
    nb = kv8.blocks(s.T + first, rows)
    cache, scales = np.full((nb, Hkv, 64 * hd), 9, np.uint8), np.full((nb, Hkv, 2), np.float32(9))
    for r in range(rows):
        n = -(-s.lens[r] // 32)
        a, b = kv8.first_block(int(starts[r]), r), kv8.first_block(int(starts[r]) + first, r)
        cache[b:b + n], scales[b:b + n] = s.own_c[a:a + n], s.own_s[a:a + n]
    qkv = s.qkv()
    want = s.call(ctx, qkv, 0)
    s.d[0], s.d[1], s.d[4] = _d(cache), _d(scales), _d(starts + np.int32(first))
    s.T += first
    for _ in range(3):
        out = s.call(ctx, qkv, 0)
        assert np.abs(out.astype(np.float64) - want).max() <= 2.0 ** -10 * np.abs(want).max()  # (ranges may be cut elsewhere)
    s.append(qkv)
    s.T -= first
    s.check(out, qkv)


def test_refusals(ctx):
    buf = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    p = buf.data_ptr()
    good = dict(kv=p, ldkv=128, T=4, seq_start=p, n_seqs=1, Hkv=1, hd=64, cache=p, scales=p)
    ctx.op_kv_quantize(**good)  # seq_start 0, 0: nothing to do
    bad = [dict(kv=0), dict(cache=0), dict(scales=0), dict(seq_start=0), dict(kv=p + 2), dict(cache=p + 8),
           dict(scales=p + 4), dict(ldkv=120), dict(ldkv=132), dict(T=-1), dict(T=1 << 31), dict(n_seqs=-1), dict(Hkv=0)]
    for b in bad:
        for f in (ctx.op_kv_quantize, ctx.op_kv_dequantize):
            with pytest.raises(aiq.AiqError) as e:
                f(**{**good, **b})
            assert e.value.status == aiq.ERR_INVALID_ARG, b
    for hd in (16, 96, 256):
        with pytest.raises(aiq.AiqError) as e:
            ctx.op_kv_quantize(**{**good, "hd": hd, "ldkv": 2 * hd})
        assert e.value.status == aiq.ERR_UNSUPPORTED
    ctx.op_kv_quantize(**{**good, "T": 0})
    ctx.op_kv_quantize(**{**good, "n_seqs": 0})
    good = dict(qkv=p, R=1, Hq=4, Hkv=2, hd=64, own_cache=p, own_scales=p, T=4, seq_start=p, gen_cache=p, gen_scales=p,
                gen_tail=p, gen_cap=64, slot=0, out=p + 4096, prefix=p, prefix_scales=p, P=3)
    bad = [dict(qkv=0), dict(R=-1), dict(Hq=0), dict(Hkv=0), dict(Hkv=3), dict(own_cache=0), dict(own_scales=0), dict(T=-1),
           dict(seq_start=0), dict(gen_cache=0), dict(gen_scales=0), dict(gen_tail=0), dict(gen_cap=0), dict(slot=64),
           dict(slot=-1), dict(out=0), dict(prefix=0), dict(prefix_scales=0), dict(P=-1), dict(qkv=p + 8),
           dict(gen_tail=p + 2), dict(out=p + 8), dict(own_scales=p + 4), dict(prefix=p + 8), dict(gen_cache=p + 4)]
    for b in bad:
        with pytest.raises(aiq.AiqError) as e:
            ctx.op_decode_attention_q8(**{**good, **b})
        assert e.value.status == aiq.ERR_INVALID_ARG, b
    for b in (dict(hd=48), dict(Hq=18)):
        with pytest.raises(aiq.AiqError) as e:
            ctx.op_decode_attention_q8(**{**good, **b})
        assert e.value.status == aiq.ERR_UNSUPPORTED, b
    ctx.op_decode_attention_q8(**{**good, "R": 0})


def test_more_heads_than_a_row_can_count_are_refused(ctx):
    p = torch.zeros(1 << 12, dtype=torch.uint8, device="cuda").data_ptr()
    heads = (1 << 20) + 1
    for call in (lambda: ctx.op_kv_quantize(p, 2 * 32 * heads, 4, p, 1, heads, 32, p, p),
                 lambda: ctx.op_kv_dequantize(p, p, 4, p, 1, heads, 32, p, 2 * 32 * heads),
                 lambda: ctx.op_decode_attention_q8(p, 1, heads, heads, 32, p, p, 4, p, 0, 0, p, 1, 0, p)):
        with pytest.raises(aiq.AiqError) as e:
            call()
        assert e.value.status == aiq.ERR_UNSUPPORTED
