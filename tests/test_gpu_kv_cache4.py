"""The 4-bit key/value cache (quantised as it is written, read back, attended and appended
to by a generation step, its prompts shared by beams) against its definition in 64 bits,
through the C-ABI (aiq_ops.h)."""
import numpy as np
import pytest

import kv4
from helpers import gpu_ctx
from kv8 import blocks, starts
from paper_2608_10139_gb300 import aiq

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

LENGTHS = [
    [1], [31], [32], [33], [64, 1], [0, 0, 5], [100, 0, 32, 31, 33, 0, 1], [7] * 45 + [200], [0, 0],
]
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
    s = np.repeat(np.exp(rng.normal(0, 1, -(-n // 16) if n else 0)), 16)[:n]
    return (rng.standard_normal((n, width)) * std * s[:, None]).astype(np.float16)


def _quantize(ctx, rows, lens, Hkv, hd, T=None, pad=0, fill=7):
    T = len(rows) if T is None else T
    width = 2 * Hkv * hd
    buf = np.full((max(T, 1), width + pad), np.float16(np.nan))
    buf[:T, pad:] = rows[:T]
    kv, st = _d(buf), _d(starts(lens))
    nb = blocks(T, len(lens))
    cache = torch.full((max(nb, 1), Hkv, kv4.tile_bytes(hd)), fill, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    ctx.op_kv_quantize4(kv.data_ptr() + 2 * pad, width + pad, T, st.data_ptr(), len(lens), Hkv, hd, cache.data_ptr())
    return cache, st


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("Hkv", [1, 3, 8])
@pytest.mark.parametrize("lens", LENGTHS, ids=lambda v: f"{len(v)}x{sum(v)}")
def test_quantize_is_exact(ctx, hd, Hkv, lens):
    rng = np.random.default_rng(hd * 10 + Hkv)
    T = sum(lens) + 3  # rows behind the last sequence
    rows = _rows(rng, T, 2 * Hkv * hd)
    rows[sum(lens):] = np.nan  # are not read
    n = sum(lens)
    ref, mask, q, s, m = kv4.build_cache(rows[:n], lens, Hkv, hd, T=T, fill=7)
    cache, st = _quantize(ctx, rows, lens, Hkv, hd, T=T, pad=8 * Hkv)
    got = cache.cpu().numpy()[:len(ref)]
    assert np.array_equal(got[mask], ref[mask])
    untouched = ~mask.any((1, 2))
    assert (got[untouched] == 7).all()
    # and back, into rows with a pitch; what lies beside and behind them stays
    back = torch.full((T, 2 * Hkv * hd + 16), 3.0, dtype=torch.float16, device="cuda")
    torch.cuda.synchronize()
    ctx.op_kv_dequantize4(cache.data_ptr(), T, st.data_ptr(), len(lens), Hkv, hd, back.data_ptr() + 16, 2 * Hkv * hd + 16)
    b = back.cpu().numpy()
    assert np.array_equal(b[:n, 8:-8], kv4.read_back(q, s, m).reshape(n, 2 * Hkv * hd))
    assert (b[n:] == 3).all() and (b[:, :8] == 3).all() and (b[:, -8:] == 3).all()


@pytest.mark.parametrize("lens", MANY, ids=lambda v: f"{len(v)}x{sum(v)}")
def test_many_sequences(ctx, lens):
    rng = np.random.default_rng(len(lens))
    rows = _rows(rng, sum(lens), 2 * 32)
    ref, mask, *_ = kv4.build_cache(rows, lens, 1, 32)
    cache, _ = _quantize(ctx, rows, lens, 1, 32)
    assert np.array_equal(cache.cpu().numpy()[:len(ref)][mask], ref[mask])


def _special(rng, n, kind, width):
    if kind == "halves":       # ranges of 15, 30 and 60: every border is a number that is there
        x = rng.integers(-30, 31, (n, width)) * 0.5 * 2.0 ** rng.integers(-10, 8, (n, 1))
    elif kind == "subnormal":
        x = rng.integers(-40, 41, (n, width)) * 2.0 ** -24
    elif kind == "whole range":
        x = rng.choice([-65504, 65504, 0, 1, -1, 2.0 ** -24, -2.0 ** -24, 4367, -32752], (n, width))
    elif kind == "far apart":  # the difference of such numbers has more than 24 bits
        x = np.where(rng.random((n, width)) < 0.5, rng.choice([-1000.0, -1.0, 15, 500], (n, width)),
                     rng.integers(-3, 4, (n, width)) * 2.0 ** -24)
        x[:, 0] = np.where(rng.random(n) < 0.5, -1000, -7.5)
    elif kind == "constant":
        x = np.repeat(rng.standard_normal((n, 1)), width, 1)
    else:                      # next to borders: neighbours of (n + 1/2) s
        s = np.float64(np.float16(rng.random(1)[0] + 0.1))
        x = (rng.integers(0, 15, (n, width)) + 0.5) * s
        x = np.nextafter(x.astype(np.float16), rng.choice([np.float16(-np.inf), np.float16(np.inf)], (n, width)))
        x[:, 0::64], x[:, 1::64] = 0, 15 * s
        x[:, 32::64], x[:, 33::64] = 0, 15 * s
    return x.astype(np.float16)


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("kind", ["halves", "subnormal", "whole range", "far apart", "constant", "borders"])
def test_codes_at_the_borders(ctx, hd, kind):
    rng = np.random.default_rng(hd)
    rows = _special(rng, 500, kind, 2 * 2 * hd)
    ref, mask, q, s, m = kv4.build_cache(rows, [500], 2, hd)
    cache, st = _quantize(ctx, rows, [500], 2, hd)
    assert np.array_equal(cache.cpu().numpy()[:len(ref)][mask], ref[mask])
    back = torch.zeros((500, 4 * hd), dtype=torch.float16, device="cuda")
    torch.cuda.synchronize()
    ctx.op_kv_dequantize4(cache.data_ptr(), 500, st.data_ptr(), 1, 2, hd, back.data_ptr(), 4 * hd)
    assert np.array_equal(back.cpu().numpy(), kv4.read_back(q, s, m).reshape(500, -1))


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
def test_what_is_not_finite_is_reported(ctx, hd, value):
    rng = np.random.default_rng(1)
    for at in (3, 2 * hd - 1):
        rows = _rows(rng, 40, 2 * hd)
        rows[37, at] = value
        with pytest.raises(aiq.AiqError) as e:
            _quantize(ctx, rows, [40], 1, hd)
        assert e.value.status == aiq.ERR_DEVICE_CHECK
    _quantize(ctx, _rows(rng, 40, 2 * hd), [40], 1, hd)


@pytest.mark.parametrize("start", [[0, 50], [-1, 5], [5, 3], [50, 60], [0, 20, 10, 30]])
def test_bad_sequences_are_reported(ctx, start):
    kv = torch.zeros((40, 128), dtype=torch.float16, device="cuda")
    st = _d(np.array(start, np.int32))
    cache = torch.zeros((blocks(40, len(start) - 1), 1, kv4.tile_bytes(64)), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    with pytest.raises(aiq.AiqError) as e:
        ctx.op_kv_quantize4(kv.data_ptr(), 128, 40, st.data_ptr(), len(start) - 1, 1, 64, cache.data_ptr())
    assert e.value.status == aiq.ERR_DEVICE_CHECK
    with pytest.raises(aiq.AiqError) as e:
        ctx.op_kv_dequantize4(cache.data_ptr(), 40, st.data_ptr(), len(start) - 1, 1, 64, kv.data_ptr(), 128)
    assert e.value.status == aiq.ERR_DEVICE_CHECK


# --------------------------------------------------------------- attention ---

class Batch:
    """A decode batch on the 4-bit cache, on the device and (codes and pairs by token) here."""

    def __init__(self, ctx, rng, hd, Hq, Hkv, beams, lens, P, gen_cap, std=0.9, fill=85, extra=0):
        self.ctx, self.hd, self.Hq, self.Hkv, self.beams, self.lens, self.P, self.gen_cap = ctx, hd, Hq, Hkv, beams, lens, P, gen_cap
        self.R, w = beams * len(lens), 2 * Hkv * hd
        T = sum(lens)
        self.T = T + extra
        self.own = _rows(rng, T, w, std)
        self.prefix = _rows(rng, P, w, std)
        cache, mask, *self.own4 = kv4.build_cache(self.own, lens, Hkv, hd, T=self.T, fill=fill)
        cache[~mask] = rng.integers(0, 256, int((~mask).sum()))  # what no key holds may be anything
        self.d_own, self.st = _d(cache), _d(starts(lens))
        cache, mask, *self.prefix4 = kv4.build_cache(self.prefix, [P], Hkv, hd)
        cache[~mask] = rng.integers(0, 256, int((~mask).sum()))
        self.d_prefix = _d(cache) if P else None
        self.gb = -(-gen_cap // 32)
        self.gen = _d(rng.integers(0, 256, (self.R, self.gb, Hkv, kv4.tile_bytes(hd)), dtype=np.uint8))
        # the guard behind the cache
        self.guard = torch.full((self.R * self.gb + 1, Hkv, kv4.tile_bytes(hd)), 0, dtype=torch.uint8, device="cuda")
        self.guard[:-1] = self.gen.view(-1, Hkv, kv4.tile_bytes(hd))
        self.guard[-1] = 77
        self.gen = self.guard[:-1].view(self.R, self.gb, Hkv, -1)
        self.gen4 = [[] for _ in range(self.R)]
        self.out = torch.full((self.R + 1, Hq * hd), 9.0, dtype=torch.float16, device="cuda")
        self.held = torch.full((self.R + 1, w), 9.0, dtype=torch.float16, device="cuda")
        torch.cuda.synchronize()

    def step(self, qkv, slot, held=True):
        d = _d(qkv)
        self.ctx.op_decode_attention_q4(d.data_ptr(), self.R, self.Hq, self.Hkv, self.hd, self.d_own.data_ptr(), self.T,
                                        self.st.data_ptr(), self.gen.data_ptr(), self.gen_cap, slot, self.out.data_ptr(),
                                        beams=self.beams, prefix=self.d_prefix.data_ptr() if self.P else 0, P=self.P,
                                        held=self.held.data_ptr() if held else 0)
        out, h = self.out.cpu().numpy(), self.held.cpu().numpy()
        assert (out[self.R] == 9).all() and (h[self.R] == 9).all() and (self.guard[-1] == 77).all()
        return out[:self.R], h[:self.R]

    def seen(self, r, slot):
        """(values [n, 2, Hkv, hd], largest |m| + 15 s [n, 2, Hkv]) that row r attends up to `slot`."""
        i = r // self.beams
        a, b = int(starts(self.lens)[i]), int(starts(self.lens)[i + 1])
        parts = [self.prefix4, [x[a:b] for x in self.own4]] + self.gen4[r][:slot + 1]
        n, s, m = (np.concatenate([p[j] for p in parts]) for j in range(3))
        return kv4.values(n, s, m), (np.abs(m.astype(np.float64)) + 15 * s.astype(np.float64)).max(-1)

    def check(self, rng, slots, std=0.9, qstd=0.9, rows=None):
        w = (self.Hq + 2 * self.Hkv) * self.hd
        for slot in slots:
            qkv = _rows(rng, self.R, w, std)
            qkv[:, :self.Hq * self.hd] = (rng.standard_normal((self.R, self.Hq * self.hd)) * qstd).astype(np.float16)
            new = kv4.quantize(qkv[:, self.Hq * self.hd:].reshape(self.R, 1, 2, self.Hkv, self.hd))
            out, held = self.step(qkv, slot)
            for r in range(self.R):
                del self.gen4[r][slot:]
                self.gen4[r].append([x[r] for x in new])
            assert np.array_equal(held, kv4.read_back(*new).reshape(self.R, -1))
            for r in range(self.R) if rows is None else rows:
                x, big = self.seen(r, slot)
                ref, tol = kv4.attend(qkv[r, :self.Hq * self.hd].astype(np.float64).reshape(self.Hq, self.hd),
                                      x[:, 0], x[:, 1], big[:, 0], big[:, 1])
                err = np.abs(out[r].astype(np.float64).reshape(self.Hq, self.hd) - ref)
                assert (err <= tol).all(), f"slot {slot} row {r}: {(err / tol).max()}"

    def cached(self, slots):
        """The generated tokens as the cache holds them."""
        for r in range(self.R):
            got = self.gen[r].cpu().numpy()
            for slot in range(slots):
                n, s, m = self.gen4[r][slot]
                at, pairs = kv4.maps(self.hd)
                tile = got[slot // 32]
                key = slot % 32
                for v in (0, 1):
                    code = tile[:, at[v][key, :, 0]] >> at[v][key, :, 1] & 15
                    assert np.array_equal(code, n[0, v])
                    pair = np.stack([tile[:, pairs[v][key] + i] for i in range(4)], -1)
                    pair = np.ascontiguousarray(pair).view(np.float16)
                    assert np.array_equal(pair[..., 0], s[0, v]) and np.array_equal(pair[..., 1], m[0, v])


HEADS = [(4, 4), (8, 2), (8, 1), (3, 1), (6, 2), (10, 2), (14, 2)]


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("Hq,Hkv", HEADS)
@pytest.mark.parametrize("beams", [1, 2, 3])
def test_attention(ctx, hd, Hq, Hkv, beams):
    rng = np.random.default_rng(hd + Hq * 8 + beams)
    b = Batch(ctx, rng, hd, Hq, Hkv, beams, [5, 0, 33, 64, 130], 17, 70, extra=9)
    b.check(rng, [0, 1, 2])
    b.cached(3)


@pytest.mark.parametrize("hd,beams", [(32, 1), (64, 1), (128, 1), (64, 4), (128, 5), (32, 8), (64, 16)])
def test_attention_over_many_steps(ctx, hd, beams):
    """Slots 0 .. 66, past two borders of blocks, in order."""
    rng = np.random.default_rng(hd + beams)
    b = Batch(ctx, rng, hd, 4, 2, beams, [3, 40], 0, 67)
    b.check(rng, range(67), rows=[0, beams, 2 * beams - 1])
    b.cached(67)


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("lens,P", [([0], 0), ([0, 0, 0], 0), ([0, 0], 1), ([1], 32), ([32], 0), ([31, 33], 31), ([1000], 100)])
@pytest.mark.parametrize("beams", [1, 4])
def test_lengths(ctx, hd, lens, P, beams):
    """Nothing but the step's own token, blocks full and not, prompts of nothing."""
    rng = np.random.default_rng(hd + len(lens))
    b = Batch(ctx, rng, hd, 8, 2, beams, lens, P, 1)
    b.check(rng, [0])


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("lens,beams", [([20000], 1), ([9000, 3, 300], 1), ([5000, 100], 3), ([700] * 40, 1), ([40000, 1] + [5] * 60, 1)])
def test_long_and_uneven_prompts(ctx, hd, lens, beams):
    rng = np.random.default_rng(hd + len(lens))
    b = Batch(ctx, rng, hd, 4, 1, beams, lens, 50, 40)
    b.check(rng, [0], rows=[0, b.R // 2, b.R - 1])
    b.gen4 = [g * 1 for g in b.gen4]
    b.check(rng, [1], rows=[0, b.R - 1])


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("rows,beams", [(700, 1), (1500, 1), (400, 4), (300, 5), (2600, 1)])
def test_many_rows(ctx, hd, rows, beams):
    rng = np.random.default_rng(rows + hd)
    lens = [int(x) for x in rng.integers(0, 120, rows)]
    lens[rows // 2] = 900
    b = Batch(ctx, rng, hd, 8, 8 if hd == 32 else 2, beams, lens, 40, 33)
    for g in b.gen4:  # a first token that is there already
        del g[:]
    b.check(rng, [0], rows=rng.choice(b.R, 60, replace=False).tolist() + [rows // 2 * beams, b.R - 1])


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("std,qstd", [(1e-6, 1e-6), (1e-3, 30.0), (20.0, 20.0), (2000.0, 1e-4), (1e-3, 6e4), (0.9, 0.0)])
def test_magnitudes(ctx, hd, std, qstd):
    """Keys, values and queries from subnormal numbers to the type's largest."""
    rng = np.random.default_rng(7)
    b = Batch(ctx, rng, hd, 4, 2, 2, [70, 0], 33, 33, std=std)
    b.own4 = [x for x in b.own4]
    w = (4 + 4) * hd
    for slot in (0, 1):
        qkv = (rng.standard_normal((b.R, w)) * std).clip(-65504, 65504).astype(np.float16)
        qkv[:, :4 * hd] = (rng.standard_normal((b.R, 4 * hd)) * qstd).clip(-65504, 65504)
        new = kv4.quantize(qkv[:, 4 * hd:].reshape(b.R, 1, 2, 2, hd))
        out, held = b.step(qkv, slot)
        assert np.array_equal(held, kv4.read_back(*new).reshape(b.R, -1))
        for r in range(b.R):
            b.gen4[r].append([x[r] for x in new])
            x, big = b.seen(r, slot)
            ref, tol = kv4.attend(qkv[r, :4 * hd].astype(np.float64).reshape(4, hd), x[:, 0], x[:, 1], big[:, 0], big[:, 1])
            assert (np.abs(out[r].astype(np.float64).reshape(4, hd) - ref) <= tol).all()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("beams", [1, 2])
def test_many_light_keys_behind_a_heavy_one(ctx, hd, beams):
    """One key outweighs each of the others by 2^18; together they weigh as much as it."""
    rng = np.random.default_rng(3)
    n = 1 << 18
    own = np.zeros((n, 2, 1, hd), np.float16)
    own[:, 1, 0] = 1.0
    own[0, 0, 0] = 1.0
    own[0, 1, 0] = -1.0
    b = Batch(ctx, rng, hd, 1, 1, beams, [1], 0, 1)
    d = _d(own.reshape(n, 2 * hd))
    st = _d(np.array([0, n], np.int32))
    cache = torch.zeros((n // 32 + 1, 1, kv4.tile_bytes(hd)), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    ctx.op_kv_quantize4(d.data_ptr(), 2 * hd, n, st.data_ptr(), 1, 1, hd, cache.data_ptr())
    b.d_own, b.st, b.T = cache, st, n
    qkv = np.zeros((b.R, 3 * hd), np.float16)
    score = 18 * np.log(2) * np.sqrt(hd) / hd
    qkv[:, :hd] = score
    out, _ = b.step(qkv, 0)
    p = np.exp(float(np.float16(score)) * hd / np.sqrt(hd))
    ref = (n - 1 - p) / (n + p)  # (the step's own key weighs 1, its value 0)
    # 2^-18 for sums and exponentials over values of size 1, 2 (hd + 16) 2^-23 S with S <= 13, fp16's rounding
    assert np.abs(out.astype(np.float64) - ref).max() <= 2.0 ** -18 + 2 * (hd + 16) * 2.0 ** -23 * 13 + 2.0 ** -11 * abs(ref) + 2.0 ** -24


def test_a_row_outside_the_tokens_is_reported_and_the_others_written(ctx):
    rng = np.random.default_rng(5)
    b = Batch(ctx, rng, 64, 4, 2, 1, [20, 20, 20], 0, 4)
    b.st[2] = 7  # sequence 1 ends before it begins, sequence 2 is longer than it was
    qkv = _rows(rng, 3, 8 * 64)
    with pytest.raises(aiq.AiqError) as e:
        b.step(qkv, 0)
    assert e.value.status == aiq.ERR_DEVICE_CHECK
    b.st[2] = 40
    b.check(rng, [0])
    b.st[3] = 1000
    with pytest.raises(aiq.AiqError) as e:
        b.step(qkv, 1)
    assert e.value.status == aiq.ERR_DEVICE_CHECK


@pytest.mark.parametrize("value", [np.nan, np.inf])
@pytest.mark.parametrize("where", ["query", "key", "value"])
def test_inputs_that_are_not_finite_are_reported(ctx, value, where):
    rng = np.random.default_rng(5)
    b = Batch(ctx, rng, 64, 4, 2, 1, [20, 20], 0, 4)
    qkv = _rows(rng, 2, 8 * 64)
    qkv[1, {"query": 100, "key": 4 * 64 + 70, "value": 6 * 64 + 127}[where]] = value
    with pytest.raises(aiq.AiqError) as e:
        b.step(qkv, 0)
    assert e.value.status == aiq.ERR_DEVICE_CHECK
    b.check(rng, [0])


def test_equal_calls_give_equal_bits(ctx):
    rng = np.random.default_rng(11)
    for lens, beams in (([3000, 17], 2), ([50] * 800, 1)):
        b = Batch(ctx, rng, 64, 8, 2, beams, lens, 20, 40)
        qkv = _rows(rng, b.R, 12 * 64)
        one, _ = b.step(qkv, 0)
        for _ in range(5):
            assert np.array_equal(one, b.step(qkv, 0, held=False)[0])
