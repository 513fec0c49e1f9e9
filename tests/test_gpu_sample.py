"""The sampling of tokens (temperature, top-k, top-p, min-p from given uniforms)
against its definition in 64 bits: equal tokens, and probabilities to their rounding."""
import numpy as np
import pytest

import kv8
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


def _run(ctx, z, u, type="f32", ld=None, offset=0, **kw):
    """z [R, V] fp32 values, stored as `type` at a pitch of ld elements, `offset` elements into their buffer."""
    code, dt = TYPES[type]
    R, V = z.shape
    ld = ld or V
    buf = torch.full((R * ld + offset + 8,), float("nan"), dtype=dt, device="cuda")
    view = buf[offset:offset + R * ld].view(R, ld)
    view[:, :V] = torch.as_tensor(z).cuda().to(dt)
    held = view[:, :V].float().cpu().numpy()
    du = torch.as_tensor(np.asarray(u, np.float32)).cuda()
    tok = torch.full((R + 1,), -9, dtype=torch.int32, device="cuda")
    prob = torch.full((R + 1,), -9.0, device="cuda")
    torch.cuda.synchronize()
    ctx.op_sample(view.data_ptr(), code, ld, R, V, du.data_ptr(), tok.data_ptr(), probs=prob.data_ptr(), **kw)
    t, p = tok.cpu().numpy(), prob.cpu().numpy()
    assert t[R] == -9 and p[R] == -9
    return held, t[:R], p[:R]


def _check(held, u, t, p, temperature=1.0, top_k=50, top_p=1.0, min_p=0.0):
    for r in range(len(held)):
        tok, prob = kv8.sample(held[r], u[r], temperature, top_k, top_p, min_p)
        assert t[r] == tok, f"row {r}: {t[r]}, not {tok}"
        # exponentials and sums in 64 bits, one rounding to 32
        assert abs(p[r] - prob) <= prob * 2.0 ** -24 * 1.01 + 1e-45


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("R,V,top_k", [(1, 1, 1), (3, 2, 2), (2, 5, 3), (7, 31, 31), (5, 33, 8), (4, 1000, 50),
                                       (33, 4096, 40), (3, 4097, 1024), (5, 32000, 50), (2, 32001, 700),
                                       (3, 128256, 1000), (1, 128256, 1), (2, 300001, 64), (200, 1500, 20)])
@pytest.mark.parametrize("kw", [dict(), dict(temperature=0.6, top_p=0.9), dict(temperature=1.7, min_p=0.05, top_p=0.7)],
                         ids=str)
def test_tokens(ctx, type, R, V, top_k, kw):
    rng = np.random.default_rng(R * V + top_k)
    z = (rng.standard_normal((R, V)) * np.exp(rng.normal(0, 0.7, (R, 1)))).astype(np.float32)
    u = rng.random(R).astype(np.float32)
    u = np.minimum(u, np.float32(1 - 2.0 ** -24))
    held, t, p = _run(ctx, z, u, type, top_k=top_k, **kw)
    _check(held, u, t, p, top_k=top_k, **kw)


@pytest.mark.parametrize("type", list(TYPES))
@pytest.mark.parametrize("ld,offset", [(1003, 0), (1003, 1), (1008, 3), (1001, 7), (2048, 5)])
def test_pitch_and_alignment(ctx, type, ld, offset):
    """Rows that begin anywhere; what lies between them (NaN) is not read."""
    rng = np.random.default_rng(ld + offset)
    z = rng.standard_normal((9, 1001)).astype(np.float32) * 2
    u = rng.random(9).astype(np.float32)
    held, t, p = _run(ctx, z, u, type, ld=ld, offset=offset, top_k=100, top_p=0.95)
    _check(held, u, t, p, top_k=100, top_p=0.95)


@pytest.mark.parametrize("V", [1, 40, 1025, 5000, 70000])
@pytest.mark.parametrize("levels", [1, 2, 3])
def test_equal_logits_go_by_index(ctx, V, levels):
    rng = np.random.default_rng(V + levels)
    z = rng.integers(0, levels, (6, V)).astype(np.float32) - 1
    z[z == 0] = np.where(rng.random((z == 0).sum()) < 0.5, 0.0, -0.0)  # -0 and +0 are equal
    u = np.array([0, 0.25, 0.5, 0.75, 0.999, 1 - 2.0 ** -24], np.float32)
    for k in sorted({1, min(V, 7), min(V, 1024)}):
        for top_p in (1.0, 0.5):
            held, t, p = _run(ctx, z, u, "f16", top_k=k, top_p=top_p)
            _check(held, u, t, p, top_k=k, top_p=top_p)


def test_tokens_ruled_out_are_never_drawn(ctx):
    rng = np.random.default_rng(2)
    z = rng.standard_normal((64, 3000)).astype(np.float32)
    z[rng.random(z.shape) < 0.99] = -np.inf  # about 30 are left, fewer than k
    z[0] = -np.inf
    z[0, 2999] = -5.0
    z[1] = np.float32(-3.4e38)  # the type's lowest, beside one that is a little more
    z[1, 7] = np.float32(-3.3e38)
    u = np.minimum(rng.random(64).astype(np.float32), np.float32(1 - 2.0 ** -24))
    u[:2] = 1 - 2.0 ** -24
    held, t, p = _run(ctx, z, u, top_k=500, top_p=0.99)
    _check(held, u, t, p, top_k=500, top_p=0.99)
    assert np.isfinite(z[np.arange(64), t]).all() and t[0] == 2999 and t[1] == 7


@pytest.mark.parametrize("temperature", [1e-310, 1e-300, 1e-3, 1e3, 1e300])
def test_extreme_temperatures(ctx, temperature):
    rng = np.random.default_rng(4)
    z = rng.standard_normal((8, 777)).astype(np.float32) * 50
    u = rng.random(8).astype(np.float32)
    held, t, p = _run(ctx, z, u, temperature=temperature, top_k=300, top_p=0.8, min_p=0.01)
    _check(held, u, t, p, temperature, 300, 0.8, 0.01)


def test_ascending_descending_and_peaked_rows(ctx):
    n = 40000
    z = np.stack([np.arange(n), np.arange(n)[::-1], np.where(np.arange(n) == 31999, 80, 0),
                  np.where(np.arange(n) % 1000 == 3, 5, -5)]).astype(np.float32) / 16
    u = np.array([0.3, 0.9, 0.5, 0.77], np.float32)
    for k in (1, 64, 1024):
        held, t, p = _run(ctx, z, u, top_k=k)
        _check(held, u, t, p, top_k=k)


@pytest.mark.parametrize("k", [300, 1000, 1024])
def test_long_rows_of_uneven_values(ctx, k):
    """The slices' lists in one: values far apart, the whole range of the type, most of them alike."""
    rng = np.random.default_rng(k)
    z = rng.standard_normal((6, 90000)).astype(np.float32)
    z[0, ::7] = 1e30
    z[1] = np.where(rng.random(90000) < 0.5, 3.4e38, -3.4e38)
    z[2, rng.integers(0, 90000, 900)] = 5.0
    z[2, 4567] = 3.3e38
    z[3] = np.where(rng.random(90000) < 0.02, z[3], -np.inf)
    z[4] = np.float32(1) + z[4] * 2.0 ** -22
    z[5, 100:] *= 1e-40
    u = np.array([0.4, 0.1, 0.999, 0.6, 0.8, 0.3], np.float32)
    for top_p in (1.0, 0.7):
        held, t, p = _run(ctx, z, u, top_k=k, top_p=top_p)
        _check(held, u, t, p, top_k=k, top_p=top_p)


def test_greedy_is_top_k_1(ctx):
    rng = np.random.default_rng(9)
    z = rng.standard_normal((50, 5000)).astype(np.float32)
    _, t, p = _run(ctx, z, rng.random(50).astype(np.float32), top_k=1)
    assert np.array_equal(t, z.argmax(1)) and (p == 1).all()


@pytest.mark.parametrize("bad,status", [(np.nan, aiq.ERR_DEVICE_CHECK), (np.inf, aiq.ERR_DEVICE_CHECK)])
@pytest.mark.parametrize("at", [0, 500, 40000])
def test_rows_without_a_draw_are_reported(ctx, bad, status, at):
    rng = np.random.default_rng(1)
    z = rng.standard_normal((3, 40001)).astype(np.float32)
    z[1, at] = bad
    with pytest.raises(aiq.AiqError) as e:
        _run(ctx, z, [0.5] * 3, top_k=5)
    assert e.value.status == status


def test_the_other_rows_are_written(ctx):
    rng = np.random.default_rng(1)
    z = rng.standard_normal((5, 900)).astype(np.float32)
    z[1] = -np.inf
    u = np.array([0.2, 0.5, -0.1, 1.0, 0.7], np.float32)
    code = aiq.LOGITS_F32
    d, du = torch.as_tensor(z).cuda(), torch.as_tensor(u).cuda()
    tok, prob = torch.full((5,), -9, dtype=torch.int32, device="cuda"), torch.full((5,), -9.0, device="cuda")
    torch.cuda.synchronize()
    with pytest.raises(aiq.AiqError) as e:
        ctx.op_sample(d.data_ptr(), code, 900, 5, 900, du.data_ptr(), tok.data_ptr(), top_k=9, probs=prob.data_ptr())
    assert e.value.status == aiq.ERR_DEVICE_CHECK
    t, p = tok.cpu().numpy(), prob.cpu().numpy()
    assert (t[1:4] == 0).all() and (p[1:4] == 0).all()
    _check(z[[0, 4]], u[[0, 4]], t[[0, 4]], p[[0, 4]], top_k=9)
    ctx.op_sample(d.data_ptr(), code, 900, 1, 900, du.data_ptr(), tok.data_ptr(), top_k=9)  # no probabilities wanted


def test_refusals(ctx):
    buf = torch.zeros(4096, device="cuda")
    p = buf.data_ptr()
    good = dict(logits=p, type=aiq.LOGITS_F32, ldl=1100, R=1, V=1100, uniforms=p, tokens=p + 8192)
    bad = [dict(logits=0), dict(uniforms=0), dict(tokens=0), dict(type=3), dict(type=-1), dict(ldl=1099), dict(R=-1),
           dict(V=0), dict(top_k=0), dict(top_k=1101), dict(top_k=-4), dict(temperature=0.0), dict(temperature=-1.0),
           dict(temperature=float("nan")), dict(temperature=float("inf")), dict(top_p=0.0), dict(top_p=1.01),
           dict(top_p=float("nan")), dict(min_p=-0.1), dict(min_p=1.5), dict(min_p=float("nan")), dict(logits=p + 2),
           dict(tokens=p + 1), dict(uniforms=p + 2), dict(probs=p + 2)]
    for b in bad:
        with pytest.raises(aiq.AiqError) as e:
            ctx.op_sample(**{**good, **b})
        assert e.value.status == aiq.ERR_INVALID_ARG, b
    with pytest.raises(aiq.AiqError) as e:
        ctx.op_sample(**{**good, "top_k": 1025})
    assert e.value.status == aiq.ERR_UNSUPPORTED
    ctx.op_sample(**{**good, "R": 0})
