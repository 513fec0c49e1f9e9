"""Arguments that the calls on the 4-bit cache and of beam search refuse.  They are refused
before the context is used, so a stand-in for one does, without a GPU."""
import ctypes as C

import pytest

from paper_2608_10139_gb300 import aiq

INVALID, UNSUPPORTED = aiq.ERR_INVALID_ARG, aiq.ERR_UNSUPPORTED
A = 1 << 20  # an address that is never used, 16-byte aligned


@pytest.fixture(scope="module")
def ctx():
    from paper_2608_10139_gb300 import build
    build.build()
    c = aiq.Context.__new__(aiq.Context)
    c.lib = aiq.load_library()
    c._stand_in = C.create_string_buffer(1 << 16)
    c.h = C.cast(c._stand_in, C.c_void_p)
    yield c
    c.h = None


def _refused(status, call, **kw):
    with pytest.raises(aiq.AiqError) as e:
        call(**kw)
    assert e.value.status == status, str(e.value)


ROWS = dict(ldkv=256, T=100, seq_start=A, n_seqs=3, Hkv=1, hd=64)


@pytest.mark.parametrize("change,status", [
    (dict(kv=0), INVALID), (dict(cache=0), INVALID), (dict(seq_start=0), INVALID), (dict(T=-1), INVALID),
    (dict(T=1 << 31), INVALID), (dict(n_seqs=-1), INVALID), (dict(Hkv=0), INVALID), (dict(hd=96), UNSUPPORTED),
    (dict(ldkv=120), INVALID), (dict(ldkv=132), INVALID), (dict(kv=A + 2), INVALID), (dict(cache=A + 8), INVALID),
    (dict(seq_start=A + 2), INVALID), (dict(Hkv=(1 << 20) + 1, ldkv=1 << 30), UNSUPPORTED)])
def test_quantize_and_dequantize(ctx, change, status):
    for call in (ctx.op_kv_quantize4, ctx.op_kv_dequantize4):
        _refused(status, call, **{**ROWS, "kv": A, "cache": A, **change})


STEP = dict(qkv=A, R=12, Hq=8, Hkv=2, hd=64, own_cache=A, T=50, seq_start=A, gen_cache=A, gen_cap=40, slot=3, out=A, beams=4,
            prefix=A, P=5, held=A)


@pytest.mark.parametrize("change,status", [
    (dict(qkv=0), INVALID), (dict(out=0), INVALID), (dict(gen_cache=0), INVALID), (dict(seq_start=0), INVALID),
    (dict(own_cache=0), INVALID), (dict(prefix=0), INVALID), (dict(R=-4), INVALID), (dict(Hq=7), INVALID), (dict(Hkv=0), INVALID),
    (dict(P=-1), INVALID), (dict(T=-1), INVALID), (dict(T=1 << 31), INVALID), (dict(gen_cap=0), INVALID), (dict(slot=-1), INVALID),
    (dict(slot=40), INVALID), (dict(beams=0), INVALID), (dict(beams=5), INVALID), (dict(beams=-4), INVALID), (dict(hd=16), UNSUPPORTED),
    (dict(Hq=18), UNSUPPORTED), (dict(qkv=A + 8), INVALID), (dict(own_cache=A + 4), INVALID), (dict(prefix=A + 8), INVALID),
    (dict(gen_cache=A + 8), INVALID), (dict(out=A + 8), INVALID), (dict(held=A + 8), INVALID), (dict(seq_start=A + 1), INVALID),
    (dict(Hq=1 << 21, Hkv=1 << 20), UNSUPPORTED), (dict(R=1 << 30, Hq=8), UNSUPPORTED)])
def test_attention(ctx, change, status):
    _refused(status, ctx.op_decode_attention_q4, **{**STEP, **change})


PICK = dict(logits=A, type=aiq.LOGITS_F32, ldl=100, n=3, beams=4, V=100, scores=A, keep=8, parents=A, tokens=A, scores_out=A, done=A,
            done_out=A)


@pytest.mark.parametrize("change,status", [
    (dict(logits=0), INVALID), (dict(scores=0), INVALID), (dict(parents=0), INVALID), (dict(tokens=0), INVALID),
    (dict(scores_out=0), INVALID), (dict(n=-1), INVALID), (dict(V=0), INVALID), (dict(ldl=99), INVALID), (dict(type=3), INVALID),
    (dict(type=-1), INVALID), (dict(beams=0), INVALID), (dict(keep=0), INVALID), (dict(beams=17), UNSUPPORTED),
    (dict(keep=33), UNSUPPORTED), (dict(V=(1 << 30) + 1, ldl=1 << 31), UNSUPPORTED), (dict(n=1 << 23), UNSUPPORTED),
    (dict(logits=A + 2), INVALID), (dict(scores=A + 2), INVALID), (dict(done=A + 1), INVALID), (dict(parents=A + 2), INVALID),
    (dict(done_out=A + 2), INVALID)])
def test_selection(ctx, change, status):
    _refused(status, ctx.op_beam_select, **{**PICK, **change})


MOVE = dict(src=A, dst=1 << 30, bytes=64, pitch=128, n=3, beams=4, parents=A, layers=2, layer_pitch=1536)


@pytest.mark.parametrize("change,status", [
    (dict(src=0), INVALID), (dict(dst=0), INVALID), (dict(parents=0), INVALID), (dict(bytes=-1), INVALID), (dict(n=-1), INVALID),
    (dict(layers=-1), INVALID), (dict(beams=0), INVALID), (dict(beams=17), UNSUPPORTED), (dict(pitch=60), INVALID),
    (dict(pitch=-128), INVALID), (dict(layer_pitch=60), INVALID), (dict(layer_pitch=1400), INVALID), (dict(dst=A + 16), INVALID),
    (dict(dst=A + 1536), INVALID), (dict(dst=A - 64), INVALID), (dict(parents=A + 2), INVALID), (dict(pitch=1 << 60), INVALID),
    (dict(layer_pitch=1 << 60), INVALID), (dict(bytes=1 << 50, pitch=1 << 50), INVALID)])
def test_reorder(ctx, change, status):
    _refused(status, ctx.op_beam_reorder, **{**MOVE, **change})


def test_outputs_that_overlap_inputs(ctx):
    apart = {k: (i + 1) << 30 for i, k in enumerate(("logits", "scores", "done", "parents", "tokens", "scores_out", "done_out"))}
    for out in ("parents", "tokens", "scores_out", "done_out"):
        for at in (apart["logits"] + 12 * 400 - 4, apart["scores"], apart["scores"] - 4 * 3 * 8 + 4, apart["done"] + 44):
            _refused(INVALID, ctx.op_beam_select, **{**PICK, **apart, out: at})
    for at in (1 << 30, (1 << 30) + 1536 + 11 * 128 + 60, (1 << 30) - 44):
        _refused(INVALID, ctx.op_beam_reorder, **{**MOVE, "parents": at})
