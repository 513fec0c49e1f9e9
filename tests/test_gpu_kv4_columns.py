"""The 4-bit attention's numbers hang on a query head's own scores alone: those of the heads and beams
that share its tiles may be of any magnitude (aiq_op_decode_attention_q4)."""
import numpy as np
import pytest

from helpers import gpu_ctx
from test_gpu_kv_cache4 import Batch

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = gpu_ctx()
    yield c
    c.close()


def _near(rng, shape, at):
    """Elements near one number, so that scores are large and close to one another."""
    return (at + 0.5 * rng.standard_normal(shape)).astype(np.float16)


# A CTA a task, tasks drawn, ranges; columns that two lanes share (up to four) and that one has.
@pytest.mark.parametrize("hd,Hq,Hkv,beams,rows,length", [(64, 4, 2, 1, 20, 150), (64, 8, 2, 2, 20, 150), (128, 4, 2, 1, 20, 150),
                                                         (32, 16, 2, 1, 20, 150), (64, 8, 4, 1, 1200, 20), (64, 16, 8, 1, 400, 500),
                                                         (128, 16, 2, 1, 900, 40)])
@pytest.mark.parametrize("who", ["head", "beam"])
def test_what_shares_a_tile_does_not_matter(ctx, hd, Hq, Hkv, beams, rows, length, who):
    """Other heads of a KV head, or the other beam, with scores of ordinary size and of 2^22 and more: the
    first one's output is the same, to the bit."""
    if who == "beam" and beams == 1:
        beams, rows = 2, max(1, rows // 2)
    rng = np.random.default_rng(hd + rows + Hq)
    lens = [int(x) for x in rng.integers(length // 2, length * 3 // 2, rows)]
    b = Batch(ctx, rng, hd, Hq, Hkv, beams, lens, 0, 40, std=0.0)
    # keys near 300 (whole tiles are quantised by the library)
    w = 2 * Hkv * hd
    kv = np.concatenate([_near(rng, (sum(lens), w // 2), 300), _near(rng, (sum(lens), w // 2), 0)], 1)
    d = torch.as_tensor(kv).cuda()
    torch.cuda.synchronize()
    ctx.op_kv_quantize4(d.data_ptr(), w, sum(lens), b.st.data_ptr(), rows, Hkv, hd, b.d_own.data_ptr())
    G, R = Hq // Hkv, rows * beams
    q = _near(rng, (R, Hkv, G, hd), 1)
    step = np.concatenate([_near(rng, (R, w // 2), 300), _near(rng, (R, w // 2), 0)], 1)
    mine = np.zeros((rows, beams, Hkv, G), bool)
    if who == "head":
        mine[:, :, :, 0] = True
    else:
        mine[:, 0] = True
    mine = mine.reshape(R, Hkv, G)
    out = []
    for factor in (1, 3000):
        x = np.where(mine[..., None], q, q * np.float16(factor)).reshape(R, -1)
        got, _ = b.step(np.concatenate([x, step], 1), 0)
        out.append(got.reshape(R, Hkv, G, hd)[mine].view(np.uint16).copy())
    # 300 hd / sqrt(hd) log2(e): 2,400 to 4,900, 2^22 after 1,700 to 900 times that
    differ = (out[0] != out[1]).sum()
    assert differ == 0, f"{differ} of {out[0].size}"
