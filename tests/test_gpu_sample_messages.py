"""What a call that draws tokens reports names what is wrong with its inputs."""
import numpy as np
import pytest

from helpers import gpu_ctx
from paper_2608_10139_gb300 import aiq
from test_gpu_transform_options import _inputs, _run, _zero_model

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = gpu_ctx()
    yield c
    c.close()


def _message(ctx, z, u, V):
    d, du = torch.as_tensor(z).cuda(), torch.as_tensor(np.asarray(u, np.float32)).cuda()
    tok = torch.zeros(len(z), dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    with pytest.raises(aiq.AiqError) as e:
        ctx.op_sample(d.data_ptr(), aiq.LOGITS_F32, V, len(z), V, du.data_ptr(), tok.data_ptr(), top_k=9)
    assert e.value.status == aiq.ERR_DEVICE_CHECK
    return str(e.value)


@pytest.mark.parametrize("V", [900, 70000])
def test_messages(ctx, V):
    z = np.random.default_rng(1).standard_normal((3, V)).astype(np.float32)
    for u in (1.0, -0.1, np.nan, np.inf):
        assert "uniform" in _message(ctx, z, [0.5, u, 0.5], V)
    for bad in (np.nan, np.inf):
        x = z.copy()
        x[2, V - 7] = bad
        assert "logit" in _message(ctx, x, [0.5] * 3, V) and "uniform" not in _message(ctx, x, [0.5] * 3, V)
    z[0] = -np.inf
    assert "logit" in _message(ctx, z, [0.5] * 3, V)


def test_message_of_a_query(ctx):
    shape, W, _ = _zero_model()
    table, prefix = _inputs(shape, 4, 3)
    u = np.full((4, 2), 0.5, np.float32)
    u[3, 1] = 1.0
    with pytest.raises(aiq.AiqError) as e:
        _run(ctx, shape, W, table, prefix, [], 2, sampling=dict(top_k=5), uniforms=u)
    assert e.value.status == aiq.ERR_DEVICE_CHECK and "uniform" in str(e.value)
