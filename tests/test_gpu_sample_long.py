"""A token of very long rows: one row's slices on every SM, and their merge."""
import numpy as np
import pytest

from helpers import gpu_ctx
from test_gpu_sample import _check, _run

pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = gpu_ctx()
    yield c
    c.close()


# 4,980,736 = 1,216 slices of 4,096; a slice's share of 1,024 candidates is then less than one
@pytest.mark.parametrize("V", [4_980_736, 4_980_735, 4_980_737, 9_944_355])
@pytest.mark.parametrize("k", [1, 96, 97, 1024])
def test_one_row_on_every_sm(ctx, V, k):
    rng = np.random.default_rng(V + k)
    z = rng.standard_normal((1, V), dtype=np.float32)
    u = np.array([0.6], np.float32)
    held, t, p = _run(ctx, z, u, "f16", top_k=k, top_p=0.95)
    _check(held, u, t, p, top_k=k, top_p=0.95)


@pytest.mark.parametrize("where", ["begin", "end", "one slice", "alike"])
def test_candidates_in_few_slices(ctx, where):
    """The largest in one place: the slices list too few of them, and the row is listed again."""
    V, k = 4_980_736, 1024
    rng = np.random.default_rng(5)
    z = rng.standard_normal((2, V), dtype=np.float32)
    at = {"begin": 0, "end": V - 3000, "one slice": 4096 * 700, "alike": 0}[where]
    if where == "alike":
        z[:] = 1.5
    else:
        z[:, at:at + 3000] += 20
    u = np.array([0.2, 0.9], np.float32)
    held, t, p = _run(ctx, z, u, top_k=k, top_p=0.9)
    _check(held, u, t, p, top_k=k, top_p=0.9)
