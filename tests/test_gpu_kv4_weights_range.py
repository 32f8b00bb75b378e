"""Attention weights of keys of next to no scale under a small softmax scale, within the tolerances of test_gpu_kv4_evict."""
import numpy as np
import pytest
import torch

from gpu_helpers import ensure_built
from test_gpu_kv4_attend import BF16, FP16, Case, queries
from test_gpu_kv4_evict import check_weights

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()
    torch.cuda.init()


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("hd,group,tokens", [(128, 5, 30), (128, 7, 40), (64, 3, 50), (64, 12, 33), (128, 7, 3), (128, 4, 70)])
@pytest.mark.parametrize("scale", [1e-3, 2.5e-5, 1e-5, 1e-7, 1e-13, 1e-20, 1e-22])
def test_keys_of_next_to_no_scale_under_a_small_one(hd, group, tokens, dtype, scale):
    """1 / (scale log2(e) key scale) is 2^31 to 2^95: with rows that are no tokens (groups that do not divide a unit's rows) each key's weight
    is still the sum over the others."""
    c = Case([300], 1, hd, 32, seed=3)
    for slot in range(300):
        p = c.params(0, slot, 0, 0, 0)
        p[:] = [(1 + slot % 4) * 2.0 ** -24, 0.5]
        if slot % 3 == 0:
            p[-1] = [0.25, -0.5]
    got, before = check_weights(c, queries(tokens, group, hd, dtype), tokens=[tokens], scale=scale)
    assert np.isfinite(got).all() and (got[0, 0, 0, :300] > before[0, 0, 0, :300]).all()
