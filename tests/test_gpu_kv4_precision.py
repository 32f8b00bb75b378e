"""How far fp16 outputs of the 4-bit cache's attention are from 64 bits, in the mean over many.

Two roundings to fp16 are left where codes and values are taken exactly, the softmax weights' and the output's.  Rounding a number to 11
bits is off by a uniform error of at most 2^-11 of its power of two: 2^-11 / sqrt 3 of that, and with mantissas evenly
spread over their logarithm (mean of 1 / m^2: 0.541) 2^-11 sqrt(0.541 / 3) = 2.07e-4 of the number, root mean square.  The weights'
errors are independent over the keys, as zero-mean values are, and so come out as large relative to the output.  Together
sqrt 2 times 2.07e-4; a tenth is added for mantissas that are not spread so.  (With K or V rounded to fp16 as well it is 3.5e-4,
with both 4.3e-4 to 5e-4.)
"""
import numpy as np
import pytest
import torch

import oracle.kv4 as ora
from gpu_helpers import ensure_built
from test_gpu_kv4_attend import FP16, Case, queries

pytestmark = pytest.mark.gpu
BOUND = 1.1 * 2 ** 0.5 * 2.0 ** -11 * (0.541 / 3) ** 0.5


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()
    torch.cuda.init()


def fill(c, make):
    """Every row of every user anew: values make(rows, hd, which) quantised."""
    n = c.page * c.hd // 2
    m = c.page * c.hd // 16
    for u, count in enumerate(c.lengths):
        for j in range(-(-int(count) // c.page)):
            rows = min(c.page, int(count) - j * c.page)
            b = c.pool[c.table[u, j], 0]
            for which in (0, 1):
                for head in range(b.shape[0]):
                    codes, par = ora.quantise(make(rows, c.hd, which).astype(np.float32))
                    b[head, which * n:which * n + rows * c.hd // 2] = (codes[:, 0::2] | codes[:, 1::2] << 4).reshape(-1)
                    b[head, 2 * n + which * m:2 * n + which * m + rows * c.hd // 16] = par.reshape(-1).view(np.uint8)


def error(got, ref):
    return np.linalg.norm(got.double().cpu().numpy() - ref) / np.linalg.norm(ref)


@pytest.mark.parametrize("hd,page", [(128, 64), (64, 16)])
@pytest.mark.parametrize("tokens,lengths", [([150, 40], [1500, 900]), ([1, 1], [1500, 900])])
def test_fp16_outputs(hd, page, tokens, lengths):
    """Keys with the few large channels that models have; prompts and single tokens."""
    c = Case(lengths, 4, hd, page, seed=hd)
    rng = np.random.default_rng(hd)
    large = 4.0 * (rng.random(hd) < 0.05)
    fill(c, lambda n, d, which: rng.standard_normal((n, d)) + (large if which == 0 else 0.0))
    q = queries(sum(tokens), 32, hd, FP16)
    got, _ = c.run(q, tokens=tokens)
    ref, _, _ = c.expected(q, tokens=tokens)
    assert error(got, ref) <= BOUND


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("key_offset,key_std", [(50.0, 0.05), (50.0, 0.2), (3.0, 0.2), (0.0, 1e-3)])
def test_keys_far_from_zero_and_small(hd, key_offset, key_std):
    """Groups of keys whose step is far below their rounding to fp16, where scores hang on the second term: 50 and 0.05 are some 3000
    steps from zero, 0.2 some 800.  Queries without a mean in each group, so that the offset drops out of the softmax.  The products'
    fp32 sum loses at most 2^-22 of its largest partial sum in each of its 2 hd / 16 steps."""
    c = Case([700], 2, hd, 64, seed=3)
    rng = np.random.default_rng(int(key_offset) + hd)
    fill(c, lambda n, d, which: rng.standard_normal((n, d)) * (key_std if which == 0 else 1.0) + (key_offset if which == 0 else 0.0))
    scale = hd ** -0.5 / key_std
    x = queries(100, 8, hd, FP16).float().view(100, 8, hd // 64, 64)
    q = (x - x.mean(-1, keepdim=True)).view(100, 8, hd).to(FP16)
    got, lse = c.run(q, tokens=[100], scale=scale)
    ref, _, ref_lse = c.expected(q, tokens=[100], scale=scale)
    partial = q.double().view(100, 8, hd // 64, 64).cumsum(-1).abs().max().item() * key_offset * scale + 10.0
    drift = 2 * hd / 16 * 2.0 ** -22 * partial
    assert error(got, ref) <= BOUND + 2 * drift
    assert np.abs(lse.double().cpu().numpy() - ref_lse).max() <= 2.0 ** -10 + drift + 2.0 ** -22 * np.abs(ref_lse).max()
