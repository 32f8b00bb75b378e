"""Attention weights far from the usual sizes: keys of next to no scale under a small softmax scale, and scores of hundreds.

The bound is the one that the header states: a weight is off by at most 2^-19 (M + |lse|) of itself, M = |scale| sum_c (16 s_c + |c_c|)
|q_c|, and a sum of r of them by r 2^-24 more.  (Few rows: sums of at most 16 steps, each off by 2^-23 of the largest magnitude
in it, at most M; the exponent's argument takes three roundings of 2^-24 at up to 1.5 (M + |lse|).  Many rows, bf16: -lse goes along
in the product, as sixteen terms of at most |lse|, under the same 16 steps.  The exponential: 2^-22, which 2^-19 M + 2^-19 |lse| hold only
where that is an eighth and more; it is added.)
"""
import numpy as np
import pytest
import torch

import oracle.kv4 as ora
from gpu_helpers import ensure_built
from test_gpu_kv4_attend import BF16, FP16, Case, queries
from test_gpu_kv4_evict import check_weights, lse_of
from test_gpu_kv4_tree import starts

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


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("hd,group,tokens,std", [(128, 8, [1, 3], 50.0), (128, 8, [40, 9], 50.0), (64, 5, [2, 4], 60.0), (64, 5, [70, 64], 60.0),
                                                 (128, 4, [100, 300], 20.0), (128, 8, [8, 5], 30.0)])
def test_scores_of_hundreds(hd, group, tokens, std, dtype):
    """lse of 50 to 250, within the stated bound of 64 bits."""
    c = Case([400, 333], 2, hd, 64, seed=4)
    q = queries(sum(tokens), 2 * group, hd, dtype, std=std)
    kv4, users = c.kv4, [0, 1]
    lse = lse_of(c, q, tokens, users, 0, 0, hd ** -0.5)
    assert 50 < lse.max() < 400
    dev = {n: torch.from_numpy(getattr(c, n)).cuda() for n in ("pool", "table", "lengths", "refs")}
    pool, m = kv4.pool(dev["pool"], 64, 1, 2, hd), kv4.page_map(dev["table"], dev["lengths"], dev["refs"])
    mass = torch.zeros(1, 2, 2, c.table.shape[1] * 64, device="cuda")
    kv4.kfl_kv4_weights(pool, m, 0, q.cuda(), torch.from_numpy(lse).cuda(), mass,
                        kv4.attend_workspace(pool, 2 * group, 2, sum(tokens), max(tokens)), q_start=starts(tokens), max_q=max(tokens))
    got, x, at = mass.double().cpu().numpy(), q.double().numpy(), 0
    for u, t in enumerate(tokens):
        n = int(c.lengths[u])
        keys = ora.causal_keys(t, n)
        for h in range(2):
            k, _ = ora.rows(c.pool, c.table[u], 0, h, n, 64, hd)
            reach = np.array([np.repeat(16 * p[:, 0] + np.abs(p[:, 1]), 64) for p in
                              (c.params(u, slot, 0, h, 0).astype(np.float64) for slot in range(n))])
            want, slack = np.zeros(n), np.zeros(n)
            for j in range(h * group, (h + 1) * group):
                qj, l = x[at:at + t, j], lse[at:at + t, j].astype(np.float64)
                w = ora.weights(qj, k, l, keys, hd ** -0.5)
                off = 2.0 ** -19 * (hd ** -0.5 * (np.abs(qj) @ reach.T) + np.abs(l)[:, None]) + 2.0 ** -22
                want, slack = want + w.sum(0), slack + (w * off).sum(0)
            slack += t * group * 2.0 ** -24 * want
            # (weights below fp32's smallest normal number may be 0)
            assert (np.abs(got[0, u, h, :n] - want) <= slack + t * group * 2.0 ** -126).all()
            assert (got[0, u, h, n:] == 0).all()
        at += t
