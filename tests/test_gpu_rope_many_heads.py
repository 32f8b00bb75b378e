"""Rotation of a token with as many heads as there may be: more than a grid has rows of blocks."""
import numpy as np
import pytest
import torch

import oracle.kv4 as ora
from gpu_helpers import ensure_built
from test_gpu_kv4_rows import BF16, FP32, THETA, freqs, int32, near, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()
    torch.cuda.init()


@pytest.mark.parametrize("heads,kv,hd,r,off,dtype", [(65536, 1, 128, 128, 1, BF16), (65536, 65536, 72, 68, 0, FP32),
                                                     (65536, 65535, 64, 64, 0, BF16)])
def test_most_heads(heads, kv, hd, r, off, dtype):
    """Rows off 16 bytes and odd parts of a head: one channel pair a thread, so that a block takes one head or two at once."""
    from paper_2609_34045_gb300 import kv4
    plan = kv4.rope_plan(kv4.kfl_rope_table(50, r, THETA))
    x = randn((2, heads + kv, hd + off), dtype, 1)[..., off:]
    q, k = x[:, :heads], x[:, heads:]
    q_out, k_out = torch.zeros(2, heads, hd, dtype=dtype, device="cuda"), torch.zeros(2, kv, hd, dtype=dtype, device="cuda")
    kv4.kfl_rope(plan, q, q_out, k, k_out, int32([49, 3]))
    angles = np.array([49, 3])[:, None] * freqs(r)
    for a, b in ((q, q_out), (k, k_out)):
        a64 = a.double().cpu().numpy()
        near(b, ora.rotate(a64, angles, False), np.abs(a64).max(-1, keepdims=True) * 2)
