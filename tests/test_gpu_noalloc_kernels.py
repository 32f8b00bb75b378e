"""The allocation-free head's first call loads the kernels of every batch: what the driver allocates for their code, it allocates
then.  In a process of its own, where none of them is loaded; tests/test_zz_no_alloc.py meets the same with the code memory
nearly full."""
import os
import subprocess
import sys

import pytest

from gpu_helpers import ensure_built

pytestmark = pytest.mark.gpu

CODE = """
import torch
from paper_2609_34045_gb300 import stage as K
d, vocab = 4096, 300
h, g = torch.randn(4, d, device="cuda"), torch.ones(d, device="cuda").bfloat16()
w, ids = torch.randn(vocab, d, device="cuda").bfloat16(), torch.zeros(4, dtype=torch.int32, device="cuda")
free = []
for batch in (1, 2, 3, 4, 3, 1):
    K.kfl_head_argmax_noalloc(h, g.view(torch.int16), w.view(torch.int16), batch, d, vocab, 1e-6, ids, None)
    torch.cuda.synchronize()
    free.append(torch.cuda.mem_get_info()[0])
assert len(set(free)) == 1, free
"""


def test_no_batch_allocates_after_the_first_call():
    ensure_built()
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", CODE], cwd=root, capture_output=True, text=True, timeout=180)
    assert r.returncode == 0, r.stderr[-2000:]
