"""Prompts of so many tiles that their list's places pass 32 bits: reported and not computed (they would run for half a minute)."""
import pytest
import torch

from gpu_helpers import ensure_built

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()
    torch.cuda.init()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,group,sequences", [(1 << 22, 16, 1), (1 << 25, 4, 1), (1 << 22, 2, 40)])
def test_more_tiles_than_32_bits(n, group, sequences, dtype):
    """Every page of the table is the same one, and every query row and output row too (their strides are 0): nothing of it is
    read or written, and were it, it would be there."""
    from paper_2609_34045_gb300 import kv4
    page, hd = 128, 64
    pool_t = torch.zeros(1, page * hd * 9 // 8, dtype=torch.uint8, device="cuda")
    p = kv4.pool(pool_t, page, 1, 1, hd)
    m = kv4.page_map(torch.zeros(1, n // page, dtype=torch.int32, device="cuda"),
                     torch.full((1,), n, dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda"))
    tokens = n // 4 if sequences > 1 else n
    q = torch.ones(1, group, hd, dtype=dtype, device="cuda").expand(tokens * sequences, group, hd)
    out_t = torch.full((1, group, hd), 7.0, dtype=dtype, device="cuda")
    start = torch.arange(0, tokens * sequences + 1, tokens, dtype=torch.int32, device="cuda")
    users = torch.zeros(sequences, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = kv4.attend_workspace(p, group, sequences, tokens * sequences, tokens)
    kv4.kfl_kv4_attend(p, m, 0, q, out_t.expand(tokens * sequences, group, hd), ws, users=users, q_start=start, max_q=tokens, status=status)
    torch.cuda.synchronize()
    assert status.item() == kv4.KFL_BAD_POSITION
    assert (out_t == 7).all()
    # a call that follows on the same workspace is as it always is
    few = torch.arange(0, 101, 100, dtype=torch.int32, device="cuda")
    status.zero_()
    q = torch.randn(100, group, hd, device="cuda").to(dtype)
    outs = [torch.empty_like(q) for _ in range(2)]
    for o, w in zip(outs, (ws, torch.zeros_like(ws))):
        kv4.kfl_kv4_attend(p, m, 0, q, o, w, users=users[:1], q_start=few, max_q=100, window=500, status=status)
    assert status.item() == 0 and torch.equal(*outs) and torch.isfinite(outs[0].float()).all()
