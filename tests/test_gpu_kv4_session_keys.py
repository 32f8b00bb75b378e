"""Keys of users whose rows are not at their positions (trees, evicted rows): turned by the position in fp32 and coded once, as every
other key is, so that a user's codes do not hang on who else is in a pass.  Everything here is to the bit.
"""
import numpy as np
import pytest
import torch

from gpu_helpers import ensure_built
from test_gpu_kv4_rows import BF16, FP16, FP32, THETA, cache, int32, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()
    torch.cuda.init()


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32], ids=["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("hd,r", [(128, 128), (128, 36), (64, 64)])
def test_a_key_is_turned_by_its_position_and_lies_at_its_slot(hd, r, layout, dtype):
    """As kfl_kv4_append at the position itself writes it."""
    n, kv, page = 90, 2, 32
    kv4, pool_t, p, m, table = cache([400, n], kv, hd, page, layers=2)
    plan = kv4.rope_plan(kv4.kfl_rope_table(400, r, THETA), layout)
    k, v = randn((n, kv, hd), dtype, 5), randn((n, kv, hd), dtype, 6)
    at = np.random.default_rng(1).permutation(400)[:n]
    a, b, a2, b2 = (torch.empty(n, kv, hd, device="cuda") for _ in range(4))
    kv4.kfl_kv4_append(p, m, 1, k, v, int32([0] * n), int32(at), rope=plan)
    kv4.kfl_kv4_read(p, m, 1, int32([0] * n), int32(at), a, b)
    odd = torch.empty(n, kv, hd + 1, dtype=dtype, device="cuda")[..., 1:]  # rows off 16 bytes
    odd.copy_(k)
    for rows in (k, odd):
        pool_t.fill_(255)
        kv4.kfl_kv4_append(p, m, 1, rows, v, int32([1] * n), int32(range(n)), rope=plan, rope_positions=int32(at))
        kv4.kfl_kv4_read(p, m, 1, int32([1] * n), int32(range(n)), a2, b2)
        assert torch.equal(a, a2) and torch.equal(b, b2)


def test_positions_and_slots_out_of_range_are_reported_and_not_written():
    kv4, pool_t, p, m, _ = cache([40], 2, 64, 16)
    plan = kv4.rope_plan(kv4.kfl_rope_table(100, 64, THETA))
    k = randn((3, 2, 64), BF16, 1)
    status, before = torch.zeros(1, dtype=torch.int32, device="cuda"), pool_t.clone()
    for slots, positions in (([5, 6, 7], [100, -1, 2 ** 31 - 1]), ([64, -1, 2 ** 31 - 1], [5, 6, 7])):
        status.zero_()
        kv4.kfl_kv4_append(p, m, 0, k, k, int32([0] * 3), int32(slots), rope=plan, rope_positions=int32(positions), status=status)
        assert status.item() == kv4.KFL_BAD_POSITION and torch.equal(pool_t, before)
    status.zero_()
    kv4.kfl_kv4_append(p, m, 0, k, k, int32([0] * 3), int32([5, 6, 39]), rope=plan, rope_positions=int32([99, -5, 0]), status=status)
    assert status.item() == kv4.KFL_BAD_POSITION and not torch.equal(pool_t, before)  # the good rows are there
    kv4.kfl_kv4_append(p, m, 0, k[:0], k[:0], int32([]), int32([]), rope=plan, rope_positions=int32([]))


def codes(s, user, n):
    """A user's rows as they lie in the pages, byte for byte, in the order of their slots."""
    out, page, hd, kv = [], s.page_tokens, s.head_dim, s.n_kv_heads
    blocks = s.pages.cpu().numpy().reshape(-1, s.n_layers, kv, page * hd * 9 // 8)
    for t in range(n):
        b = blocks[int(s.table[user, t // page])]
        for at, size in ((0, hd // 2), (page * hd // 2, hd // 2), (page * hd, hd // 16), (page * hd + page * hd // 16, hd // 16)):
            out.append(b[..., at + t % page * size:at + (t % page + 1) * size].copy())
    return np.concatenate([o.ravel() for o in out])


HEADS, KV, HD = 4, 2, 64


def a_session(**kw):
    from paper_2609_34045_gb300.kv4_session import Session
    return Session(2, HEADS, KV, HD, n_users=3, max_ctx=128, n_pages=24, page_tokens=16, masses=True, max_positions=512, **kw)


def rows_of(user, n, seed):
    g = torch.Generator().manual_seed(100 * user + seed)
    return [[torch.randn(n, h, HD, generator=g).to(BF16).cuda() for h in (HEADS, KV, KV)] for _ in range(2)]


def run(s, counts, seed, parents=None):
    step = s.begin(counts, parents)
    mine = {u: rows_of(u, n, seed) for u, n in counts.items()}
    for layer in range(2):
        s.attend(layer, step, *(torch.cat([mine[u][layer][i] for u in counts]) for i in range(3)))
    assert s.status.item() == 0
    return step


def test_a_users_codes_do_not_hang_on_the_others():
    """A user that lost nothing, in passes with one that did, and alone."""
    together, alone = a_session(), a_session()
    run(together, {0: 30, 1: 70}, 1)
    run(alone, {0: 30}, 1)
    assert together.evict(40, [1], first=2, recent=8) == {1: 30}
    for seed in (2, 3):
        run(together, {1: 2, 0: 1}, seed)
        run(alone, {0: 1}, seed)
    assert np.array_equal(codes(together, 0, 32), codes(alone, 0, 32))


def test_a_chain_of_drafts_is_coded_as_its_tokens_are():
    trees, tokens = a_session(), a_session()
    run(trees, {0: 30}, 1), run(tokens, {0: 30}, 1)
    step = run(trees, {0: 12}, 2, {})
    run(tokens, {0: 12}, 2)
    assert np.array_equal(codes(trees, 0, 42), codes(tokens, 0, 42))
    trees.accept(step, {0: list(range(12))})
    assert np.array_equal(codes(trees, 0, 42), codes(tokens, 0, 42))


def test_rows_that_were_evicted_before_do_not_change_later_ones_codes():
    """The same key at the same position, whatever its slot."""
    cut, whole = a_session(), a_session()
    run(cut, {1: 70}, 1), run(whole, {1: 70}, 1)
    cut.evict(33, [1], first=1, recent=8)
    run(cut, {1: 5}, 2), run(whole, {1: 5}, 2)
    a, b = codes(cut, 1, 38).reshape(38, -1), codes(whole, 1, 75).reshape(75, -1)
    assert np.array_equal(a[33:], b[70:])
