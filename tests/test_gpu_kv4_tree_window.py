"""Sliding windows over trees of drafted tokens: a node sees the last `window` rows of the context and its own path together, itself
among them, as the same tokens do that are checked one path at a time.  Views to the bit; attention with the
tolerances of test_gpu_kv4_tree.
"""
import numpy as np
import pytest
import torch

import oracle.kv4 as ora
from gpu_helpers import ensure_built
from test_gpu_kv4_attend import BF16, FP16, Case, assert_near, queries
from test_gpu_kv4_tree import attend_tree, i32, random_tree, starts

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()
    torch.cuda.init()


def windowed(parents, window):
    """Which nodes each node sees: itself and the window - 1 before it on its path."""
    seen = np.zeros((len(parents), len(parents)), dtype=bool)
    for i in range(len(parents)):
        at, left = i, window or len(parents)
        while at >= 0 and left > 0:
            seen[i, at] = True
            at, left = parents[at], left - 1
    return seen


@pytest.mark.parametrize("counts", [[1], [4, 1, 0, 7], [33, 32, 31], [1024], [5, 1000, 64]])
@pytest.mark.parametrize("spread", [1, 3])
@pytest.mark.parametrize("window", [0, 1, 2, 7, 32, 33, 500, 2 ** 31 - 1])
def test_views_of_windows(counts, spread, window):
    from paper_2609_34045_gb300 import kv4
    rng = np.random.default_rng(len(counts) + spread)
    parents = [random_tree(rng, n, spread) for n in counts]
    n, max_q = sum(counts), max(counts)
    views = torch.full((n, -(-max_q // 32)), 77, dtype=torch.int32, device="cuda")
    positions, status = torch.full((n,), 7, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    kv4.kfl_kv4_tree(i32(sum(parents, [])), views, positions, q_start=starts(counts), max_q=max_q, window=window, status=status)
    want = [ora.tree_words(windowed(p, window), max_q) for p in parents]
    assert np.array_equal(views.cpu().numpy(), np.concatenate(want).view(np.int32))
    assert np.array_equal(positions.cpu().numpy(), np.concatenate([ora.tree_seen(p)[1] for p in parents]))  # (ancestors, seen or not)
    assert status.item() == 0


@pytest.mark.parametrize("hd,group,tokens,dtype", [(128, 8, [4, 3], BF16), (64, 4, [9, 16], FP16), (128, 8, [40, 7], BF16), (128, 3, [90, 130], FP16)])
@pytest.mark.parametrize("window", [1, 2, 5, 33, 64, 150])
def test_a_chain_with_a_window_is_causal_with_it(hd, group, tokens, dtype, window):
    """Paths longer than the window among them."""
    c = Case([400, 222], 2, hd, 32, seed=5)
    q = queries(sum(tokens), 2 * group, hd, dtype)
    seen = [windowed(list(range(-1, t - 1)), window) for t in tokens]
    for t, s, n in zip(tokens, seen, (400, 222)):
        assert np.array_equal(ora.tree_keys(s, n, window), ora.causal_keys(t, n, window))
    got, lse, ref, size, ref_lse = attend_tree(c, q, seen, window=window)
    assert_near(got, lse, ref, size, ref_lse)
    causal, causal_lse = c.run(q, tokens=tokens, window=window)
    assert_near(causal, causal_lse, ref, size, ref_lse)


def rows(s, head, n, kv_heads, hd):
    """User 0's keys, values and the values' centres of one head of a one-layer session."""
    page = s.page_tokens
    pool, row = s.pages.cpu().numpy().reshape(-1, 1, kv_heads, page * hd * 9 // 8), s.table[0].cpu().numpy()
    k, v = ora.rows(pool, row, 0, head, n, page, hd)
    centre = [np.repeat(ora.unpack(pool[row[t // page], 0, head], page, hd)[3][t % page, :, 1].astype(np.float64), 64) for t in range(n)]
    return k, v, np.array(centre)


@pytest.mark.parametrize("window,nodes,masses", [(3, 6, False), (3, 40, False), (6, 40, False), (6, 6, False), (45, 40, False), (6, 6, True),
                                                 (45, 40, True), (0, 40, True)])
def test_a_sessions_chain_of_drafts_sees_what_its_tokens_see(window, nodes, masses):
    """The same tokens through the session as a tree's one path and as tokens one behind the other."""
    from paper_2609_34045_gb300.kv4_session import Session
    heads, kv_heads, hd, context = 8, 2, 64, 50
    outs = []
    for parents in (None, {0: list(range(-1, nodes - 1))}):
        g = torch.Generator(device="cuda").manual_seed(3)
        s = Session(1, heads, kv_heads, hd, n_users=2, max_ctx=128, n_pages=16, page_tokens=16, masses=masses)

        def qkv(n):
            return [torch.randn(n, h, hd, generator=g, device="cuda").to(BF16) for h in (heads, kv_heads, kv_heads)]  # noqa: B023
        s.attend(0, s.begin({0: context}), *qkv(context))
        outs.append(s.attend(0, s.begin({0: nodes}, parents), *qkv(nodes), window=window).double())
        assert s.status.item() == 0
        most = max(abs(rows(s, h, context + nodes, kv_heads, hd)[1]).max() for h in range(kv_heads))
    # each is off the 64-bit value by its rounding and 2^-8 of the weighted mean of |v| + |v - c|, no more than 2.1 times the largest |v|
    # (c is within 8 of 15 steps of both ends)
    assert (outs[0] - outs[1]).abs().max() <= 2 * (2.0 ** -9 * outs[0].abs().max() + 2.0 ** -8 * 2.1 * most)


@pytest.mark.parametrize("window", [2, 4, 60])
def test_a_sessions_tree_is_its_paths(window):
    """Each node's output against the oracle over the rows that its path's window holds."""
    from paper_2609_34045_gb300 import kv4
    from paper_2609_34045_gb300.kv4_session import Session
    heads, kv_heads, hd, context, page = 8, 2, 64, 50, 16
    parents = [-1, 0, 0, 1, 3, 4, 2, 5, -1, 8]
    g = torch.Generator(device="cuda").manual_seed(4)
    s = Session(1, heads, kv_heads, hd, n_users=1, max_ctx=128, n_pages=8, page_tokens=page)
    given = []
    real = kv4.kfl_kv4_attend_tree

    def record(p, m, layer, q, *args, **kw):
        given.append(q.double().cpu().numpy())
        real(p, m, layer, q, *args, **kw)

    def qkv(n):
        return [torch.randn(n, h, hd, generator=g, device="cuda").to(BF16) for h in (heads, kv_heads, kv_heads)]
    s.attend(0, s.begin({0: context}), *qkv(context))
    kv4.kfl_kv4_attend_tree = record
    try:
        out = s.attend(0, s.begin({0: len(parents)}, {0: parents}), *qkv(len(parents)), window=window)
    finally:
        kv4.kfl_kv4_attend_tree = real
    n = context + len(parents)
    seen = windowed(parents, window)
    keys = ora.tree_keys(seen, n, window)
    assert (keys.sum(1) == window).all() or window == 60
    ref, size = np.zeros(given[0].shape), np.zeros(given[0].shape)
    for j in range(heads):
        k, v, centre = rows(s, j // (heads // kv_heads), n, kv_heads, hd)
        ref[:, j], size[:, j], _ = ora.attend_keys(given[0][:, j], k, v, keys, hd ** -0.5)
        size[:, j] += ora.attend_keys(given[0][:, j], k, v - centre, keys, hd ** -0.5)[1]
    assert_near(out, None, ref, size, None)
