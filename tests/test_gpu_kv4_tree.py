"""Trees of drafted tokens over the 4-bit paged cache against the 64-bit oracle: views and positions to the bit, attention
with the tolerances of test_gpu_kv4_attend (the same kernels, the same roundings: only which keys are seen differs), but for
the size that the weights' rounding is relative to.  With few rows a value c + (u - 8) s enters as two terms: p c with an fp32
weight, and (p s) (u - 8) with p s rounded to fp16, which is off by up to 2^-11 of it.  Where c and (u - 8) s nearly cancel
and few keys are seen, that is more than 2^-11 p |v|: the size is the weighted mean of |v| + |v - c|.
"""
import numpy as np
import pytest
import torch

import oracle.kv4 as ora
from gpu_helpers import ensure_built
from test_gpu_kv4_attend import BF16, FP16, Case, assert_near, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()
    torch.cuda.init()


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device="cuda")


def starts(counts):
    return i32(np.concatenate([[0], np.cumsum(counts)]))


def random_tree(rng, n, spread=4):
    return [int(rng.integers(max(-1, i - spread), i)) if i else -1 for i in range(n)]


def views_of(seen, max_q):
    return torch.from_numpy(np.concatenate([ora.tree_words(s, max_q) for s in seen]).view(np.int32)).cuda()


def centres(c, user, layer, head, n):
    """The centres of a user's V rows [n][hd]."""
    out = np.zeros((n, c.hd))
    for slot in range(n):
        out[slot] = np.repeat(c.params(user, slot, layer, head, 1)[:, 1].astype(np.float64), 64)
    return out


def attend_tree(c, q, seen, users=None, layer=0, window=0, scale=None, max_q=None, status=None, views=None, out=None, lse=True,
                workspace=None, q_start=True):
    """The kernel's output and lse, and the oracle's."""
    tokens = [len(s) for s in seen]
    max_q = max_q or max(1, *tokens)
    kv4 = c.kv4
    dev = {n: torch.from_numpy(getattr(c, n)).cuda() for n in ("pool", "table", "lengths", "refs")}
    pool, m = kv4.pool(dev["pool"], c.page, c.layers, c.pool.shape[2], c.hd), kv4.page_map(dev["table"], dev["lengths"], dev["refs"])
    q = q.cuda() if not q.is_cuda else q
    out = torch.full_like(q, 7.0) if out is None else out
    lse = torch.full(q.shape[:2], 7.0, device="cuda") if lse else None
    ws = kv4.attend_workspace(pool, q.shape[1], len(seen), q.shape[0], max_q) if workspace is None else workspace
    kv4.kfl_kv4_attend_tree(pool, m, layer, q, out, views_of(seen, max_q) if views is None else views, ws,
                            users=None if users is None else i32(users), q_start=starts(tokens) if q_start else None, max_q=max_q,
                            window=window, scale=scale, lse=lse, status=status)
    torch.cuda.synchronize()
    group = q.shape[1] // c.pool.shape[2]
    x = q.double().cpu().numpy()
    ref, size, ref_lse = np.zeros(x.shape), np.zeros(x.shape), np.zeros(x.shape[:2])
    at = 0
    for i, s in enumerate(seen):
        u, t = (users[i] if users is not None else i), len(s)
        n = int(c.lengths[u])
        keys = ora.tree_keys(s, n, window)
        for h in range(c.pool.shape[2]):
            k, v = ora.rows(c.pool, c.table[u], layer, h, n, c.page, c.hd)
            rest = v - centres(c, u, layer, h, n)
            for j in range(h * group, (h + 1) * group):
                s = c.hd ** -0.5 if scale is None else scale
                ref[at:at + t, j], size[at:at + t, j], ref_lse[at:at + t, j] = ora.attend_keys(x[at:at + t, j], k, v, keys, s)
                size[at:at + t, j] += ora.attend_keys(x[at:at + t, j], k, rest, keys, s)[1]
        at += t
    return out, lse, ref, size, ref_lse


@pytest.mark.parametrize("counts", [[1], [4, 1, 0, 7], [33, 32, 31], [128] * 3, [1024], [5, 1000, 64] * 20])
@pytest.mark.parametrize("spread", [1, 3, 1000])
def test_views_and_positions(counts, spread):
    from paper_2609_34045_gb300 import kv4
    rng = np.random.default_rng(len(counts) + spread)
    parents = [random_tree(rng, n, spread) for n in counts]
    n, max_q = sum(counts), max(counts) + 5 if max(counts) < 1000 else 1024
    first = rng.integers(0, 10 ** 6, len(counts))
    views = torch.full((n, -(-max_q // 32)), 77, dtype=torch.int32, device="cuda")
    positions, status = torch.full((n,), 7, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    kv4.kfl_kv4_tree(i32(sum(parents, [])), views, positions, q_start=starts(counts), first=i32(first), max_q=max_q, status=status)
    seen = [ora.tree_seen(p) for p in parents]
    assert np.array_equal(views.cpu().numpy(), np.concatenate([ora.tree_words(s, max_q) for s, _ in seen]).view(np.int32))
    assert np.array_equal(positions.cpu().numpy(), np.concatenate([f + d for f, (_, d) in zip(first, seen)]))
    assert status.item() == 0
    again = torch.zeros_like(views)
    kv4.kfl_kv4_tree(i32(sum(parents, [])), again, q_start=starts(counts), max_q=max_q)  # no first, no positions
    assert torch.equal(again, views)


def test_single_nodes_without_starts():
    from paper_2609_34045_gb300 import kv4
    views, positions = torch.zeros(5, 1, dtype=torch.int32, device="cuda"), torch.zeros(5, dtype=torch.int32, device="cuda")
    kv4.kfl_kv4_tree(i32([-1] * 5), views, positions, first=i32([3, 1, 4, 1, 5]))
    assert views.flatten().tolist() == [1] * 5 and positions.tolist() == [3, 1, 4, 1, 5]


def test_bad_parents_and_starts_are_reported():
    from paper_2609_34045_gb300 import kv4
    views, positions = torch.full((9, 1), 7, dtype=torch.int32, device="cuda"), torch.full((9,), 7, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kv4.kfl_kv4_tree(i32([-1, 1, -2, 2, 9, 4, 0, 0, 0]), views, positions, q_start=i32([0, 6, 9, 20]), max_q=6, status=status)
    # nodes 1, 2 and 4 name no earlier node: roots; the second sequence's first node too; the third does not fit
    assert views.flatten().tolist() == [1, 2, 4, 12, 16, 48, 1, 3, 5]
    assert positions.tolist() == [0, 0, 0, 1, 0, 1, 0, 1, 1] and status.item() == kv4.KFL_BAD_POSITION


SHAPES = [(128, 2, 8, 64, BF16), (128, 2, 7, 16, FP16), (64, 2, 4, 32, BF16), (64, 1, 1, 128, FP16), (128, 1, 12, 128, BF16)]


@pytest.mark.parametrize("hd,kv_heads,group,page,dtype", SHAPES)
@pytest.mark.parametrize("tokens,lengths", [([1, 3], [1, 3]), ([4, 2, 0], [200, 2, 70]), ([8, 5], [700, 69]), ([16, 1, 9], [333, 64, 9]),
                                            ([33, 12], [96, 500]), ([63] * 3, [1000, 63, 130]), ([200], [260])])
def test_trees(tokens, lengths, hd, kv_heads, group, page, dtype):
    rng = np.random.default_rng(sum(tokens) + group)
    c = Case(lengths, kv_heads, hd, page, seed=sum(tokens))
    seen = [ora.tree_seen(random_tree(rng, t))[0] for t in tokens]
    assert_near(*attend_tree(c, queries(sum(tokens), kv_heads * group, hd, dtype), seen))


@pytest.mark.parametrize("tokens", [[4, 3], [40, 3], [90, 130]])
def test_a_chain_is_causal(tokens):
    """The tree in which every node hangs on the one before it, bit for bit as kfl_kv4_attend: the same keys in the same order."""
    c = Case([400, 222], 2, 128, 64, seed=5)
    q = queries(sum(tokens), 16, 128)
    got, lse, *ref = attend_tree(c, q, [np.tril(np.ones((t, t), dtype=bool)) for t in tokens])
    causal, causal_lse = c.run(q, tokens=tokens)
    assert_near(got, lse, *ref)
    assert (got.float() - causal.float()).abs().max() <= 2.0 ** -6 and (lse - causal_lse).abs().max() <= 2.0 ** -8


@pytest.mark.parametrize("group,tokens", [(8, [3, 4]), (3, [2, 9]), (8, [30, 11]), (5, [100, 64])])
@pytest.mark.parametrize("window", [1, 3, 17, 64, 200, 5000])
def test_windows(window, group, tokens):
    rng = np.random.default_rng(window)
    c = Case([300, 129], 2, 128, 32, seed=window)
    seen = [ora.tree_seen(random_tree(rng, t, 3))[0] for t in tokens]
    assert_near(*attend_tree(c, queries(sum(tokens), 2 * group, 128), seen, window=window))


@pytest.mark.parametrize("group,tokens", [(4, [2, 7]), (8, [20, 64])])
def test_any_bits(group, tokens):
    """Views that are no trees': later nodes, none at all; bits behind the last node count for nothing."""
    rng = np.random.default_rng(3)
    c = Case([250, tokens[1]], 2, 64, 16, seed=3)  # the second has no context: a row without bits sees nothing
    seen = [rng.random((t, t)) < 0.4 for t in tokens]
    for s in seen:
        s[0] = False
    max_q = max(tokens) + 40
    views = views_of(seen, max_q)
    for i, t in enumerate(tokens):  # rubbish behind the nodes
        rows = slice(sum(tokens[:i]), sum(tokens[:i + 1]))
        noise = ora.tree_words(rng.random((t, max_q)) < np.where(np.arange(max_q) < t, 0.0, 0.5), max_q).view(np.int32)
        views[rows] |= torch.from_numpy(noise).cuda()
    got, lse, ref, size, ref_lse = attend_tree(c, queries(sum(tokens), 2 * group, 64), seen, max_q=max_q, views=views)
    assert_near(got, lse, ref, size, ref_lse)
    assert (got[tokens[0]] == 0).all() and torch.isneginf(lse[tokens[0]]).all()


@pytest.mark.parametrize("group,tokens", [(4, [6]), (8, [40])])
def test_fewer_rows_than_nodes(group, tokens):
    """Nodes stand at the user's last rows: the first ones of a tree that is longer than them are not there."""
    c = Case([4], 1, 64, 16, seed=3)
    rng = np.random.default_rng(3)
    seen = [ora.tree_seen(random_tree(rng, tokens[0], 9))[0]]
    assert_near(*attend_tree(c, queries(tokens[0], group, 64), seen))


@pytest.mark.parametrize("tokens", [[3, 1, 2], [30, 50, 2]])
def test_users_layers_and_strides(tokens):
    rng = np.random.default_rng(1)
    c = Case([90, 200, 33, 257], 2, 128, 32, layers=3, seed=4)
    seen = [ora.tree_seen(random_tree(rng, t))[0] for t in tokens]
    q = queries(sum(tokens), 3 * 16, 128).cuda()[:, 16:32]
    out = torch.full((16, sum(tokens), 128), 7.0, dtype=BF16, device="cuda").transpose(0, 1)
    assert_near(*attend_tree(c, q, seen, users=[3, 0, 3], layer=2, out=out))
    odd = torch.zeros(sum(tokens), 16, 131, dtype=BF16, device="cuda")[..., 3:]  # rows off 16 bytes
    odd.copy_(q)
    out = torch.zeros(sum(tokens), 16, 129, dtype=BF16, device="cuda")[..., :128]
    assert_near(*attend_tree(c, odd, seen, users=[1, 1, 0], layer=1, out=out))


@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("group,tokens", [(4, 4), (8, 8), (8, 40), (4, 64)])
def test_nan_of_a_node_reaches_only_its_descendants(group, tokens, which):
    rng = np.random.default_rng(tokens)
    c = Case([100 + tokens], 2, 128, 16, seed=9)
    seen = ora.tree_seen(random_tree(rng, tokens, 3))[0]
    node = next(j for j in range(1, tokens) if 1 < seen[:, j].sum() < tokens - 1)
    c.params(0, 100 + node, 0, 1, which)[1] = np.nan
    got, *_ = attend_tree(c, queries(tokens, 2 * group, 128), [seen], lse=False)
    bad = torch.isnan(got.float()).cpu().numpy()
    assert not bad[:, :group].any() and not bad[~seen[:, node]].any()
    assert bad[seen[:, node]][:, group:, 64:].all()
    assert bad[seen[:, node]][:, group:, :64].all() == (which == 0)


@pytest.mark.parametrize("tokens", [[2, 2, 1], [20, 33, 1]])
def test_bad_users_and_pages_are_reported(tokens):
    c = Case([100, 100, 100], 1, 64, 16, seed=8)
    seen = [np.tril(np.ones((t, t), dtype=bool)) for t in tokens]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = queries(sum(tokens), 4, 64)
    good = attend_tree(c, q, seen, status=status)[0]
    assert status.item() == 0
    c.table[1, 2] = 10 ** 6
    kv4, at = c.kv4, tokens[0]
    dev = {n: torch.from_numpy(getattr(c, n)).cuda() for n in ("pool", "table", "lengths", "refs")}
    pool, m = kv4.pool(dev["pool"], 16, 1, 1, 64), kv4.page_map(dev["table"], dev["lengths"], dev["refs"])
    for users, bits in ((None, kv4.KFL_BAD_PAGE), ([0, 9, 2], kv4.KFL_BAD_USER)):
        status.zero_()
        bad = torch.full_like(good, 7.0)
        kv4.kfl_kv4_attend_tree(pool, m, 0, q.cuda(), bad, views_of(seen, max(tokens)),
                                kv4.attend_workspace(pool, 4, 3, sum(tokens), max(tokens)), q_start=starts(tokens),
                                users=None if users is None else i32(users), max_q=max(tokens), status=status)
        assert status.item() == bits and torch.isfinite(bad.float()).all()
        assert torch.equal(good[:at], bad[:at]) and torch.equal(good[-1:], bad[-1:])


def test_one_workspace_and_captured_calls():
    """The causal and the tree call by turns on one workspace, and both replayed in a graph."""
    c = Case([3000, 17, 2100, 64], 2, 128, 64, seed=8)
    kv4, tokens = c.kv4, [40, 3, 64, 9]
    rng = np.random.default_rng(4)
    seen = [ora.tree_seen(random_tree(rng, t))[0] for t in tokens]
    dev = {n: torch.from_numpy(getattr(c, n)).cuda() for n in ("pool", "table", "lengths", "refs")}
    pool, m = kv4.pool(dev["pool"], 64, 1, 2, 128), kv4.page_map(dev["table"], dev["lengths"], dev["refs"])
    ws = kv4.attend_workspace(pool, 16, 4, 116, 64)
    q, views, start = queries(116, 16, 128).cuda(), views_of(seen, 64), starts(tokens)
    outs = [torch.zeros_like(q) for _ in range(2)]

    def both():
        stream = torch.cuda.current_stream().cuda_stream
        kv4.kfl_kv4_attend_tree(pool, m, 0, q, outs[0], views, ws, q_start=start, max_q=64, cuda_stream=stream)
        kv4.kfl_kv4_attend(pool, m, 0, q, outs[1], ws, q_start=start, max_q=64, cuda_stream=stream)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    want = [o.clone() for o in outs]
    assert torch.equal(want[1], c.run(q, tokens=tokens)[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for o in outs:
        o.zero_()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_more_sequences_than_one_launch_takes():
    rng = np.random.default_rng(2)
    tokens = [1 + i % 3 for i in range(600)]
    c = Case([t + (i * 37) % 60 for i, t in enumerate(tokens)], 1, 64, 32, seed=8)
    seen = [ora.tree_seen(random_tree(rng, t))[0] for t in tokens]
    assert_near(*attend_tree(c, queries(sum(tokens), 2, 64), seen))
    tokens = [20 + i % 7 for i in range(530)]  # the many-row kernel
    c = Case([t + (i * 11) % 60 for i, t in enumerate(tokens)], 1, 64, 32, seed=9)
    seen = [ora.tree_seen(random_tree(rng, t))[0] for t in tokens]
    assert_near(*attend_tree(c, queries(sum(tokens), 4, 64), seen))


@pytest.mark.parametrize("hd,group,dtype", [(128, 4, BF16), (64, 2, FP16)])
def test_the_largest_trees(hd, group, dtype):
    """1024 nodes: their words fill a row of 32, and several tiles are theirs alone."""
    rng = np.random.default_rng(7)
    c = Case([1024 + 77, 1024], 1, hd, 64, seed=2)
    seen = [ora.tree_seen(random_tree(rng, 1024, s))[0] for s in (40, 3)]
    assert_near(*attend_tree(c, queries(2048, group, hd, dtype), seen))


def test_long_contexts_cut_between_blocks():
    """Row blocks whose tiles several thread blocks share, the nodes in the last one's."""
    rng = np.random.default_rng(8)
    c = Case([9000, 40, 3333], 1, 128, 128, seed=2)
    for tokens in ([5, 2, 1], [60, 33, 50]):
        seen = [ora.tree_seen(random_tree(rng, t))[0] for t in tokens]
        assert_near(*attend_tree(c, queries(sum(tokens), 8, 128), seen))
