"""Forms of the tree and eviction operators that the other tests do not take: scales of their own, a chain to the bit, every call on a
side stream and captured, and the session's passes with what its kernels were really given.

Tolerances: attention as in test_gpu_kv4_tree; weights as in test_gpu_kv4_weights_range.  The session's queries are taken as they
reach the kernel (turned and rounded), its log-sum-exps as kfl_kv4_attend wrote them, its keys and values from the pages: nothing is
left to allow for but the operators' own errors.
"""
import numpy as np
import pytest
import torch

import oracle.kv4 as ora
from gpu_helpers import ensure_built
from test_gpu_kv4_attend import BF16, FP16, Case, assert_near, queries
from test_gpu_kv4_tree import attend_tree, i32, random_tree, starts, views_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()
    torch.cuda.init()


@pytest.mark.parametrize("group,tokens,dtype", [(4, [3, 9], BF16), (8, [8, 2], FP16), (8, [40, 3], BF16), (4, [100, 64], FP16)])
@pytest.mark.parametrize("scale,std", [(0.0, 1.0), (-0.05, 1.0), (-1.0, 0.1), (128 ** -0.5 / 1000, 1000.0)])
@pytest.mark.parametrize("window", [0, 20])
def test_trees_with_a_scale_of_their_own(scale, std, group, tokens, dtype, window):
    rng = np.random.default_rng(sum(tokens))
    c = Case([300, 129], 2, 128, 32, seed=7)
    seen = [ora.tree_seen(random_tree(rng, t))[0] for t in tokens]
    assert_near(*attend_tree(c, queries(sum(tokens), 2 * group, 128, dtype, std=std), seen, scale=scale, window=window))


@pytest.mark.parametrize("hd,group,tokens,dtype", [(128, 8, [4, 3], BF16), (64, 4, [1, 2], FP16), (128, 5, [3, 12], BF16)])
def test_a_chain_of_few_rows_is_causal_to_the_bit(hd, group, tokens, dtype):
    """The same keys in the same tiles.  (Not so with many rows: a tree's row blocks read the tiles behind their last token too, so the
    list is cut at other places.)"""
    c = Case([700, 222], 2, hd, 64, seed=5)
    q = queries(sum(tokens), 2 * group, hd, dtype)
    got, lse, *_ = attend_tree(c, q, [np.tril(np.ones((t, t), dtype=bool)) for t in tokens])
    causal, causal_lse = c.run(q, tokens=tokens)
    assert torch.equal(got, causal) and torch.equal(lse, causal_lse)


@pytest.mark.parametrize("tokens", [[3, 2], [40, 9]])
def test_a_step_of_trees_on_a_side_stream_and_captured(tokens):
    """Views, attention, and the weights, the choice and the keeping of rows, one behind the other; replayed on other inputs."""
    c = Case([600, 90], 2, 128, 32, seed=6)
    kv4 = c.kv4
    group, n, max_q = 4, sum(tokens), max(tokens)
    dev = {name: torch.from_numpy(getattr(c, name)).cuda() for name in ("pool", "table", "lengths", "refs")}
    pool, m = kv4.pool(dev["pool"], 32, 1, 2, 128), kv4.page_map(dev["table"], dev["lengths"], dev["refs"])
    rng = np.random.default_rng(2)
    trees = [[random_tree(rng, t) for t in tokens] for _ in range(2)]
    parents, q = i32(sum(trees[0], [])), queries(n, 2 * group, 128).cuda()
    start, users = starts(tokens), i32([0, 1])
    views, positions = torch.empty(n, -(-max_q // 32), dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
    out, lse, mass = torch.empty_like(q), torch.empty(n, 2 * group, device="cuda"), torch.zeros(1, 2, 2, c.table.shape[1] * 32, device="cuda")
    rows, counts = torch.empty(1, 2, 2, 50, dtype=torch.int32, device="cuda"), torch.empty(2, dtype=torch.int32, device="cuda")
    ws, scratch, status = kv4.attend_workspace(pool, 2 * group, 2, n, max_q), kv4.pages_workspace(pool), torch.zeros(1, dtype=torch.int32, device="cuda")
    state = [dev["pool"], dev["table"], dev["lengths"], dev["refs"], mass]
    kept = [t.clone() for t in state]

    def step():
        stream = dict(status=status, cuda_stream=torch.cuda.current_stream().cuda_stream)
        kv4.kfl_kv4_tree(parents, views, positions, q_start=start, max_q=max_q, **stream)
        kv4.kfl_kv4_attend_tree(pool, m, 0, q, out, views, ws, q_start=start, max_q=max_q, lse=lse, **stream)
        kv4.kfl_kv4_weights(pool, m, 0, q, lse, mass, ws, q_start=start, max_q=max_q, **stream)
        kv4.kfl_kv4_select(pool, m, mass, users, 50, rows, counts, first=2, recent=10, **stream)
        kv4.kfl_kv4_keep(pool, m, users, rows, counts, scratch, mass=mass, **stream)

    def inputs(i):
        parents.copy_(i32(sum(trees[i], [])))
        q.copy_(queries(n, 2 * group, 128, seed=5 + i))
        for t, x in zip(state, kept):
            t.copy_(x)

    outputs = [out, lse, views, positions, rows, counts, *state]
    side = torch.cuda.Stream()
    want = []
    for i in range(2):
        inputs(i)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        want.append([t.clone() for t in outputs])
    seen = [ora.tree_seen(t)[0] for t in trees[0]]
    assert np.array_equal(want[0][2].cpu().numpy(), views_of(seen, max_q).cpu().numpy())
    assert torch.equal(want[0][0], attend_tree(c, queries(n, 2 * group, 128, seed=5), seen)[0])
    assert not torch.equal(want[0][4], want[1][4]) and want[0][8].tolist() == [50, 50]
    inputs(0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in (0, 1, 0):
        inputs(i)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outputs, want[i]))
    assert status.item() == 0


# ---- the session, with what its kernels are given

KV, GROUP, HD, PAGE = 2, 4, 64, 16


class Watched:
    """A session of one layer whose calls of attention and of weights are checked one by one."""

    def __init__(self, monkeypatch):
        from paper_2609_34045_gb300 import kv4
        from paper_2609_34045_gb300.kv4_session import Session
        self.kv4 = kv4
        self.s = Session(1, KV * GROUP, KV, HD, n_users=3, max_ctx=256, n_pages=60, page_tokens=PAGE, masses=True, max_positions=1024)
        self.seen, self.calls = None, []
        for name in ("kfl_kv4_attend", "kfl_kv4_attend_tree", "kfl_kv4_weights"):
            monkeypatch.setattr(kv4, name, lambda *a, _real=getattr(kv4, name), _name=name, **kw: self.call(_real, _name, a, kw))

    def call(self, real, name, a, kw):
        mass = self.s.mass.double().cpu().numpy()
        real(*a, **kw)
        self.calls.append(name)
        q = a[3].double().cpu().numpy()
        users = kw["users"].tolist()
        start = list(range(len(users) + 1)) if kw["q_start"] is None else kw["q_start"].tolist()
        pool = self.s.pages.cpu().numpy().reshape(-1, 1, KV, PAGE * HD * 9 // 8)
        ref, size, ref_lse = np.zeros(q.shape), np.zeros(q.shape), np.zeros(q.shape[:2])
        want, slack = mass.copy(), np.zeros(mass.shape)
        for i, u in enumerate(users):
            rows = slice(start[i], start[i + 1])
            n, t = int(self.s.lengths[u]), start[i + 1] - start[i]
            table = self.s.table[u].cpu().numpy()
            keys = ora.tree_keys(self.seen[u], n, kw["window"]) if name == "kfl_kv4_attend_tree" else ora.causal_keys(t, n, kw["window"])
            for h in range(KV):
                k, v = ora.rows(pool, table, 0, h, n, PAGE, HD)
                par = [ora.unpack(pool[table[s // PAGE], 0, h], PAGE, HD) for s in range(n)]
                centre = np.array([np.repeat(p[3][s % PAGE, :, 1].astype(np.float64), 64) for s, p in enumerate(par)]).reshape(n, HD)
                reach = np.array([np.repeat(np.abs(p[2][s % PAGE].astype(np.float64)) @ [16, 1], 64) for s, p in enumerate(par)]).reshape(n, HD)
                for j in range(h * GROUP, (h + 1) * GROUP):
                    x = q[rows, j]
                    if name == "kfl_kv4_weights":
                        lse = a[4][rows, j].double().cpu().numpy()
                        w = ora.weights(x, k, lse, keys, HD ** -0.5)
                        off = 2.0 ** -19 * (HD ** -0.5 * (np.abs(x) @ reach.T) + np.abs(np.where(np.isfinite(lse), lse, 0))[:, None]) + 2.0 ** -22
                        want[0, u, h, :n] += w.sum(0)
                        slack[0, u, h, :n] += (w * off).sum(0)
                    else:
                        ref[rows, j], size[rows, j], ref_lse[rows, j] = ora.attend_keys(x, k, v, keys, HD ** -0.5)
                        size[rows, j] += ora.attend_keys(x, k, v - centre, keys, HD ** -0.5)[1]
        if name == "kfl_kv4_weights":
            got = self.s.mass.double().cpu().numpy()
            assert (np.abs(got - want) <= slack + (kw["max_q"] * GROUP + 3) * 2.0 ** -24 * np.abs(want)).all()
        else:
            assert_near(a[4], kw["lse"], ref, size, ref_lse)

    def run(self, counts, seed, parents=None, window=0):
        step = self.s.begin(counts, parents)
        if parents is not None:
            self.seen = {u: ora.tree_seen(parents.get(u, list(range(-1, n - 1))))[0] for u, n in counts.items()}
        g, n = torch.Generator().manual_seed(seed), sum(counts.values())
        q, k, v = (torch.randn(n, h, HD, generator=g).to(BF16).cuda() for h in (KV * GROUP, KV, KV))
        self.s.attend(0, step, 2 * q, 2 * k, v, window=window)  # (scores of some deviations of 4: a few keys have the weight)
        return step


TREE = [-1, 0, 0, 1, 1, 2, -1, 6]


@pytest.mark.parametrize("window", [0, 40])
def test_a_session_call_by_call(window, monkeypatch):
    w = Watched(monkeypatch)
    w.run({0: 70, 1: 33}, 1, window=window)
    step = w.run({0: 8, 1: 3}, 2, {0: TREE}, window=window)
    w.s.accept(step, {0: [0, 1, 4], 1: [0]})
    w.s.evict(40, [0], first=4, recent=10)
    w.run({0: 1, 1: 1}, 3, window=window)
    step = w.run({1: 8, 0: 8}, 4, {0: TREE, 1: TREE}, window=window)
    w.s.accept(step, {0: [0, 2, 5], 1: [6, 7]})
    w.run({2: 20, 0: 2}, 5, window=window)
    assert w.s.status.item() == 0
    assert w.calls.count("kfl_kv4_attend_tree") == 2 and w.calls.count("kfl_kv4_weights") == 5
