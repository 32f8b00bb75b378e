"""The session's trees, accepted paths and evictions, run together as a serving loop does, against the 64-bit oracle.

After every pass each layer's outputs are held against attention over the rows that the cache holds (read from its bytes), with
the keys that the tokens should see, at the queries' true positions; keys in the cache against the rotated inputs, within
half a step of their coding; masses against sums of the oracle's weights.  Tolerances: outputs as in test_gpu_kv4_tree, plus the
rounding of the rotated queries to bf16 (2^-9 of each of head_dim terms, 2^-8 of a score of a few at six deviations: 2^-6 of the
weighted mean size at most); masses, whose weights are off by the same, 2^-5.
"""
import numpy as np
import pytest
import torch

import oracle.kv4 as ora
from gpu_helpers import ensure_built

pytestmark = pytest.mark.gpu
HD, KV, GROUP, PAGE, LAYERS = 64, 2, 4, 16, 2


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()
    torch.cuda.init()


class Loop:
    """A session beside what its cache should hold: every user's rows as (position, k, v) per layer and head."""

    def __init__(self, **kw):
        from paper_2609_34045_gb300.kv4_session import Session
        self.s = Session(LAYERS, KV * GROUP, KV, HD, n_users=4, max_ctx=256, n_pages=70, page_tokens=PAGE, masses=True,
                         max_positions=1024, **kw)
        self.rng = np.random.default_rng(5)
        self.rows = [[[[] for _ in range(KV)] for _ in range(LAYERS)] for _ in range(4)]
        self.mass = np.zeros((LAYERS, 4, KV, self.s.mass.shape[3]))
        self.next = [0] * 4  # true positions
        self.freq = 1e6 ** (-np.arange(0, HD, 2) / HD)

    def cached(self, user, layer, head, n):
        pool = self.s.pages.cpu().numpy().reshape(-1, LAYERS, KV, PAGE * HD * 9 // 8)
        return ora.rows(pool, self.s.table[user].cpu().numpy(), layer, head, n, PAGE, HD)

    def turned(self, x, positions):
        return ora.rotate(x.double().numpy(), np.asarray(positions)[:, None] * self.freq, False)

    def run(self, counts, parents=None, window=0):
        step = self.s.begin(counts, parents)
        n = sum(counts.values())
        seen, positions, users = {}, [], []
        for u, c in counts.items():
            tree = (parents or {}).get(u, list(range(-1, c - 1)))
            seen[u], depth = ora.tree_seen(tree) if parents is not None else (np.tril(np.ones((c, c), dtype=bool)), np.arange(c))
            positions += [self.next[u] + int(d) for d in depth]
            users += [u] * c
        assert step["positions"].tolist() == positions
        g = torch.Generator().manual_seed(int(self.rng.integers(1 << 30)))
        data = []
        for layer in range(LAYERS):
            q, k, v = (torch.randn(n, h, HD, generator=g).to(torch.bfloat16) for h in (KV * GROUP, KV, KV))
            out = self.s.attend(layer, step, q.cuda(), k.cuda(), v.cuda(), window=window).double().cpu().numpy()
            qt, kt = self.turned(q, positions), self.turned(k, positions)
            for t, u in enumerate(users):
                for h in range(KV):
                    self.rows[u][layer][h].append((positions[t], kt[t, h], v[t, h].double().numpy()))
            data.append((q, qt))
            self.check_layer(layer, counts, seen, qt, out, window, parents is None)
        assert self.s.status.item() == 0
        self.check_masses()
        return step, (counts, seen, data)

    def check_layer(self, layer, counts, seen, qt, out, window, weigh):
        at = 0
        for u, c in counts.items():
            n = len(self.rows[u][layer][0])
            assert int(self.s.lengths[u]) == n
            keys = ora.causal_keys(c, n, window) if weigh else ora.tree_keys(seen[u], n, window)
            for h in range(KV):
                k, v = self.cached(u, layer, h, n)
                for got, want in ((k, [r[1] for r in self.rows[u][layer][h]]), (v, [r[2] for r in self.rows[u][layer][h]])):
                    want = np.array(want).reshape(n, HD)
                    step = (want.max(1) - want.min(1))[:, None] / 15 if n else 0
                    assert (np.abs(got - want) <= 0.52 * step + 2.0 ** -6).all()  # half a step; k is rounded to bf16 where slots moved
                for j in range(h * GROUP, (h + 1) * GROUP):
                    ref, size, lse = ora.attend_keys(qt[at:at + c, j], k, v, keys, HD ** -0.5)
                    assert (np.abs(out[at:at + c, j] - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -6 * (size + 1)).all()
                    if weigh:
                        self.mass[layer, u, h, :n] += ora.weights(qt[at:at + c, j], k, lse, keys, HD ** -0.5).sum(0)
            at += c

    def check_masses(self):
        got = self.s.mass.double().cpu().numpy()
        assert (np.abs(got - self.mass) <= 2.0 ** -5 * self.mass + 1e-6).all()
        for u in range(4):
            assert (got[:, u, :, len(self.rows[u][0][0]):] == 0).all()

    def advance(self, counts):
        for u, c in counts.items():
            self.next[u] += c

    def accept(self, step, info, paths, window=0):
        counts, seen, data = info
        self.s.accept(step, paths)
        for u, c in counts.items():
            path = paths.get(u, [])
            for layer in range(LAYERS):
                for h in range(KV):
                    rows = self.rows[u][layer][h]
                    base = len(rows) - c
                    self.rows[u][layer][h] = rows[:base] + [rows[base + j] for j in path]
            self.next[u] += len(path)
        at = 0
        for u, c in counts.items():
            path = paths.get(u, [])
            n = len(self.rows[u][0][0])
            assert int(self.s.lengths[u]) == n
            keys = ora.causal_keys(len(path), n, window)
            for layer in range(LAYERS):
                for h in range(KV):
                    k, v = self.cached(u, layer, h, n)
                    for j in range(h * GROUP, (h + 1) * GROUP):
                        x = data[layer][1][[at + i for i in path], j].reshape(len(path), HD)
                        lse = ora.attend_keys(x, k, v, keys, HD ** -0.5)[2]
                        self.mass[layer, u, h, :n] += ora.weights(x, k, lse, keys, HD ** -0.5).sum(0)
            at += c
        assert self.s.status.item() == 0
        self.check_masses()

    def evict(self, budget, users, first, recent):
        before = self.s.mass.cpu().numpy()
        lost = self.s.evict(budget, users, first=first, recent=recent)
        for u in users:
            n = len(self.rows[u][0][0])
            assert lost.get(u, 0) == max(0, n - budget)
            for layer in range(LAYERS):
                for h in range(KV):
                    keep = ora.select(before[layer, u, h], n, budget, first, recent)
                    self.rows[u][layer][h] = [self.rows[u][layer][h][i] for i in keep]
                    kept = self.mass[layer, u, h, keep]
                    self.mass[layer, u, h] = 0
                    self.mass[layer, u, h, :len(keep)] = kept
        assert self.s.status.item() == 0
        self.check_masses()
        # every page is held by as many users as say so
        held = np.bincount(self.s.table[self.s.table >= 0].cpu().numpy(), minlength=70)
        assert np.array_equal(held, self.s.refs.cpu().numpy())


TREE = [-1, 0, 0, 1, 1, 2, -1, 6]


@pytest.mark.parametrize("window", [0, 40])
def test_a_loop_of_prompts_drafts_and_evictions(window):
    loop = Loop()
    counts = {0: 70, 1: 33, 3: 5}
    loop.run(counts, window=window)
    loop.advance(counts)
    for _ in range(2):
        step, info = loop.run({0: 8, 3: 8, 1: 3}, {0: TREE, 3: TREE}, window=window)
        loop.accept(step, info, {0: [0, 1, 4], 3: [6, 7], 1: [0]}, window)
    loop.evict(40, [0, 1, 3], 4, 10)
    for counts in ({0: 1, 1: 1, 3: 1}, {0: 1, 3: 1}):
        loop.run(counts, window=window)
        loop.advance(counts)
    step, info = loop.run({0: 8, 1: 8}, {0: TREE, 1: TREE}, window=window)  # positions beyond the slots
    loop.accept(step, info, {0: [0, 2, 5]}, window)                          # nothing of user 1's tree stays
    loop.evict(20, [0, 3], 0, 0)
    loop.run({0: 20, 3: 1}, window=window)


def test_shared_pages_are_left_to_the_others():
    """A fork, an eviction of one of the two, then of the other: each goes on with rows of its own."""
    loop = Loop()
    loop.run({0: 70})
    loop.advance({0: 70})
    loop.s.fork([0], [2])
    loop.rows[2] = [[list(r) for r in layer] for layer in loop.rows[0]]
    loop.next[2], loop.mass[:, 2] = loop.next[0], loop.mass[:, 0]
    loop.check_masses()
    loop.evict(30, [2], 2, 5)
    loop.run({0: 1, 2: 1})
    loop.advance({0: 1, 2: 1})
    loop.evict(30, [0], 2, 5)
    loop.run({0: 2, 2: 2})
    loop.s.free([0])
    loop.rows[0], loop.mass[:, 0], loop.next[0] = [[[] for _ in range(KV)] for _ in range(LAYERS)], 0, 0
    loop.run({0: 3, 2: 0})


def test_evictions_without_room_for_shared_pages_are_refused():
    from paper_2609_34045_gb300.kv4_session import NoRoom, Session
    s = Session(1, 4, 2, 64, n_users=2, max_ctx=64, n_pages=5, page_tokens=16, masses=True)
    s.begin({0: 64})
    s.fork([0], [1])
    table, lengths = s.table.clone(), s.lengths.clone()
    with pytest.raises(NoRoom):
        s.evict(40, [1], recent=8)
    assert torch.equal(s.table, table) and torch.equal(s.lengths, lengths) and s.evicted == [0, 0]
    assert s.evict(16, [1], first=0, recent=0) == {1: 48} and s.lengths.tolist() == [64, 16]


@pytest.mark.parametrize("masses", [False, True])
def test_users_that_there_are_none_of_are_reported_when_freed(masses):
    from paper_2609_34045_gb300.kv4 import KFL_BAD_USER
    from paper_2609_34045_gb300.kv4_session import Session
    s = Session(1, 4, 2, 64, n_users=2, max_ctx=64, n_pages=8, page_tokens=16, masses=masses)
    s.begin({0: 20, 1: 30})
    s.evicted = [3, 5]
    if masses:
        s.mass.fill_(1)
    s.free([-1, 2, 0])
    assert s.status.item() == KFL_BAD_USER and s.lengths.tolist() == [0, 30] and s.evicted == [0, 5]
    if masses:
        assert not s.mass[:, 0].any() and (s.mass[:, 1] == 1).all()
    s.free([])
    assert s.lengths.tolist() == [0, 30]


def test_a_window_shorter_than_a_path_is_refused_where_masses_are_kept():
    """(A node sees all of its path, whatever the window; the accepted tokens' weights are those of the window's rows.)"""
    from paper_2609_34045_gb300.kv4_session import Session
    for masses in (False, True):
        s = Session(1, 4, 2, 64, n_users=2, max_ctx=64, n_pages=8, page_tokens=16, masses=masses)
        q, k = (torch.randn(9, h, 64, device="cuda").to(torch.bfloat16) for h in (4, 2))
        step = s.begin({0: 5, 1: 4}, {1: [-1, 0, 0, 2]})  # a chain of five, and a path of three
        if masses:
            before = s.pages.clone()
            with pytest.raises(ValueError):
                s.attend(0, step, q, k, k, window=4)
            assert torch.equal(s.pages, before)
        else:
            s.attend(0, step, q, k, k, window=4)
        s.attend(0, step, q, k, k, window=5)
        s.accept(step, {0: [0, 1, 2, 3, 4], 1: [0, 2, 3]})
        assert s.lengths.tolist() == [5, 3] and s.status.item() == 0
        if masses:  # an accepted token's weights sum to one in each of four heads, to 1e-5 (lse, weights)
            got = s.mass[0, :2].sum(dim=(1, 2)).tolist()
            assert got == pytest.approx([20, 12], abs=1e-3)
