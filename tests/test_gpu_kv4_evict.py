"""Rows that leave the 4-bit paged cache, against the 64-bit oracle: weights within the bounds below, the choice of rows and
their moving to the bit.

Tolerance of a weight exp(x - lse).  The products of codes and queries are exact; a score x = scale sum_g (s acc + c sum q) comes from
fp32 sums of at most 8 products of 16 terms each and a few fp32 steps, each off by at most 2^-23 of the largest magnitude in it
(the matrix unit truncates), which is at most M = scale sum_c (16 s_c + |c_c|) |q_c|: 16 steps, 2^-19 M.  The exponent's
argument, x log2(e) - lse log2(e), is rounded three times at up to 1.5 (|x| + |lse|) each: 2^-21 (|x| + |lse|).  The
exponential is off by 2^-22, and the sum of r weights by at most (r + 2) 2^-24 of itself.
"""
import numpy as np
import pytest
import torch

import oracle.kv4 as ora
from gpu_helpers import ensure_built
from test_gpu_kv4_attend import BF16, FP16, Case, queries
from test_gpu_kv4_tree import i32, starts

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()
    torch.cuda.init()


def lse_of(c, q, tokens, users, layer, window, scale):
    """The rows' log-sum-exp in fp32, from the oracle."""
    x, group = q.double().cpu().numpy(), q.shape[1] // c.pool.shape[2]
    out, at = np.zeros(x.shape[:2], dtype=np.float32), 0
    for u, t in zip(users, tokens):
        n = int(c.lengths[u])
        keys = ora.causal_keys(t, n, window)
        for j in range(x.shape[1]):
            k, v = ora.rows(c.pool, c.table[u], layer, j // group, n, c.page, c.hd)
            out[at:at + t, j] = ora.attend_keys(x[at:at + t, j], k, v, keys, scale)[2]
        at += t
    return out


def check_weights(c, q, tokens=None, users=None, layer=0, window=0, scale=None, lse=None, max_q=None, tile=None):
    kv4 = c.kv4
    seqs = [1] * q.shape[0] if tokens is None else tokens
    who = list(range(len(seqs))) if users is None else users
    heads, group = c.pool.shape[2], q.shape[1] // c.pool.shape[2]
    s = c.hd ** -0.5 if scale is None else scale
    dev = {n: torch.from_numpy(getattr(c, n)).cuda() for n in ("pool", "table", "lengths", "refs")}
    pool, m = kv4.pool(dev["pool"], c.page, c.layers, heads, c.hd), kv4.page_map(dev["table"], dev["lengths"], dev["refs"])
    lse = lse_of(c, q, seqs, who, layer, window, s) if lse is None else lse
    slots = c.table.shape[1] * c.page
    before = np.random.default_rng(2).random((c.layers, len(c.lengths), heads, slots)).astype(np.float32)
    mass = torch.from_numpy(before).cuda()
    max_q = max_q or max(1, *seqs)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kv4.kfl_kv4_weights(pool, m, layer, q.cuda(), torch.from_numpy(lse).cuda(), mass,
                        kv4.attend_workspace(pool, q.shape[1], len(seqs), q.shape[0], max_q),
                        users=None if users is None else i32(users), q_start=None if tokens is None else starts(tokens), max_q=max_q,
                        window=window, scale=scale, status=status)
    got = mass.cpu().numpy()
    want, slack = before.astype(np.float64), np.zeros(before.shape)
    at, x = 0, q.double().cpu().numpy()
    for u, t in zip(who, seqs):
        n = int(c.lengths[u])
        keys = ora.causal_keys(t, n, window)
        for h in range(heads):
            k, _ = ora.rows(c.pool, c.table[u], layer, h, n, c.page, c.hd)
            reach = np.zeros((n, c.hd))
            for slot in range(n):
                p = np.abs(c.params(u, slot, layer, h, 0).astype(np.float64))
                reach[slot] = np.repeat(16 * p[:, 0] + p[:, 1], 64)
            for j in range(h * group, (h + 1) * group):
                qj, l = x[at:at + t, j], lse[at:at + t, j].astype(np.float64)
                w = ora.weights(qj, k, l, keys, s)
                off = 2.0 ** -19 * abs(s) * (np.abs(qj) @ reach.T) + 2.0 ** -21 * (np.abs(qj @ k.T * s) + np.abs(np.where(np.isfinite(l), l, 0))[:, None]) + 2.0 ** -22
                want[layer, u, h, :n] += w.sum(0)
                slack[layer, u, h, :n] += (w * off).sum(0)
        at += t
    slack += ((max_q * group + 3) * 2.0 ** -24) * np.abs(want)
    assert (np.isnan(got) == np.isnan(want)).all()
    fine = ~np.isnan(want)
    worst = (np.abs(got - want) - slack)[fine].max()
    assert worst <= 0, worst
    untouched = np.ones(before.shape, dtype=bool)
    for u in who:
        untouched[layer, u, :, :int(c.lengths[u])] = False
    assert (got == before)[untouched].all()
    assert status.item() == 0
    return got, before


SHAPES = [(128, 2, 8, 64, BF16), (128, 2, 7, 16, FP16), (64, 2, 4, 32, BF16), (64, 1, 1, 128, FP16), (128, 1, 12, 128, BF16),
          (64, 3, 5, 16, FP16)]


@pytest.mark.parametrize("hd,kv_heads,group,page,dtype", SHAPES)
@pytest.mark.parametrize("tokens,lengths", [(None, [1, 15, 16, 17, 63, 64, 65, 300]), ([2, 1, 3], [300, 5, 64]), ([4, 0, 1], [4, 20, 130]),
                                            ([5, 2], [3, 0]), ([33, 12], [96, 500]), ([140], [700]), ([64, 200], [300, 210])])
def test_weights(tokens, lengths, hd, kv_heads, group, page, dtype):
    c = Case(lengths, kv_heads, hd, page, seed=hd + group)
    check_weights(c, queries(len(lengths) if tokens is None else sum(tokens), kv_heads * group, hd, dtype), tokens=tokens)


@pytest.mark.parametrize("group,tokens", [(8, None), (8, [3, 4]), (5, [100, 64])])
@pytest.mark.parametrize("window", [1, 17, 64, 200, 5000])
def test_windows(window, group, tokens):
    c = Case([300, 129], 2, 128, 32, seed=window)
    check_weights(c, queries(2 if tokens is None else sum(tokens), 2 * group, 128), tokens=tokens, window=window)


@pytest.mark.parametrize("tokens", [None, [30, 40]])
@pytest.mark.parametrize("scale,std", [(0.0, 1.0), (-0.05, 1.0), (1.0, 0.1), (128 ** -0.5 / 3000, 3000.0)])
def test_unusual_scales(scale, std, tokens):
    c = Case([150, 83], 2, 128, 16, seed=6)
    check_weights(c, queries(2 if tokens is None else 70, 8, 128, std=std), tokens=tokens, scale=scale)


@pytest.mark.parametrize("tokens", [[3, 1], [30, 50]])
def test_users_layers_and_strides(tokens):
    c = Case([90, 200, 33, 257], 2, 128, 32, layers=3, seed=4)
    q = queries(sum(tokens), 3 * 16, 128).cuda()[:, 16:32]
    check_weights(c, q, tokens=tokens, users=[3, 0], layer=2)
    odd = torch.zeros(sum(tokens), 16, 131, dtype=BF16, device="cuda")[..., 3:]
    odd.copy_(q)
    check_weights(c, odd, tokens=tokens, users=[1, 2], layer=1)


@pytest.mark.parametrize("group,tokens", [(4, 5), (8, 40)])
def test_nan_keys_rows_and_sums(group, tokens):
    """A NaN key makes its own mass NaN where a row sees it; a NaN row all that it sees; a row that saw nothing adds nothing, NaN
    keys included."""
    c = Case([100 + tokens], 2, 128, 16, seed=9)
    q = queries(tokens, 2 * group, 128)
    lse = lse_of(c, q, [tokens], [0], 0, 0, 128 ** -0.5)
    c.params(0, 57, 0, 1, 0)[1] = np.nan                # one group of a key of the second head
    got, _ = check_weights(c, q, tokens=[tokens], lse=lse)
    assert np.isnan(got).sum() == 1 and np.isnan(got[0, 0, 1, 57])
    c.params(0, 57, 0, 1, 0)[1] = np.inf
    assert not np.isfinite(check_weights_raw(c, q, tokens, lse)[0, 0, 1, 57])
    c.params(0, 57, 0, 1, 0)[1] = 0.0
    c.params(0, 100 + tokens - 1, 0, 0, 0)[0] = np.nan  # the last key: only the last token sees it
    lse[-1] = -np.inf                                   # which says that it saw nothing
    got = check_weights_raw(c, q, tokens, lse)
    assert np.isfinite(got).all()
    lse[-1], lse[2, 1] = 3.0, np.nan
    got = check_weights_raw(c, q, tokens, lse)
    assert np.isnan(got[0, 0, 0, :100 + 3]).all() and np.isfinite(got[0, 0, 0, 103:-1][: tokens - 4]).all()
    assert np.isfinite(got[0, 0, 1]).all()


def check_weights_raw(c, q, tokens, lse, mass=None, users=None, status=None):
    kv4, heads = c.kv4, c.pool.shape[2]
    dev = {n: torch.from_numpy(getattr(c, n)).cuda() for n in ("pool", "table", "lengths", "refs")}
    pool, m = kv4.pool(dev["pool"], c.page, c.layers, heads, c.hd), kv4.page_map(dev["table"], dev["lengths"], dev["refs"])
    mass = torch.zeros(c.layers, len(c.lengths), heads, c.table.shape[1] * c.page, device="cuda") if mass is None else mass
    tokens = [tokens] if isinstance(tokens, int) else tokens
    kv4.kfl_kv4_weights(pool, m, 0, q.cuda(), torch.from_numpy(lse).cuda(), mass,
                        kv4.attend_workspace(pool, q.shape[1], len(tokens), q.shape[0], max(tokens)), q_start=starts(tokens),
                        users=None if users is None else i32(users), max_q=max(tokens), status=status)
    return mass.cpu().numpy()


@pytest.mark.parametrize("tokens", [[2, 2, 1], [20, 33, 1]])
def test_users_twice_and_bad_pages_are_reported(tokens):
    c = Case([100, 100, 100], 1, 64, 16, seed=8)
    q = queries(sum(tokens), 4, 64)
    lse = lse_of(c, q, tokens, [0, 1, 2], 0, 0, 64 ** -0.5)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    good = check_weights_raw(c, q, tokens, lse, status=status)
    assert status.item() == 0
    for users, left in (([0, 7, 2], [0, 2]), ([0, 0, 2], [0, 2]), ([0, -1, 2], [0, 2])):
        status.zero_()
        got = check_weights_raw(c, q, tokens, lse, users=users, status=status)
        assert status.item() == c.kv4.KFL_BAD_USER
        assert (got[:, left] == good[:, left]).all() and (got[:, 1] == 0).all()
    c.table[1, 2] = 10 ** 6
    status.zero_()
    got = check_weights_raw(c, q, tokens, lse, status=status)
    assert status.item() == c.kv4.KFL_BAD_PAGE
    assert (got[:, [0, 2]] == good[:, [0, 2]]).all() and (got[0, 1, 0, 32:48] == 0).all() and (got[0, 1, 0, :32] == good[0, 1, 0, :32]).all()


def test_more_sequences_than_one_launch_takes():
    lengths = [1 + (i * 37) % 90 for i in range(700)]
    c = Case(lengths, 1, 64, 32, seed=8)
    q = queries(700, 2, 64)
    check_weights(c, q)
    users = list(range(700))
    users[650] = 3  # named before, in the first launch
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lse = np.zeros((700, 2), dtype=np.float32)
    got = check_weights_raw(c, q, [1] * 700, lse, users=users, status=status)
    assert status.item() == c.kv4.KFL_BAD_USER and (got[0, 650] == 0).all()


@pytest.mark.parametrize("tokens", [[1, 1, 1, 1], [300, 3, 64, 9]])
def test_weights_repeat_to_the_bit(tokens):
    c = Case([3000, 17, 2100, 64], 2, 128, 64, seed=8)
    q = queries(sum(tokens), 16, 128)
    lse = np.full((sum(tokens), 16), 5.0, dtype=np.float32)
    first = check_weights_raw(c, q, tokens, lse)
    for _ in range(4):
        assert (check_weights_raw(c, q, tokens, lse) == first).all()


# ---- the choice of rows

def run_select(lengths, mass, page, budget, first, recent, users=None, layers=1, heads=1, capacity=None, status=None):
    from paper_2609_34045_gb300 import kv4
    n = len(lengths)
    need = max(1, *[-(-v // page) for v in lengths])
    pages = capacity or need
    p = kv4.pool(None, page, layers, heads, 64, n_pages=10)
    m = kv4.page_map(torch.zeros(n, pages, dtype=torch.int32, device="cuda"), i32(lengths), torch.zeros(10, dtype=torch.int32, device="cuda"))
    users = list(range(n)) if users is None else users
    rows = torch.full((layers, len(users), heads, budget), 7, dtype=torch.int32, device="cuda")
    counts = torch.full((len(users),), 7, dtype=torch.int32, device="cuda")
    kv4.kfl_kv4_select(p, m, mass, i32(users), budget, rows, counts, first=first, recent=recent, status=status)
    return rows.cpu().numpy(), counts.cpu().numpy()


def check_select(lengths, budget, first, recent, page=64, layers=1, heads=1, kind="spread", users=None, capacity=None, strided=False):
    rng = np.random.default_rng(sum(lengths) + budget)
    slots = (capacity or max(1, *[-(-v // page) for v in lengths])) * page
    shape = (layers, len(lengths), heads, slots)
    mass = np.exp(3 * rng.standard_normal(shape)).astype(np.float32)
    if kind == "ties":
        mass = rng.integers(0, 4, shape).astype(np.float32)
    elif kind == "equal":
        mass[:] = 0.25
    elif kind == "odd":
        mass = rng.choice(np.array([0.0, -0.0, np.inf, -np.inf, np.nan, -np.nan, 1.0, -1.0, 1e-42, -1e-42, 3.4e38], dtype=np.float32), shape)
    t = torch.from_numpy(mass).cuda()
    if strided:
        t = torch.zeros(shape[1], shape[0], shape[2], shape[3] + 5, device="cuda")[..., 3:-2].transpose(0, 1).copy_(t)
    rows, counts = run_select(lengths, t, page, budget, first, recent, users, layers, heads, capacity)
    for i, u in enumerate(users if users is not None else range(len(lengths))):
        n = lengths[u]
        assert counts[i] == min(n, budget)
        for l in range(layers):
            for h in range(heads):
                want = ora.select(mass[l, u, h], n, budget, first, recent)
                assert np.array_equal(rows[l, i, h, :len(want)], want), (kind, i, l, h)
                assert (rows[l, i, h, len(want):] == -1).all()


@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "odd"])
@pytest.mark.parametrize("lengths,budget,first,recent", [([0, 1, 2, 3], 1, 0, 0), ([100, 33, 64], 33, 1, 4), ([700, 699, 1], 64, 4, 60),
                                                         ([5000], 1000, 0, 0), ([2049, 513], 512, 512, 0), ([4097], 4096, 3, 100)])
def test_select(lengths, budget, first, recent, kind):
    check_select(lengths, budget, first, recent, kind=kind)


@pytest.mark.parametrize("kind", ["spread", "ties", "equal"])
@pytest.mark.parametrize("length,budget", [(20000, 3333), (70000, 16384), (131072, 100000), (131072, 5)])
def test_select_of_long_rows(length, budget, kind):
    """Rows that a cluster of blocks shares, among short ones that its other blocks have nothing of."""
    check_select([length, 9000, 40], budget, 0, 0 if budget < 10 else 7, kind=kind, page=128)


def test_select_layers_heads_users_and_strides():
    check_select([300, 120, 777, 64], 100, 4, 10, layers=3, heads=2, users=[2, 0, 2, 3], strided=True)
    check_select([900] * 40, 100, 4, 10, layers=5, heads=8, page=16, capacity=700)


def test_select_reads_again_what_does_not_fit():
    """More keys of a block than its shared memory holds."""
    check_select([400000, 330001], 50000, 5, 1000, page=128)


def test_select_reports_bad_users():
    from paper_2609_34045_gb300 import kv4
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    mass = torch.rand(1, 2, 1, 128, device="cuda")
    rows, counts = run_select([100, 90], mass, 64, 16, 0, 4, users=[5, 1, -1], status=status)
    assert status.item() == kv4.KFL_BAD_USER and counts.tolist() == [0, 16, 0]
    assert (rows[0, [0, 2]] == -1).all() and (rows[0, 1] >= 0).all()


# ---- rows kept in place

class Cache:
    """Users' pages with random bytes, some of them held by several users, and masses."""

    def __init__(self, lengths, page, hd, layers, heads, seed, shared=(), spare=20):
        from paper_2609_34045_gb300 import kv4
        self.kv4, self.page, self.hd = kv4, page, hd
        rng = self.rng = np.random.default_rng(seed)
        need = [-(-n // page) for n in lengths]
        n_pages = sum(need) + spare
        order = [int(v) for v in rng.permutation(n_pages)]
        table = np.full((len(lengths), max(max(need), 1) + 1), -1, dtype=np.int32)
        refs = np.zeros(n_pages, dtype=np.int32)
        for u, n in enumerate(need):
            for j in range(n):
                src = next((a for a, b, k in shared if b == u and j < k), None)  # (a, b, k): b holds a's first k pages
                table[u, j] = table[src, j] if src is not None else order.pop()
                refs[table[u, j]] += 1
        self.tables = ora.Pages(table, np.array(lengths, dtype=np.int32), refs, page)
        self.pool = rng.integers(0, 256, (n_pages, layers, heads, page * hd * 9 // 8)).astype(np.uint8)
        self.mass = rng.random((layers, len(lengths), heads, table.shape[1] * page)).astype(np.float32)
        self.shape = (layers, heads)

    def keep(self, users, first, counts, lists=None, per_head=True, mass=True, want=None):
        """One call against the oracle's; lists [layer][i][head][j]."""
        layers, heads = self.shape
        most = max(1, *counts)
        if lists is None:
            lists = np.full((layers if per_head else 1, len(users), heads if per_head else 1, most), -1, dtype=np.int32)
            for idx in np.ndindex(lists.shape[:3]):
                i = idx[1]
                n = int(self.tables.lengths[users[i]])
                lists[idx][:counts[i]] = np.sort(self.rng.choice(np.arange(first[i], n), counts[i], replace=False)) if counts[i] else []
        rows = torch.from_numpy(lists).cuda().expand(layers, len(users), heads, lists.shape[3])
        kv4, t = self.kv4, self.tables
        dev = [torch.from_numpy(x.copy()).cuda() for x in (self.pool, t.table, t.lengths, t.refs, self.mass)]
        p, m = kv4.pool(dev[0], self.page, layers, heads, self.hd), kv4.page_map(*dev[1:4])
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        kv4.kfl_kv4_keep(p, m, i32(users), rows, i32(counts), kv4.pages_workspace(p), first=i32(first),
                         mass=dev[4] if mass else None, status=status)
        full = np.broadcast_to(lists, rows.shape)
        lengths, source = t.lengths.copy(), self.pool.copy()
        old = t.keep(users, first, counts)
        for i, (u, row) in enumerate(zip(users, old)):
            if row is None:
                continue
            f, c = first[i], counts[i]
            for l in range(layers):
                for h in range(heads):
                    part = source.copy() if len(source) < 40 else source
                    ora.keep_bytes(part, row, t.table[u], l, h, full[l, i, h, :c], f, self.page, self.hd)
                    touched = [j for j in range(f // self.page, -(-(f + c) // self.page))]
                    for j in touched:
                        self.pool[t.table[u, j], l, h] = part[t.table[u, j], l, h]
                    if mass:
                        moved = self.mass[l, u, h, full[l, i, h, :c]].copy()
                        self.mass[l, u, h, f:f + c] = moved
                        self.mass[l, u, h, f + c:lengths[u]] = 0
        for name, got, ref in (("table", dev[1], t.table), ("lengths", dev[2], t.lengths), ("refs", dev[3], t.refs),
                               ("mass", dev[4], self.mass), ("pool", dev[0], self.pool)):
            assert np.array_equal(got.cpu().numpy(), ref), name
        assert status.item() == (want or 0)


@pytest.mark.parametrize("hd,page", [(128, 64), (64, 16), (128, 32), (64, 128)])
@pytest.mark.parametrize("lengths,first,counts", [([70, 33], [54, 17], [5, 16]), ([1, 130], [0, 0], [0, 64]), ([300, 64, 65], [0, 0, 0], [150, 1, 64]),
                                                  ([128, 128], [64, 0], [0, 128]), ([200], [100], [1])])
def test_keep(hd, page, lengths, first, counts):
    c = Cache(lengths, page, hd, 2, 2, sum(lengths))
    c.keep(list(range(len(lengths))), first, counts)


@pytest.mark.parametrize("page", [16, 64])
def test_keep_with_shared_pages(page):
    """Users that went on from one another: pages that both hold are left alone, and rows before the first moved one come along."""
    lengths = [200, 150, 190, 33]
    c = Cache(lengths, page, 128, 2, 2, page, shared=[(0, 1, 128 // page), (0, 2, 64 // page)])
    c.keep([0, 2], [70, 10], [100, 60])
    c.keep([1, 3, 0, 2], [0, 3, 150, 0], [100, 20, 5, 5], mass=False)
    c.keep([1, 0], [7, 155], [40, 0])


def test_keep_broadcast_lists_and_long_ones():
    c = Cache([3000, 2500], 64, 64, 3, 1, 4)
    c.keep([1, 0], [2400, 0], [17, 2000], per_head=False)
    c.keep([0, 1], [0, 0], [900, 2417], per_head=False)


def test_keep_the_same_row_twice():
    """Entries at or behind their own place may repeat."""
    c = Cache([40], 16, 64, 1, 1, 4)
    c.keep([0], [8], [6], lists=np.array([9, 12, 12, 39, 39, 39], dtype=np.int32).reshape(1, 1, 1, 6))


def test_keep_reports_entries_out_of_place():
    """An entry before its own slot, or behind the last row: its slot stays what it was."""
    c = Cache([40], 16, 64, 2, 1, 4)
    table = c.tables.table.copy()
    pool, mass = c.pool.copy(), c.mass.copy()
    bad = np.array([9, 3, 40, 39, -1], dtype=np.int32).reshape(1, 1, 1, 5)
    kv4 = c.kv4
    dev = [torch.from_numpy(x.copy()).cuda() for x in (pool, table, c.tables.lengths, c.tables.refs, mass)]
    p, m = kv4.pool(dev[0], 16, 2, 1, 64), kv4.page_map(*dev[1:4])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kv4.kfl_kv4_keep(p, m, i32([0]), torch.from_numpy(bad).cuda().expand(2, 1, 1, 5), i32([5]), kv4.pages_workspace(p),
                     first=i32([8]), mass=dev[4], status=status)
    assert status.item() == kv4.KFL_BAD_POSITION
    as_if = np.array([9, 9, 10, 39, 12], dtype=np.int32).reshape(1, 1, 1, 5)
    c.keep([0], [8], [5], lists=as_if)
    assert np.array_equal(dev[0].cpu().numpy(), c.pool) and np.array_equal(dev[4].cpu().numpy(), c.mass)


def test_keep_leaves_bad_users_as_they_were():
    c = Cache([100, 90, 80, 70], 16, 64, 1, 2, 4)
    kv4, t = c.kv4, c.tables
    dev = [torch.from_numpy(x.copy()).cuda() for x in (c.pool, t.table, t.lengths, t.refs, c.mass)]
    p, m = kv4.pool(dev[0], 16, 1, 2, 64), kv4.page_map(*dev[1:4])
    rows = torch.arange(20, dtype=torch.int32, device="cuda").expand(1, 4, 2, 20)
    for users, first, counts, bit in (([4, -1, 9, 7], [0] * 4, [5] * 4, kv4.KFL_BAD_USER),
                                      ([0, 1, 2, 3], [-1, 90, 75, 0], [5, 1, 6, -1], kv4.KFL_BAD_POSITION),
                                      ([0, 1, 2, 3], [0] * 4, [21] * 4, kv4.KFL_BAD_POSITION)):
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        kv4.kfl_kv4_keep(p, m, i32(users), rows, i32(counts), kv4.pages_workspace(p), first=i32(first), mass=dev[4], status=status)
        assert status.item() == bit
        for d, x in zip(dev, (c.pool, t.table, t.lengths, t.refs, c.mass)):
            assert np.array_equal(d.cpu().numpy(), x)
    # a page out of range, and a user named twice: the others are cut all the same
    dev[1][2, 4] = 10 ** 6
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kv4.kfl_kv4_keep(p, m, i32([2, 0, 0, 3]), rows, i32([5, 5, 9, 4]), kv4.pages_workspace(p), status=status)
    assert status.item() == kv4.KFL_BAD_USER | kv4.KFL_BAD_PAGE
    assert dev[2].tolist() == [5, 90, 80, 4]


def test_keep_without_room_leaves_users_as_they_were():
    """Shared pages that would need new ones, of which the pool has too few: the first user gets them, the second stays."""
    c = Cache([64, 64, 64], 16, 64, 1, 1, 4, shared=[(0, 1, 4), (0, 2, 4)], spare=-8 + 3)
    assert (c.tables.refs == 0).sum() == 3
    c.keep([1, 2], [0, 0], [40, 20], want=c.kv4.KFL_NO_PAGES)


def test_keep_on_a_side_stream_and_in_a_graph():
    """Captured with the reservation that follows it, and replayed: lengths come round, pages are given back and taken again."""
    c = Cache([200, 90], 16, 128, 2, 2, 4)
    kv4, t = c.kv4, c.tables
    dev = [torch.from_numpy(x.copy()).cuda() for x in (c.pool, t.table, t.lengths, t.refs, c.mass)]
    p, m = kv4.pool(dev[0], 16, 2, 2, 128), kv4.page_map(*dev[1:4])
    rows = torch.arange(30, dtype=torch.int32, device="cuda").mul(2).add(10).expand(2, 2, 2, 30)
    users, first, counts, new, ws = i32([0, 1]), i32([10, 10]), i32([30, 20]), i32([160, 60]), kv4.pages_workspace(p)

    def both():
        stream = torch.cuda.current_stream().cuda_stream
        kv4.kfl_kv4_keep(p, m, users, rows, counts, ws, first=first, mass=dev[4], cuda_stream=stream)
        kv4.kfl_kv4_reserve(p, m, users, new, ws, cuda_stream=stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    once = [d.clone() for d in dev]
    for d, x in zip(dev, (c.pool, t.table, t.lengths, t.refs, c.mass)):
        d.copy_(torch.from_numpy(x))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(dev, once))
    graph.replay()
    torch.cuda.synchronize()
    assert dev[2].tolist() == [200, 90] and int(dev[3].sum()) == int((dev[1] >= 0).sum())


def test_weights_of_long_caches_and_many_prompts():
    """Key tiles whose rows several thread blocks share, and lists of many sequences."""
    c = Case([5000, 40], 1, 128, 64, seed=3)
    check_weights(c, queries(2, 8, 128))
    c = Case([700, 300], 1, 128, 64, seed=3)
    check_weights(c, queries(700, 4, 128), tokens=[600, 100])
    lengths = [40 + (i * 13) % 70 for i in range(60)]
    c = Case(lengths, 1, 64, 16, seed=3)
    check_weights(c, queries(60 * 35, 2, 64), tokens=[35] * 60)


@pytest.mark.parametrize("group", [3, 17, 100, 128])
def test_weights_of_unusual_groups(group):
    """Groups that do not divide a unit's rows, up to the largest; one token and several."""
    c = Case([70, 33], 1, 64, 16, seed=3)
    check_weights(c, queries(2, group, 64))
    check_weights(c, queries(9, group, 64), tokens=[7, 2])


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("tokens", [[3], [70]])
def test_weights_of_keys_without_spread_and_far_from_zero(dtype, tokens):
    """Groups of scale 0 (any code), of a centre thousands of steps from zero, and of next to no scale."""
    c = Case([170], 1, 128, 32, seed=3)
    for slot in range(0, 150, 3):
        p = c.params(0, slot, 0, 0, 0)
        p[slot % 2] = [(0.0, 0.75), (2.0 ** -24, -0.5), (0.01, 50.0), (0.0, 0.0), (3e-5, 2.0)][slot // 3 % 5]
    check_weights(c, queries(tokens[0], 4, 128, dtype, std=0.25), tokens=tokens)


def test_rows_of_other_sequences_do_not_reach_a_tail():
    """A unit's rows behind a sequence's last token are the next sequence's, NaN and infinities among them."""
    c = Case([100, 90], 1, 128, 64, seed=5)
    q = queries(40 + 30, 4, 128)
    q[40:, :, 5] = float("nan")
    q[40:, 1, 7] = float("inf")
    lse = lse_of(c, torch.nan_to_num(q, 0.0, 0.0), [40, 30], [0, 1], 0, 0, 128 ** -0.5)
    both = check_weights_raw(c, q, [40, 30], lse)
    alone = check_weights_raw(c, q[:40].contiguous(), [40], lse[:40].copy())
    assert np.isfinite(both[0, 0]).all() and (both[0, 0] == alone[0, 0]).all()


def test_keep_many_users():
    rng = np.random.default_rng(1)
    lengths = [int(v) for v in rng.integers(1, 60, 300)]
    c = Cache(lengths, 16, 64, 1, 1, 4, shared=[(0, u, 1) for u in range(1, 40)], spare=80)
    order = [int(u) for u in rng.permutation(300)][:260]
    first = [int(rng.integers(0, lengths[u] + 1)) for u in order]
    c.keep(order, first, [int(rng.integers(0, lengths[u] - f + 1)) for u, f in zip(order, first)])


def test_select_of_many_users():
    check_select([1 + (i * 29) % 300 for i in range(1024)], 90, 2, 5, page=16)


def test_offsets_behind_4_gib():
    """Pages, and masses, behind 32-bit byte offsets: weights of both kernels, and rows kept."""
    from paper_2609_34045_gb300 import kv4
    page, hd, heads, layers = 128, 128, 8, 40
    n_pages = (5 << 30) // (page * hd * 9 // 8 * heads * layers)
    pool_t = torch.zeros(n_pages, layers, heads, page * hd * 9 // 8, dtype=torch.uint8, device="cuda")
    table = torch.tensor([[-1, -1], [n_pages - 1, n_pages - 2]], dtype=torch.int32, device="cuda")
    lengths, refs = i32([0, 200]), torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    refs[-2:] = 1
    p, m = kv4.pool(pool_t, page, layers, heads, hd), kv4.page_map(table, lengths, refs)
    g = torch.Generator().manual_seed(3)
    k = torch.randn(200, heads, hd, generator=g).to(BF16).cuda()
    pos, user = torch.arange(200, dtype=torch.int32, device="cuda"), torch.ones(200, dtype=torch.int32, device="cuda")
    kv4.kfl_kv4_append(p, m, layers - 1, k, k, user, pos)
    mass = torch.zeros(layers, 2, heads, 14_000_000, device="cuda")[..., :256]  # the last layer's are 36 GB on
    kd = ora.values(*ora.quantise(k.float().cpu().numpy()))
    want = np.zeros((heads, 200))
    for t in (1, 40):
        q = queries(t, 8 * heads, hd)
        lse = torch.full((t, 8 * heads), 5.0, device="cuda")
        kv4.kfl_kv4_weights(p, m, layers - 1, q.cuda(), lse, mass, kv4.attend_workspace(p, 8 * heads, 1, t, t), users=i32([1]),
                            q_start=i32([0, t]), max_q=t)
        for h in range(heads):
            for j in range(8 * h, 8 * h + 8):
                want[h] += ora.weights(q[:, j].double().numpy(), kd[:, h], np.full(t, 5.0), ora.causal_keys(t, 200), hd ** -0.5).sum(0)
    got = mass[layers - 1, 1, :, :200].double().cpu().numpy()
    assert (np.abs(got - want) <= 2.0 ** -14 * want).all()
    rows = torch.arange(100, 200, dtype=torch.int32, device="cuda").expand(layers, 1, heads, 100)
    kv4.kfl_kv4_keep(p, m, i32([1]), rows, i32([100]), kv4.pages_workspace(p), mass=mass)
    k2, v2 = torch.empty_like(k[:100]), torch.empty_like(k[:100])
    kv4.kfl_kv4_read(p, m, layers - 1, user[:100], pos[:100], k2, v2)
    assert torch.equal(k2.cpu(), torch.from_numpy(kd[100:].astype(np.float32)).to(BF16)) and torch.equal(v2, k2)
    assert torch.equal(mass[layers - 1, 1, :, :100].double().cpu(), torch.from_numpy(got[:, 100:]))
    assert (mass[layers - 1, 1, :, 100:200] == 0).all() and lengths.tolist() == [0, 100] and table[1].tolist() == [n_pages - 1, -1]
