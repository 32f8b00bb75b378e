"""Pages of the 4-bit cache against the oracle's tables: whole numbers and copied bytes, so equal to the bit."""
import numpy as np
import pytest
import torch

import oracle.kv4 as ora
from gpu_helpers import ensure_built

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()
    torch.cuda.init()


def int32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


class Both:
    """The library's buffers and the oracle's tables, side by side."""

    def __init__(self, n_users, max_pages, n_pages, page=16, layers=2, kv=2, hd=64, seed=0):
        from paper_2609_34045_gb300 import kv4
        self.kv4, self.page = kv4, page
        self.table = torch.full((n_users, max_pages), -1, dtype=torch.int32, device="cuda")
        self.lengths = torch.zeros(n_users, dtype=torch.int32, device="cuda")
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
        self.bytes = torch.randint(0, 256, (n_pages, layers * kv * page * hd * 9 // 8), dtype=torch.uint8,
                                   generator=torch.Generator().manual_seed(seed)).cuda()
        self.pool = kv4.pool(self.bytes, page, layers, kv, hd)
        self.map = kv4.page_map(self.table, self.lengths, self.refs)
        self.ws = kv4.pages_workspace(self.pool)
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.ora = ora.Pages(self.table.cpu().numpy(), self.lengths.cpu().numpy(), self.refs.cpu().numpy(), page)
        self.want = self.bytes.cpu().numpy().copy()

    def check(self, status=0):
        assert np.array_equal(self.table.cpu().numpy(), self.ora.table)
        assert np.array_equal(self.lengths.cpu().numpy(), self.ora.lengths)
        assert np.array_equal(self.refs.cpu().numpy(), self.ora.refs)
        assert np.array_equal(self.bytes.cpu().numpy(), self.want)
        assert self.status.item() == status
        self.status.zero_()

    def reserve(self, users, n):
        self.kv4.kfl_kv4_reserve(self.pool, self.map, int32(users), int32(n), self.ws, status=self.status)
        self.ora.reserve(users, n)

    def free(self, users):
        self.kv4.kfl_kv4_free(self.pool, self.map, int32(users), status=self.status)
        self.ora.free(users)

    def fork(self, src, dst):
        self.kv4.kfl_kv4_fork(self.pool, self.map, int32(src), int32(dst), self.ws, status=self.status)
        for a, b in self.ora.fork(src, dst):
            self.want[b] = self.want[a]

    def compact(self, out=False):
        n_live = torch.zeros(1, dtype=torch.int32, device="cuda")
        table, refs = (torch.full_like(self.table, 7), torch.full_like(self.refs, 7)) if out else (self.table, self.refs)
        self.kv4.kfl_kv4_compact(self.pool, self.map, table, refs, n_live, self.ws, status=self.status)
        moves, n = self.ora.compact()
        for a, b in moves:
            self.want[b] = self.want[a]
        assert n_live.item() == n
        if out:
            self.table.copy_(table), self.refs.copy_(refs)


@pytest.mark.parametrize("n_users,max_pages,n_pages,page", [(1, 1, 1, 16), (5, 7, 20, 16), (40, 33, 700, 32), (300, 9, 2000, 128)])
@pytest.mark.parametrize("seed", range(3))
def test_random_sessions(n_users, max_pages, n_pages, page, seed):
    rng = np.random.default_rng(seed)
    b = Both(n_users, max_pages, n_pages, page, layers=1 if page == 128 else 2, seed=seed)
    for step in range(25):
        k = int(rng.integers(1, n_users + 1))
        users = [int(u) for u in rng.permutation(n_users)[:k]]
        kind = rng.choice(["reserve", "reserve", "fork", "free", "compact"])
        if kind == "reserve":
            room = [max_pages * page - int(b.ora.lengths[u]) for u in users]
            # some of the room, none, or all of it: the pool runs out now and then
            n = [int(rng.choice([0, 1, r, int(rng.integers(0, r + 1))])) if r else 0 for r in room]
            want = [int(v) + b_ for v, b_ in zip(n, b.ora.lengths[users])]
            b.reserve(users, n)
            short = any(int(b.ora.lengths[u]) != w for u, w in zip(users, want))
            b.check(b.kv4.KFL_NO_PAGES if short else 0)
        elif kind == "fork":
            src = [int(u) for u in rng.integers(0, n_users, k)]
            ends = sum(int(b.ora.lengths[a]) % page > 0 and a != d for a, d in zip(src, users))
            short = ends > int((b.ora.refs == 0).sum())
            b.fork(src, users)
            b.check(b.kv4.KFL_NO_PAGES if short else 0)
        elif kind == "free":
            b.free(users[:max(1, k // 3)])
            b.check()
        else:
            b.compact(out=bool(rng.integers(0, 2)))
            b.check()


def test_beams_change_places():
    b = Both(4, 6, 40)
    b.reserve([0, 1], [50, 33])
    b.fork([0, 0], [2, 3])
    b.check()
    b.fork([1, 0, 3, 2], [0, 1, 2, 3])  # every one source and destination
    b.check()
    b.fork([2, 2], [2, 0])  # one stays
    b.check()
    b.fork([0], [1])
    b.free([0, 1, 2, 3])
    b.check()
    assert (b.refs == 0).all()


def test_refusals_on_the_device():
    b = Both(3, 4, 8)
    b.reserve([0, 1], [30, 10])
    b.check()
    kv4 = b.kv4
    kv4.kfl_kv4_reserve(b.pool, b.map, int32([0, 7, 0, -1]), int32([1, 1, 1, 1]), b.ws, status=b.status)
    b.ora.reserve([0], [1])  # the first mention counts
    b.check(kv4.KFL_BAD_USER)
    kv4.kfl_kv4_reserve(b.pool, b.map, int32([1, 2]), int32([-1, 65]), b.ws, status=b.status)
    b.check(kv4.KFL_BAD_USER | kv4.KFL_NO_PAGES)  # a negative count; a row of four pages cannot hold 65
    kv4.kfl_kv4_fork(b.pool, b.map, int32([0, 0, 9]), int32([2, 2, 1]), b.ws, status=b.status)
    for a, d in b.ora.fork([0], [2]):
        b.want[d] = b.want[a]
    b.check(kv4.KFL_BAD_USER)
    kv4.kfl_kv4_free(b.pool, b.map, int32([1, 1, 3]), status=b.status)
    b.ora.free([1])
    b.check(kv4.KFL_BAD_USER)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    kv4.kfl_kv4_copy_pages(b.pool, int32([0, 8]), int32([-1, 2]), status=status)
    b.check()
    assert status.item() == kv4.KFL_BAD_PAGE


@pytest.mark.parametrize("n_pages", [16384, 16385, 70001])
def test_many_pages(n_pages):
    """Pools of more pages than one pass of the plan's scan, the free ones at the end."""
    b = Both(8, n_pages // 2, n_pages, layers=1, kv=1)
    used = n_pages - 40
    for u in range(8):
        b.reserve([u], [used // 8 * 16 + 3 * u])
    b.check()
    b.free([1, 4])
    b.reserve([1, 4, 2], [100, 1, 17])
    b.check()
    b.free([0])
    b.compact()
    b.check()
    b.compact(out=True)  # nothing left to move
    b.check()


@pytest.mark.parametrize("layers,kv,hd,page", [(1, 1, 64, 16), (3, 8, 128, 64), (1, 3, 64, 128)])
def test_copied_pages(layers, kv, hd, page):
    b = Both(1, 1, 50, page, layers, kv, hd)
    src, dst = [3, 3, 49, 0], [10, 11, 12, 48]
    b.kv4.kfl_kv4_copy_pages(b.pool, int32(src), int32(dst))
    b.want[dst] = b.want[src]
    b.check()
    b.kv4.kfl_kv4_copy_pages(b.pool, int32([]), int32([]))
    b.check()


def test_a_thousand_users_in_one_call():
    b = Both(1024, 3, 4000, layers=1, kv=1)
    rng = np.random.default_rng(5)
    b.reserve(list(range(1024)), [int(v) for v in rng.integers(0, 40, 1024)])
    b.check()
    b.fork([int(v) for v in rng.integers(0, 1024, 1024)], [int(v) for v in rng.permutation(1024)])
    b.check()
    b.free(list(range(0, 1024, 3)))
    b.check()


def test_session_of_the_operators_together():
    """The example's session on small sizes: prompts, steps, beams, leavers and a compaction, every layer's attention against
    the oracle on the rows that the cache then holds (tolerance: as in test_gpu_kv4_attend)."""
    from paper_2609_34045_gb300 import kv4
    from paper_2609_34045_gb300.kv4_session import Session
    layers, heads, kv, hd, page = 2, 8, 2, 64, 16
    s = Session(layers, heads, kv, hd, n_users=5, max_ctx=200, n_pages=60, page_tokens=page, max_tokens=64)
    g = torch.Generator().manual_seed(0)
    angle = 1e6 ** (-np.arange(0, hd, 2) / hd)

    def go(counts):
        step = s.begin(counts)
        pos = step["positions"].cpu().numpy()
        for layer in range(layers):
            q, k, v = (torch.randn(len(pos), h, hd, generator=g).to(torch.bfloat16).cuda() for h in (heads, kv, kv))
            out = s.attend(layer, step, q, k, v)
            turned = torch.from_numpy(ora.rotate(q.double().cpu().numpy(), pos[:, None] * angle, False)).to(torch.bfloat16)
            pool = s.pages.view(60, layers, kv, -1).cpu().numpy()
            table, lengths, at = s.table.cpu().numpy(), s.lengths.cpu().numpy(), 0
            for u, n in counts.items():
                for h in range(heads):
                    kk, vv = ora.rows(pool, table[u], layer, h // (heads // kv), int(lengths[u]), page, hd)
                    ref, size, _ = ora.attend(turned[at:at + n, h].double().numpy(), kk, vv, pos[at:at + n], hd ** -0.5)
                    err = np.abs(out[at:at + n, h].double().cpu().numpy() - ref)
                    # (q's own rounding to bf16 after the rotation may fall the other way: 2^-9 of its scores, below 2^-6)
                    assert (err <= 2.0 ** -9 * np.abs(ref) + 2.0 ** -6 * size).all()
                at += n

    go({0: 33, 1: 7, 2: 50})
    go({0: 1, 1: 1, 2: 1})
    s.fork([0, 2], [3, 4])
    go({0: 1, 3: 2, 4: 1})
    s.fork([4, 3], [3, 4])
    go({3: 1, 4: 5})
    s.free([0, 2])
    s.compact()
    go({1: 1, 3: 1, 4: 1})
    go({0: 64})
    assert s.status.item() == 0
    assert int((s.refs != 0).sum()) == len(set(s.table[s.table >= 0].tolist()))
