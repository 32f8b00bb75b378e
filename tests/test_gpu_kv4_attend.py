"""Attention over the 4-bit paged cache against the 64-bit oracle.

Tolerances.  An output's own rounding is at most 2^-8 (bf16; half of it is allowed for, the rest falls to the slack of the next
term) or 2^-11 (fp16) of it.  Beside it every term p v is off by the
rounding of its weight to fp16 (2^-12 at most, as with v in prompts) and by the error of its score: in the few-row kernel
fp32 sums of exact codes, below 1e-4; in prompts the rounding of k to fp16, 2^-12 of each of head_dim random terms, below
2^-9 at six deviations for the scores of these cases (|scale q k| of a few).  Together: at most 2^-8 of the weighted mean
of |v|.  lse is off by its scores' error: 2^-8 absolute, and fp32's rounding.
"""
import numpy as np
import pytest
import torch

import oracle.kv4 as ora
from gpu_helpers import ensure_built

pytestmark = pytest.mark.gpu
BF16, FP16 = torch.bfloat16, torch.float16


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()
    torch.cuda.init()


class Case:
    """Users' rows in scattered pages, every slot that holds none of them NaN."""

    def __init__(self, lengths, kv_heads, hd, page, layers=1, seed=0, spare=2, value_std=1.0):
        from paper_2609_34045_gb300 import kv4
        self.kv4, self.page, self.hd, self.layers = kv4, page, hd, layers
        self.rng = rng = np.random.default_rng(seed)
        self.lengths = np.array(lengths, dtype=np.int32)
        need = [-(-n // page) for n in lengths]
        n_pages = sum(need) + spare
        order = rng.permutation(n_pages).astype(np.int32)
        self.table = np.full((len(lengths), max(max(need), 1) + 1), -1, dtype=np.int32)
        at = 0
        for u, n in enumerate(need):
            self.table[u, :n] = order[at:at + n]
            at += n
        block = page * hd * 9 // 8
        self.pool = np.full((n_pages, layers, kv_heads, block), 255, dtype=np.uint8)
        n, m = page * hd // 2, page * hd // 16
        for u, count in enumerate(lengths):
            for j in range(need[u]):
                rows = min(page, count - j * page)
                for i, std in ((0, 1.0), (1, value_std)):
                    x = rng.standard_normal((layers, kv_heads, rows, hd)) * std + (0.5 * std if i else 0.0)
                    codes, par = ora.quantise(x.astype(np.float32))
                    b = self.pool[self.table[u, j]]
                    b[..., i * n:i * n + rows * hd // 2] = (codes[..., 0::2] | codes[..., 1::2] << 4).reshape(layers, kv_heads, -1)
                    b[..., 2 * n + i * m:2 * n + i * m + rows * hd // 16] = \
                        par.reshape(layers, kv_heads, -1).view(np.uint8)
        self.refs = np.zeros(n_pages, dtype=np.int32)
        self.refs[order[:at]] = 1

    def params(self, user, slot, layer, head, which):
        """A writable view of the (scale, centre) pairs of one row."""
        b = self.pool[self.table[user, slot // self.page], layer, head]
        m = self.page * self.hd // 16
        p = b[self.page * self.hd + which * m:self.page * self.hd + (which + 1) * m].view(np.float16)
        return p.reshape(self.page, self.hd // 64, 2)[slot % self.page]

    def run(self, q, tokens=None, users=None, layer=0, window=0, scale=None, lse=True, out=None, status=None, max_q=None,
            workspace=None, stream=None):
        kv4 = self.kv4
        dev = {n: torch.from_numpy(getattr(self, n)).cuda() for n in ("pool", "table", "lengths", "refs")}
        pool = kv4.pool(dev["pool"], self.page, self.layers, self.pool.shape[2], self.hd)
        m = kv4.page_map(dev["table"], dev["lengths"], dev["refs"])
        q = q.cuda() if not q.is_cuda else q
        out = torch.full_like(q, 7.0) if out is None else out
        lse = torch.full(q.shape[:2], 7.0, device="cuda") if lse else None
        start = None if tokens is None else torch.tensor(np.concatenate([[0], np.cumsum(tokens)]), dtype=torch.int32, device="cuda")
        max_q = max(tokens) if tokens is not None and max_q is None else (max_q or 1)
        max_q = max(1, max_q)
        users = None if users is None else torch.tensor(users, dtype=torch.int32, device="cuda")
        n_seqs = len(tokens) if tokens is not None else q.shape[0]
        ws = workspace if workspace is not None else kv4.attend_workspace(pool, q.shape[1], n_seqs, q.shape[0], max_q)
        kv4.kfl_kv4_attend(pool, m, layer, q, out, ws, users=users, q_start=start, max_q=max_q, window=window, scale=scale,
                           lse=lse, status=status, cuda_stream=stream)
        torch.cuda.synchronize()
        return out, lse

    def expected(self, q, tokens=None, users=None, layer=0, window=0, scale=None):
        heads, group = q.shape[1], q.shape[1] // self.pool.shape[2]
        tokens = [1] * q.shape[0] if tokens is None else tokens
        users = range(len(tokens)) if users is None else users
        x = q.double().cpu().numpy()
        out, size, lse = np.zeros(x.shape), np.zeros(x.shape), np.zeros(x.shape[:2])
        at = 0
        for u, t in zip(users, tokens):
            n = int(self.lengths[u])
            for h in range(self.pool.shape[2]):
                k, v = ora.rows(self.pool, self.table[u], layer, h, n, self.page, self.hd)
                for j in range(h * group, (h + 1) * group):
                    out[at:at + t, j], size[at:at + t, j], lse[at:at + t, j] = ora.attend(
                        x[at:at + t, j], k, v, np.arange(n - t, n), self.hd ** -0.5 if scale is None else scale, window)
            at += t
        assert heads == group * self.pool.shape[2]
        return out, size, lse

    def check(self, q, **kw):
        got, lse = self.run(q, **{k: v for k, v in kw.items()})
        ref, size, ref_lse = self.expected(q, **{k: v for k, v in kw.items() if k in ("tokens", "users", "layer", "window", "scale")})
        assert_near(got, lse, ref, size, ref_lse)
        return got, lse


def assert_near(got, lse, ref, size, ref_lse):
    u = 2.0 ** -9 if got.dtype == BF16 else 2.0 ** -11
    g = got.double().cpu().numpy()
    assert (np.isnan(g) == np.isnan(ref)).all()
    err = np.abs(g - ref) - (u * np.abs(ref) + 2.0 ** -8 * size + 2.0 ** -24)
    worst = np.unravel_index(np.nanargmax(err), err.shape) if err.size else None
    assert not err.size or not (err > 0).any(), (worst, g[worst], ref[worst], size[worst])
    if lse is not None:
        got_lse = lse.double().cpu().numpy()
        assert (np.isneginf(got_lse) == np.isneginf(ref_lse)).all()
        fine = np.isfinite(ref_lse)
        assert (np.isnan(got_lse) == np.isnan(ref_lse)).all()
        assert (np.abs(got_lse - ref_lse)[fine] <= 2.0 ** -8 + 2.0 ** -20 * np.abs(ref_lse[fine])).all()


def queries(n, heads, hd, dtype=BF16, seed=1, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(n, heads, hd, generator=g) * std).to(dtype)


LENGTHS = {"one": [1], "edges": [1, 15, 16, 17, 63, 64, 65], "ragged": [130, 1, 700, 333, 64], "long": [4099], "many": [5, 70] * 23}


@pytest.mark.parametrize("dtype", [BF16, FP16], ids=["bf16", "fp16"])
@pytest.mark.parametrize("hd,kv_heads,group,page", [(128, 2, 8, 64), (128, 4, 7, 16), (64, 2, 4, 32), (128, 1, 1, 128),
                                                    (64, 1, 12, 16), (128, 2, 16, 128), (64, 3, 5, 128)])
@pytest.mark.parametrize("lengths", list(LENGTHS), ids=list(LENGTHS))
def test_single_tokens(hd, kv_heads, group, page, lengths, dtype):
    c = Case(LENGTHS[lengths], kv_heads, hd, page, seed=hd + group)
    c.check(queries(len(LENGTHS[lengths]), kv_heads * group, hd, dtype))


@pytest.mark.parametrize("hd,kv_heads,group,page", [(128, 2, 8, 64), (64, 2, 3, 16), (128, 1, 5, 128)])
@pytest.mark.parametrize("window", [1, 17, 64, 100, 5000])
def test_windows(hd, kv_heads, group, page, window):
    c = Case([1, 64, 129, 700], kv_heads, hd, page, seed=window)
    c.check(queries(4, kv_heads * group, hd), window=window)
    c.check(queries(10, kv_heads * group, hd), tokens=[1, 3, 4, 2], window=window)


@pytest.mark.parametrize("tokens,lengths", [([2, 1, 2], [300, 5, 64]), ([1, 0, 2], [10, 20, 30]), ([2, 2], [1, 2]),
                                            ([2, 2], [0, 1]), ([5, 5, 5, 5], [300, 51, 177, 235]), ([40], [100]),
                                            ([1, 12, 7], [12, 12, 400]), ([129, 3], [129, 500]), ([300], [300]),
                                            ([64, 200], [700, 450]), ([17, 30], [5, 90])])
@pytest.mark.parametrize("hd,kv_heads,group,page,dtype", [(128, 2, 8, 64, BF16), (128, 2, 7, 16, FP16), (64, 2, 4, 32, BF16),
                                                          (64, 1, 1, 128, FP16), (128, 1, 5, 128, BF16)])
def test_several_tokens(tokens, lengths, hd, kv_heads, group, page, dtype):
    c = Case(lengths, kv_heads, hd, page, seed=sum(tokens))
    c.check(queries(sum(tokens), kv_heads * group, hd, dtype), tokens=tokens)


@pytest.mark.parametrize("tokens", [[1, 1, 1], [3, 1, 2], [30, 50, 2]])
def test_users_layers_and_strides(tokens):
    c = Case([90, 200, 33, 257], 2, 128, 32, layers=3, seed=4)
    q = queries(sum(tokens), 3 * 16, 128).cuda()[:, 16:32]  # a slice of a wider projection
    out = torch.full((16, sum(tokens), 128), 7.0, dtype=BF16, device="cuda").transpose(0, 1)  # heads outermost
    c.check(q, tokens=tokens, users=[3, 0, 3], layer=2, out=out)
    odd = torch.zeros(sum(tokens), 16, 131, dtype=BF16, device="cuda")[..., 3:]  # rows off 16 bytes
    odd.copy_(q)
    out = torch.zeros(sum(tokens), 16, 129, dtype=BF16, device="cuda")[..., :128]
    c.check(odd, tokens=tokens, users=[1, 1, 0], layer=1, out=out)


@pytest.mark.parametrize("group,tokens", [(8, None), (8, [2, 2]), (8, [6, 40])])
def test_nan_reaches_only_the_rows_that_see_it(group, tokens):
    """A value's NaN group reaches its own 64 channels, a key's NaN the whole row; neither a row that stands before it."""
    t = tokens or [1, 1]
    for which in (0, 1):
        c = Case([200, 70], 2, 128, 16, seed=9)
        for user in (0, 1):
            c.params(user, int(c.lengths[user]) - 1, 0, 1, which)[1] = np.nan  # only the last token sees it
        q = queries(sum(t), 2 * group, 128)
        got, _ = c.check(q, tokens=tokens, lse=False) if which else (c.run(q, tokens=tokens, lse=False)[0], None)
        bad = np.isnan(got.float().cpu().numpy())
        assert not bad[:, :group].any()
        last = np.cumsum(t) - 1
        rest = np.setdiff1d(np.arange(sum(t)), last)
        assert not bad[rest].any()
        assert bad[last][:, group:, 64:].all()
        assert bad[last][:, group:, :64].all() == (which == 0)


def test_infinite_and_nan_queries_stay_in_their_rows():
    c = Case([100, 100], 1, 128, 64, seed=2)
    q = queries(2, 8, 128)
    q[0, 3, 5], q[1, 2, 0] = float("inf"), float("nan")
    got, _ = c.run(q)
    bad = torch.isnan(got.float()).all(-1).cpu().numpy()
    expect = np.zeros((2, 8), dtype=bool)
    expect[0, 3] = expect[1, 2] = True
    assert (bad == expect).all()
    assert not torch.isnan(got.float()).any(-1).cpu().numpy()[~expect].any()


@pytest.mark.parametrize("std", [1e-3, 30.0, 3000.0])
@pytest.mark.parametrize("tokens", [None, [30, 40]])
def test_scales_of_queries_and_values(std, tokens):
    """Large queries (a nearly one-hot softmax) and values far from one: the scores are kept to a few by `scale`."""
    c = Case([150, 333], 2, 128, 64, seed=3, value_std=std)
    q = queries(2 if tokens is None else 70, 16, 128, std=std)
    c.check(q, tokens=tokens, scale=128 ** -0.5 / std)


@pytest.mark.parametrize("tokens", [None, [20, 33]])
@pytest.mark.parametrize("scale", [0.0, -0.05, 1.0])
def test_unusual_scales(scale, tokens):
    c = Case([150, 33], 2, 64, 16, seed=6)
    q = queries(2 if tokens is None else 53, 8, 64, std=0.25 if scale == 1.0 else 1.0)
    c.check(q, tokens=tokens, scale=scale)


def test_values_of_one_size_and_zero():
    """Groups without spread have scale 0: every code reads as the centre."""
    for value in (0.0, 2.5):
        c = Case([100], 1, 128, 64, seed=5)
        for slot in range(100):
            c.params(0, slot, 0, 0, 1)[:] = [0.0, value]
        got, _ = c.run(queries(1, 8, 128))
        assert (got.float() == value).all()


def test_empty_users_write_zeros():
    c = Case([0, 40], 2, 64, 16, seed=5)
    got, lse = c.check(queries(2, 8, 64))
    assert (got[0] == 0).all() and torch.isneginf(lse[0]).all()
    got, lse = c.check(queries(60, 8, 64), tokens=[30, 30])
    assert (got[:30] == 0).all() and torch.isneginf(lse[:30]).all()


@pytest.mark.parametrize("tokens", [None, [20, 33, 1]])
def test_bad_users_and_pages_are_reported(tokens):
    c = Case([100, 100, 100], 1, 64, 16, seed=8)
    n = 3 if tokens is None else sum(tokens)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = queries(n, 4, 64)
    c.run(q, tokens=tokens, users=[0, 7, -1], status=status)
    assert status.item() == c.kv4.KFL_BAD_USER
    status.zero_()
    good, _ = c.run(q, tokens=tokens, status=status)
    assert status.item() == 0
    c.table[1, 2] = 10 ** 6
    bad, _ = c.run(q, tokens=tokens, status=status)
    assert status.item() == c.kv4.KFL_BAD_PAGE
    at = 1 if tokens is None else 20
    assert torch.equal(good[:at], bad[:at]) and torch.equal(good[n - 1:], bad[n - 1:])
    assert torch.isfinite(bad.float()).all()


def test_more_sequences_than_one_launch_takes():
    lengths = [1 + (i * 37) % 90 for i in range(700)]
    c = Case(lengths, 1, 64, 32, seed=8)
    c.check(queries(700, 2, 64))


@pytest.mark.parametrize("tokens,max_q", [([1, 1, 1, 1], 2), ([40, 3, 64, 9], 64)])
def test_workspace_is_left_as_found_and_results_repeat(tokens, max_q):
    """The same call on the same workspace, alone and after other sizes, gives the same bits; results do not hang on the
    order in which blocks arrive."""
    c = Case([3000, 17, 2100, 64], 2, 128, 64, seed=8)
    kv4 = c.kv4
    pool = kv4.pool(torch.from_numpy(c.pool).cuda(), c.page, 1, 2, 128)
    ws = kv4.attend_workspace(pool, 16, 4, sum(tokens), max_q)
    q = queries(sum(tokens), 16, 128)
    first, lse = c.run(q, tokens=tokens, workspace=ws, max_q=max_q)
    for _ in range(5):
        c.run(queries(4, 16, 128, seed=5), workspace=ws)
        again, lse2 = c.run(q, tokens=tokens, workspace=ws, max_q=max_q)
        assert torch.equal(first, again) and torch.equal(lse, lse2)


def test_offsets_behind_4_gib():
    """Pages behind the 32-bit byte offsets of a pool."""
    from paper_2609_34045_gb300 import kv4
    page, hd, heads, layers = 128, 128, 8, 40
    n_pages = (5 << 30) // (page * hd * 9 // 8 * heads * layers)
    pool_t = torch.zeros(n_pages, layers, heads, page * hd * 9 // 8, dtype=torch.uint8, device="cuda")
    table = torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([200], dtype=torch.int32, device="cuda")
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    p, m = kv4.pool(pool_t, page, layers, heads, hd), kv4.page_map(table, lengths, refs)
    g = torch.Generator().manual_seed(3)
    k, v = (torch.randn(200, heads, hd, generator=g).to(BF16).cuda() for _ in range(2))
    pos = torch.arange(200, dtype=torch.int32, device="cuda")
    user = torch.zeros(200, dtype=torch.int32, device="cuda")
    kv4.kfl_kv4_append(p, m, layers - 1, k, v, user, pos)
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    kv4.kfl_kv4_read(p, m, layers - 1, user, pos, k2, v2)
    kd, vd = (ora.values(*ora.quantise(x.float().cpu().numpy())) for x in (k, v))
    assert torch.equal(k2.cpu(), torch.from_numpy(kd.astype(np.float32)).to(BF16))
    assert torch.equal(v2.cpu(), torch.from_numpy(vd.astype(np.float32)).to(BF16))
    for t in (1, 40):
        q = queries(t, 8 * heads, hd)
        out, start = torch.empty_like(q, device="cuda"), torch.tensor([0, t], dtype=torch.int32, device="cuda")
        kv4.kfl_kv4_attend(p, m, layers - 1, q.cuda(), out, kv4.attend_workspace(p, 8 * heads, 1, t, t), q_start=start, max_q=t)
        for h in (0, 8 * heads - 1):
            ref, size, _ = ora.attend(q[:, h].double().numpy(), kd[:, h // 8], vd[:, h // 8], np.arange(200 - t, 200), hd ** -0.5)
            err = np.abs(out[:, h].double().cpu().numpy() - ref)
            assert (err <= 2.0 ** -9 * np.abs(ref) + 2.0 ** -8 * size).all()


def test_one_workspace_serves_calls_of_all_smaller_sizes():
    """Calls of other shapes leave nothing where a call looks for its tickets."""
    c = Case([3000, 17, 2100, 64] + [90] * 60, 2, 128, 64, seed=8)
    kv4 = c.kv4
    pool = kv4.pool(torch.from_numpy(c.pool).cuda(), c.page, 1, 2, 128)
    ws = kv4.attend_workspace(pool, 16, 64, 400, 200)
    shapes = [dict(tokens=[1] * 64), dict(tokens=[6, 1, 4] + [1] * 61), dict(tokens=[2] * 64), dict(tokens=[200, 17, 50, 1] + [1] * 60), dict()]
    alone = []
    for kw in shapes:
        n = sum(kw.get("tokens", [1] * 64))
        alone.append(c.run(queries(n, 16, 128, seed=n), **kw)[0])
    for _ in range(2):
        for kw, want in zip(shapes + shapes[::-1], alone + alone[::-1]):
            n = sum(kw.get("tokens", [1] * 64))
            got, _ = c.run(queries(n, 16, 128, seed=n), workspace=ws, **kw)
            assert torch.equal(got, want)


@pytest.mark.parametrize("hd,kv_heads,group,page,dtype", [(128, 2, 8, 64, BF16), (128, 2, 7, 16, FP16), (64, 2, 12, 32, BF16), (64, 1, 1, 128, FP16)])
@pytest.mark.parametrize("window", [0, 40])
def test_drafts_in_blocks_of_rows(hd, kv_heads, group, page, dtype, window):
    """Token counts whose rows fill one to three blocks of sixteen, mixed, some of them more than there are cached rows."""
    most = 48 // group
    tokens = [1, most, (most + 1) // 2, 0, most, min(most, 3)]
    c = Case([5, 700, 64, 9, most - 1 if most > 1 else 1, 130], kv_heads, hd, page, seed=group)
    c.check(queries(sum(tokens), kv_heads * group, hd, dtype), tokens=tokens, window=window)


def test_long_contexts_keep_the_precision_of_short_ones():
    """65536 rows of nearly even weights: the small mean of many values of either sign.  The weights' rounding to fp16 (2^-12)
    is independent over the rows, as the values are: relative to the output 2^-12 as well, and an fp16 output's own 2^-11."""
    n, hd = 65536, 128
    c = Case([n], 1, hd, 128, seed=1)
    q = queries(1, 8, hd, FP16, std=0.2)
    got, _ = c.run(q)
    ref, _, _ = c.expected(q)
    err = np.linalg.norm(got.double().cpu().numpy() - ref) / np.linalg.norm(ref)
    assert err <= 2.0 ** -11 + 2.0 ** -12


@pytest.mark.parametrize("hd,page,lengths", [(128, 64, [70000]), (64, 128, [50000, 20]), (128, 128, [1] * 40 + [40000])])
def test_one_segment_over_many_blocks(hd, page, lengths):
    """A KV head's keys split over dozens of blocks, alone and among many short users."""
    c = Case(lengths, 1, hd, page, seed=8)
    c.check(queries(len(lengths), 4, hd, FP16))


@pytest.mark.parametrize("group,tokens", [(8, [8, 7, 1]), (1, [64, 49, 2]), (16, [4, 3, 4]), (5, [12, 11, 10])])
@pytest.mark.parametrize("hd,page,window", [(128, 64, 0), (64, 16, 70)])
def test_four_blocks_of_rows(group, tokens, hd, page, window):
    c = Case([1000, 333, 64], 2, hd, page, seed=9)
    c.check(queries(sum(tokens), 2 * group, hd, FP16), tokens=tokens, window=window)
