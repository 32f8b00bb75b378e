"""The many-row kernel of the 4-bit cache's attention in its steady state, against the 64-bit oracle: thread blocks that work
on several tiles of a row block and on several row blocks, so that references are kept and moved, buffers and flags are
used again, and row blocks are cut between thread blocks in the middle.

A list of n tiles of 128 keys is cut in pieces of ceil(n / SMs); ``Case.tiles`` counts them as the kernel's list does, and
each test says how many tiles a piece has at least.  Tolerances as in test_gpu_kv4_attend, wider by the scores' error where a
test makes scores that are larger than those it was derived for.
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


def pieces(c, tokens, group, window=0, users=None):
    """Tiles of a thread block's piece."""
    most = max(tokens) * group
    rows_per_block, tiles = 256 if most > 128 else 128, 0
    assert most > 64  # (else the few-row kernel may take the call)
    for u, t in zip(users or range(len(tokens)), tokens):
        n = int(c.lengths[u])
        for b in range(0, t * group, rows_per_block):
            last = (min(t * group, b + rows_per_block) - 1) // group
            begin = max(0, n - t + b // group + 1 - window) if window else 0
            tiles += max(1, -(-max(n - t + last + 1, 0) // 128) - begin // 128)
    n_sm = torch.cuda.get_device_properties(0).multi_processor_count
    return -(-tiles * c.pool.shape[2] // n_sm)


def write_row(c, user, slot, head, which, x):
    """One row's codes and parameters, quantised from x [hd]."""
    codes, par = ora.quantise(x[None].astype(np.float32))
    n = c.page * c.hd // 2
    b, s = c.pool[c.table[user, slot // c.page], 0, head], slot % c.page
    b[which * n + s * c.hd // 2:which * n + (s + 1) * c.hd // 2] = codes[0, 0::2] | codes[0, 1::2] << 4
    c.params(user, slot, 0, head, which)[:] = par[0]


@pytest.mark.parametrize("hd,kv_heads,group,page,dtype", [(128, 8, 2, 64, BF16), (64, 8, 3, 16, FP16), (128, 4, 5, 128, FP16),
                                                          (64, 8, 2, 32, BF16)])
@pytest.mark.parametrize("window", [0, 1000])
def test_pieces_of_several_tiles(hd, kv_heads, group, page, dtype, window):
    """Row blocks of 256 rows, their ends of fewer than 128, and sequences of one block, in pieces that cut them anywhere."""
    tokens = [150, 1, 300, 20, 77]
    c = Case([3000, 2000, 4100, 130, 1500], kv_heads, hd, page, seed=hd + group)
    assert pieces(c, tokens, group, window) >= (4 if window == 0 else 2)
    c.check(queries(sum(tokens), kv_heads * group, hd, dtype), tokens=tokens, window=window)


@pytest.mark.parametrize("window", [1, 100, 129])
@pytest.mark.parametrize("hd,page", [(128, 64), (64, 128)])
def test_short_windows(hd, page, window):
    """A row block's tiles begin inside the context, and its first and last tiles are seen in part."""
    tokens = [700, 33, 513]
    c = Case([2500, 33, 600], 8, hd, page, seed=window)
    assert pieces(c, tokens, 2, window) >= 2
    c.check(queries(sum(tokens), 16, hd), tokens=tokens, window=window)


def test_blocks_of_128_rows():
    """At most 128 query rows per KV head in every sequence: one half of the softmax warps has nothing to do."""
    tokens = [60, 64, 7, 33] * 4
    c = Case([3000, 1200, 2050, 64] * 4, 8, 128, 64, seed=4)
    assert pieces(c, tokens, 2) >= 10
    c.check(queries(sum(tokens), 16, 128), tokens=tokens)


@pytest.mark.parametrize("which", [0, 1])
@pytest.mark.parametrize("hd", [64, 128])
def test_nan_in_middle_tiles(which, hd):
    """Rows that read as NaN in the middle of a piece's tiles, some of them behind some tokens: a key's reaches every token
    that sees it, a value's its own group."""
    tokens = [100, 90]
    c = Case([3000, 2800], 8, hd, 64, seed=hd + which)
    assert pieces(c, tokens, 2) >= 3
    group = hd // 64 - 1
    for head, slot in ((1, 1000), (2, 2999), (3, 2930), (4, 0), (5, 2816)):
        c.params(0, slot, 0, head, which)[group] = np.nan
    c.params(1, 700, 0, 7, which)[0, 0] = np.nan
    c.params(1, 2750, 0, 6, which)[0, 1] = np.inf  # (an infinite centre reads as NaN or as an infinity: not compared)
    q = queries(190, 16, hd)
    got, lse = c.run(q, tokens=tokens)
    ref, size, ref_lse = c.expected(q, tokens=tokens)
    sees = np.zeros((190, 16), dtype=bool)
    sees[100:, 12:14] = (2800 - 90 + np.arange(90) >= 2750)[:, None]
    g, r = got.clone(), ref.copy()
    assert not torch.isfinite(g.float()).all(-1).cpu().numpy()[sees].any()
    g[torch.from_numpy(sees)], r[sees], size[sees] = 0.0, 0.0, 0.0
    lse[torch.from_numpy(sees)], ref_lse[sees] = 0.0, 0.0
    assert_near(g, lse, r, size, ref_lse)
    assert np.isnan(ref).any() and not np.isnan(ref).all()


@pytest.mark.parametrize("hd,dtype", [(128, BF16), (64, FP16)])
@pytest.mark.parametrize("order", [1, -1])
def test_scores_that_grow_along_the_context(hd, dtype, order):
    """Keys whose scores grow by some hundred powers of two from the first to the last (or fall): a row's reference has to
    move again and again, the sums and outputs with it.  Scores are up to 80: their error is the rounding of the decoded key to
    fp16, 2^-11 of each product q k at most, independent over the channels; six deviations of that (uniform: 1 / sqrt 3) on the
    weights, twice, since weight and sum have it."""
    tokens, heads = [160, 100], 8
    lengths = [2600, 2400]
    c = Case(lengths, heads, hd, 64, seed=7)
    assert pieces(c, tokens, 2) >= 4
    rng = np.random.default_rng(3)
    sign = rng.choice([-1.0, 1.0], hd)
    for u, n in enumerate(lengths):
        for head in (0, 3):  # (the other heads as they are)
            for t in range(n):
                grow = (t if order > 0 else n - t) / n
                write_row(c, u, t, head, 0, sign * (4.0 * grow) + 0.3 * rng.standard_normal(hd))
    q = queries(sum(tokens), 2 * heads, hd, dtype)
    for head in (0, 3):
        base = torch.from_numpy(sign * 20.0 / hd ** 0.5).to(dtype)
        q[:, 2 * head:2 * head + 2] = base + 0.25 * q[:, 2 * head:2 * head + 2]
    ref, size, ref_lse = c.expected(q, tokens=tokens)
    largest = np.nanmax(ref_lse)
    assert largest > 60
    # sqrt(sum (q_c k_c scale)^2) of the largest keys
    x = np.abs(q.double().numpy()).max(1)
    spread = 5.5 * np.sqrt((x ** 2).sum(-1)) * hd ** -0.5
    sigma = 2.0 ** -11 / 3 ** 0.5 * spread.max()
    got, lse = c.run(q, tokens=tokens)
    g, l = got.double().cpu().numpy(), lse.double().cpu().numpy()
    u = 2.0 ** -9 if dtype == BF16 else 2.0 ** -11
    assert (np.abs(g - ref) <= u * np.abs(ref) + (2.0 ** -8 + 12 * sigma) * size).all()
    assert (np.abs(l - ref_lse) <= 2.0 ** -8 + 6 * sigma + 2.0 ** -20 * np.abs(ref_lse)).all()


def test_more_sequences_than_one_launch_takes():
    """600 sequences of one token to a hundred, in two launches, and users in another order than the sequences."""
    rng = np.random.default_rng(2)
    tokens = [int(t) for t in rng.integers(1, 4, 600)]
    for i in (0, 100, 511, 512, 599):
        tokens[i] = 100
    lengths = [int(n) for n in rng.integers(100, 400, 600)]
    c = Case(lengths, 2, 64, 32, seed=8)
    users = [int(u) for u in rng.permutation(600)]
    assert pieces(c, tokens, 1, users=users) >= 3
    c.check(queries(sum(tokens), 2, 64), tokens=tokens, users=users)


def test_results_do_not_hang_on_the_order_of_arrival():
    """Row blocks cut in the middle of their tiles: the same bits every time, on a workspace that other calls use as well."""
    tokens = [150, 300, 20]
    c = Case([3000, 4100, 130], 8, 128, 64, seed=1)
    assert pieces(c, tokens, 2) >= 4
    pool = c.kv4.pool(torch.from_numpy(c.pool).cuda(), 64, 1, 8, 128)
    ws = c.kv4.attend_workspace(pool, 16, 3, sum(tokens), 300)
    q = queries(sum(tokens), 16, 128)
    first, lse = c.run(q, tokens=tokens, workspace=ws)
    for _ in range(4):
        c.run(queries(3, 16, 128, seed=5), workspace=ws)
        again, lse2 = c.run(q, tokens=tokens, workspace=ws)
        assert torch.equal(first, again) and torch.equal(lse, lse2)
