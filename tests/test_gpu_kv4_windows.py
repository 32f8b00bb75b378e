"""Windows at least as long as any context: the same as none, to the bit, for tokens with and without rows."""
import pytest
import torch

from gpu_helpers import ensure_built
from test_gpu_kv4_attend import Case, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()
    torch.cuda.init()


@pytest.mark.parametrize("group,tokens,lengths", [(2, [10, 3, 4], [5, 40, 1]), (8, [300, 40, 9], [200, 500, 5])])
@pytest.mark.parametrize("hd,page", [(64, 16), (128, 64)])
def test_a_window_longer_than_every_context(group, tokens, lengths, hd, page):
    """Some sequences have more tokens than rows: length - tokens - window passes the least 32-bit number where the window is
    the largest."""
    c = Case(lengths, 2, hd, page, seed=hd)
    q = queries(sum(tokens), 2 * group, hd)
    want, want_lse = c.check(q, tokens=tokens)
    capacity = c.table.shape[1] * page
    for window in (capacity - 1, capacity, capacity + 1, 1 << 26, 2 ** 31 - 200, 2 ** 31 - 1):
        got, lse = c.check(q, tokens=tokens, window=window)
        assert torch.equal(got, want) and torch.equal(lse, want_lse)
