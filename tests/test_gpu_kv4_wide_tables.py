"""Tables of the most columns that there may be, whose rows could stand for 2^31 tokens."""
import pytest
import torch

from gpu_helpers import ensure_built
from test_gpu_kv4_pages import Both

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()
    torch.cuda.init()


@pytest.mark.parametrize("page,max_pages", [(128, 1 << 24), (64, 1 << 24), (128, (1 << 24) - 1)])
def test_forks_in_the_widest_tables(page, max_pages):
    b = Both(2, max_pages, 12, page, layers=1, kv=1)
    b.reserve([0, 1], [2 * page + 5, page])
    b.check()
    b.fork([0], [1])
    b.check()
    b.reserve([1], [page])
    b.fork([1, 0], [0, 1])
    b.check()
    b.free([0])
    b.check()
