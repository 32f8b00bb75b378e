"""Which users kfl_kv4_keep finds pages for when there are too few, against the oracle's tables."""
import pytest
import torch

from gpu_helpers import ensure_built

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    ensure_built()
    torch.cuda.init()


def test_a_pool_without_room_for_one_user_has_none_for_those_behind_it():
    """As in a reservation: of three free pages the first user wants five and the second one."""
    from test_gpu_kv4_evict import Cache
    c = Cache([80, 80, 80, 40], 16, 64, 1, 1, 4, shared=[(0, 1, 5), (0, 2, 5)], spare=3 - 10)
    assert (c.tables.refs == 0).sum() == 3
    before = c.tables.lengths.copy()
    c.keep([1, 2, 3], [0, 0, 5], [70, 10, 20], want=c.kv4.KFL_NO_PAGES)
    assert c.tables.lengths.tolist() == [*before[:3], 25]  # (the last one needs none)
