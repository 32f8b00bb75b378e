"""What the binding of the 4-bit cache refuses before a call reaches the library, and what it lets through."""
import pytest
import torch

from paper_2609_34045_gb300 import kv4
from test_kv4_cpu import lib  # noqa: F401


class Fake:
    """Stands for a tensor in device memory; only what the binding looks at."""
    is_cuda = True

    def __init__(self, numel, dtype=torch.uint8, contiguous=True, device=0):
        self.n, self.dtype, self.contiguous, self.device_index = numel, dtype, contiguous, device

    def numel(self):
        return self.n

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return self.contiguous

    def data_ptr(self):
        return 1 << 20

    def get_device(self):
        return self.device_index


def pool(n_pages):
    return kv4.pool(None, 64, 14, 4, 128, n_pages=n_pages)


@pytest.mark.parametrize("made_for,used_for", [(400, 1400), (10, 1035), (10, 11), (1, 5), (1000, 2048)])
def test_a_smaller_pools_workspace_is_refused(lib, made_for, used_for):  # noqa: F811
    """The kernels' regions in it start at places computed from the pool's pages: behind the end of a smaller one's."""
    size = kv4.kfl_kv4_pages_workspace_bytes(pool(made_for))
    assert size < kv4.kfl_kv4_pages_workspace_bytes(pool(used_for))
    with pytest.raises(ValueError, match="pages_workspace"):
        kv4._scratch(pool(used_for), Fake(size))


def test_a_pools_own_workspace_is_taken(lib):  # noqa: F811
    p = pool(1400)
    need = kv4.kfl_kv4_pages_workspace_bytes(p)
    assert need >= 4 * (4 + 3 * (1400 + 1024))  # a count, and three lists of the pages and of a call's users
    for ok in (Fake(need), Fake(need + 100), Fake(-(-need // 4), torch.int32)):
        assert kv4._scratch(p, ok) == 1 << 20
    for bad in (Fake(need - 1), Fake(need // 4 - 1, torch.int32), Fake(need, contiguous=False)):
        with pytest.raises(ValueError, match="pages_workspace"):
            kv4._scratch(p, bad)
    p.n_pages = 3000  # (a description that changes is looked at anew)
    with pytest.raises(ValueError, match="pages_workspace"):
        kv4._scratch(p, Fake(need))
