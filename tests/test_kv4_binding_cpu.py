"""What the binding of the 4-bit cache refuses before a call reaches the library, and what it lets through."""
import ctypes as C

import pytest
import torch

from paper_2609_34045_gb300 import kv4
from paper_2609_34045_gb300 import stage as K
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


class OnDevice:
    """A tensor that says it lies in a device's memory."""
    is_cuda = True

    def __init__(self, t, device=0):
        self.t, self.index = t, device

    def get_device(self):
        return self.index

    def __getattr__(self, name):
        return getattr(self.t, name)


def calls(place):
    """Every call with tensors, as (function, arguments by name) in the binding's own order; place(name, tensor) puts each
    where it shall be."""
    def i32(name, n):
        return place(name, torch.zeros(n, dtype=torch.int32))

    def rows(name, n, heads, dtype=torch.bfloat16):
        return place(name, torch.zeros(n, heads, 64, dtype=dtype))

    def pool(name="pages"):
        return kv4.pool(place(name, torch.zeros(5 * 2 * 16 * 72, dtype=torch.uint8)), 16, 1, 2, 64)

    def page_map():
        return kv4.page_map(place("table", torch.zeros(3, 4, dtype=torch.int32)), i32("lengths", 3), i32("refs", 5))

    def plan():
        return kv4.rope_plan(place("cos_sin", torch.zeros(9, 32, 2)))

    def scratch():
        return place("workspace", torch.zeros(1 << 15, dtype=torch.uint8))

    status = i32("status", 1)
    yield lambda: kv4.kfl_rope_table(9, 64, 1e4, out=place("out", torch.zeros(9, 32, 2)))
    yield lambda: kv4.kfl_rope(plan(), rows("q", 2, 4), rows("q_out", 2, 4), rows("k", 2, 2), rows("k_out", 2, 2),
                               i32("positions", 2), status=status)
    yield lambda: kv4.kfl_kv4_append(pool(), page_map(), 0, rows("k", 2, 2), rows("v", 2, 2), i32("users", 2), i32("positions", 2),
                                     rope=plan(), status=status)
    yield lambda: kv4.kfl_kv4_read(pool(), page_map(), 0, i32("users", 2), i32("positions", 2), rows("k_out", 2, 2),
                                   rows("v_out", 2, 2), status=status)
    yield lambda: kv4.kfl_kv4_attend(pool(), page_map(), 0, rows("q", 2, 4), rows("out", 2, 4), scratch(), users=i32("users", 1),
                                     q_start=i32("q_start", 2), max_q=2, lse=place("lse", torch.zeros(2, 4)), status=status)
    yield lambda: kv4.kfl_kv4_reserve(pool(), page_map(), i32("users", 2), i32("n_new", 2), scratch(), status=status)
    yield lambda: kv4.kfl_kv4_fork(pool(), page_map(), i32("src", 2), i32("dst", 2), scratch(), status=status)
    yield lambda: kv4.kfl_kv4_free(pool(), page_map(), i32("users", 2), status=status)
    yield lambda: kv4.kfl_kv4_compact(pool(), page_map(), i32("table_out", 12), i32("refs_out", 5), i32("n_live", 1), scratch(),
                                      status=status)
    yield lambda: kv4.kfl_kv4_copy_pages(pool(), i32("src", 2), i32("dst", 2), status=status)


class Names(list):
    def __init__(self):
        super().__init__()
        self.args = []


@pytest.fixture
def recorded(monkeypatch, lib):  # noqa: F811
    """The library's calls do nothing and succeed; a list of their names."""
    made = Names()

    class Library:
        def __getattr__(self, name):
            if name.endswith("_bytes"):
                return getattr(lib, name)
            return lambda *a: made.append(name) or made.args.append(a) or 0

    monkeypatch.setattr(kv4, "lib", lambda: Library())
    monkeypatch.setattr(kv4, "_several", False)
    return made


def test_host_tensors_are_refused(recorded):
    """Each tensor of each call: its address would go to a kernel as it is."""
    names = []
    for call in calls(lambda name, t: names.append(name) or OnDevice(t)):
        call()
    assert len(recorded) == 10
    for host in sorted(set(names)):
        del recorded[:]
        refused = 0
        for call in calls(lambda name, t: t if name == host else OnDevice(t)):  # noqa: B023
            try:
                call()
            except ValueError as e:
                assert "current CUDA device" in str(e)
                refused += 1
        assert refused > 0 and refused + len(recorded) == 10, host


def test_tensors_of_another_device_are_refused(recorded, monkeypatch):
    monkeypatch.setattr(kv4, "_several", True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in calls(lambda name, t: OnDevice(t, 1)):
        call()
    assert len(recorded) == 10
    del recorded[:]
    for call in calls(lambda name, t: OnDevice(t, 0)):
        with pytest.raises(ValueError, match="current CUDA device"):
            call()
    assert recorded == []
    # descriptions that were made while another device was the current one
    p = kv4.pool(OnDevice(torch.zeros(5 * 16 * 72, dtype=torch.uint8), 1), 16, 1, 1, 64)
    m = kv4.page_map(*(OnDevice(torch.zeros(s, dtype=torch.int32), 1) for s in ((3, 4), 3, 5)))
    plan = kv4.rope_plan(OnDevice(torch.zeros(9, 32, 2), 1))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for h in (p, m, plan):
        with pytest.raises(ValueError, match="current CUDA device"):
            kv4._handle(h)


def test_the_attentions_workspace_is_memory_of_its_size(recorded):
    """What is handed on as its size is the bytes behind its address: not an expanded tensor's count, nor that of its elements."""
    pool = kv4.pool(OnDevice(torch.zeros(5 * 16 * 72, dtype=torch.uint8)), 16, 1, 1, 64)
    m = kv4.page_map(*(OnDevice(torch.zeros(s, dtype=torch.int32)) for s in ((3, 4), 3, 5)))
    q, out = (OnDevice(torch.zeros(2, 4, 64, dtype=torch.bfloat16)) for _ in range(2))
    for bad in (torch.zeros(1, dtype=torch.uint8).expand(1 << 24), torch.zeros(1 << 16, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError, match="workspace"):
            kv4.kfl_kv4_attend(pool, m, 0, q, out, OnDevice(bad))
    assert recorded == []
    for ok in (torch.zeros(1 << 16, dtype=torch.uint8), torch.zeros(1 << 14, dtype=torch.float32)):
        kv4.kfl_kv4_attend(pool, m, 0, q, out, OnDevice(ok))
        assert recorded.args[-1][-3] == 1 << 16


def test_a_table_has_room_for_its_angles(recorded):
    for bad in (torch.zeros(8, 32, 2), torch.zeros(9, 32, 2, dtype=torch.float64), torch.zeros(9, 32, 4)[..., ::2],
                torch.zeros(1).expand(9, 32, 2)):
        with pytest.raises(ValueError, match="out is"):
            kv4.kfl_rope_table(9, 64, 1e4, out=OnDevice(bad))
    assert recorded == []
    for ok in (torch.zeros(9, 32, 2), torch.zeros(600)):
        kv4.kfl_rope_table(9, 64, 1e4, out=OnDevice(ok))
    assert recorded == ["kfl_rope_table"] * 2


@pytest.mark.parametrize("off", [1, 2, 4, 12])
def test_a_table_off_its_pairs_alignment_is_refused(lib, off):  # noqa: F811
    """cos and sin are stored as a pair of 8 bytes."""
    cfg = kv4.kfl_rope_cfg(64, 0, 1e4, 1.0, 0.0, 0.0, 0.0, 0.0)
    assert lib.kfl_rope_table(C.byref(cfg), 10, (1 << 20) + off, None) == K.KFL_ERR_ARG
    assert "aligned" in K.kfl_last_error_detail()


def test_more_query_rows_than_are_counted_are_refused(lib):  # noqa: F811
    """2^24 tokens of 128 heads per KV head: their count would pass 31 bits on the device."""
    def attend(n, max_q, n_seqs=1):
        q = kv4.kfl_heads(1 << 20, 256 * 64, 64, 256, 0)
        p = kv4.kfl_kv4_pool(1 << 20, 10, 16, 1, 2, 64)
        m = kv4.kfl_kv4_map(1 << 20, 1 << 20, 1 << 20, 3, 4)
        return lib.kfl_kv4_attend(C.byref(p), C.byref(m), 0, C.byref(q), C.byref(q), None, None, 1 << 20, n_seqs, n, max_q, 1.0, 0,
                                  1 << 20, 1 << 50, None, None)

    for n, max_q in ((1 << 24, 1 << 24), ((1 << 23) + 1, 2 ** 31 - 1), (2 ** 31 - 1, (1 << 23) + 1)):
        assert attend(n, max_q) == K.KFL_ERR_RANGE
        assert "query rows" in K.kfl_last_error_detail()
