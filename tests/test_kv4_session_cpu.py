"""The example's session without a GPU: what it hands to the library's calls, which are recorded in their place."""
import types

import pytest
import torch

from paper_2609_34045_gb300 import kv4, kv4_session

STREAM = 0x5EED
CALLS = ("kfl_rope_table", "kfl_rope", "kfl_kv4_reserve", "kfl_kv4_append", "kfl_kv4_attend", "kfl_kv4_fork", "kfl_kv4_free",
         "kfl_kv4_compact")


@pytest.fixture
def session(monkeypatch):
    """A session on CPU tensors, on a torch stream of address STREAM; `session.calls` lists (name, arguments by name)."""
    calls = []
    for name in CALLS:
        def record(*args, _name=name, **kw):
            calls.append((_name, kw))
            return torch.zeros(8, 4, 2) if _name == "kfl_rope_table" else None
        monkeypatch.setattr(kv4, name, record)
    for name in ("empty", "full", "zeros", "tensor"):
        def on_cpu(*args, _made=getattr(torch, name), device=None, **kw):
            return _made(*args, **kw)
        monkeypatch.setattr(torch, name, on_cpu)
    monkeypatch.setattr(kv4, "pool", lambda *a, **kw: None)
    monkeypatch.setattr(kv4, "page_map", lambda *a, **kw: None)
    monkeypatch.setattr(kv4, "rope_plan", lambda *a, **kw: None)
    monkeypatch.setattr(kv4, "pages_workspace", lambda *a, **kw: None)
    monkeypatch.setattr(kv4, "attend_workspace", lambda *a, **kw: None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(cuda_stream=STREAM))
    s = kv4_session.Session(1, 4, 2, 64, n_users=3, max_ctx=64, n_pages=8, page_tokens=16)
    s.calls = calls
    return s


def test_every_call_is_on_torchs_current_stream(session):
    """Inputs and outputs belong to that stream: a kernel on another one reads rows before they are written."""
    step = session.begin({0: 2, 1: 1})
    q, k = torch.zeros(3, 4, 64), torch.zeros(3, 2, 64)
    session.attend(0, step, q, k, k)
    session.fork([0], [2])
    session.free([1])
    session.compact()
    assert {name for name, _ in session.calls} == set(CALLS)
    assert [name for name, kw in session.calls if kw.get("cuda_stream") != STREAM] == []


def reserved(s):
    return [name for name, _ in s.calls].count("kfl_kv4_reserve")


def test_a_pass_that_has_no_room_is_refused_before_it_begins(session):
    """8 pages of 16 tokens, 5 of them held: by user 0 with 60 tokens (4 pages) and user 1 with 16 (1)."""
    session.lengths[:2] = torch.tensor([60, 16], dtype=torch.int32)
    session.refs[:5] = 1
    for ok in ({0: 4}, {1: 48}, {0: 4, 1: 17, 2: 16}, {2: 48}, {0: 0, 1: 0}):
        session.begin(ok)
    assert reserved(session) == 5
    for bad in ({2: 49}, {0: 4, 1: 17, 2: 17}, {1: 33, 2: 17}):  # four pages, of three
        with pytest.raises(kv4_session.NoRoom, match="free"):
            session.begin(bad)
    for bad in ({0: 5}, {2: 1, 0: 100}):  # 64 tokens a user
        with pytest.raises(kv4_session.NoRoom, match="user 0"):
            session.begin(bad)
    for bad in ({3: 1}, {-1: 1}, {0: -1, 1: 1}):
        with pytest.raises(ValueError):
            session.begin(bad)
    assert reserved(session) == 5


def test_a_row_that_ends_behind_the_longest_context(session):
    """A table's row may have room behind max_ctx, for which there are no angles."""
    session.max_ctx = 60
    session.begin({0: 60})
    with pytest.raises(kv4_session.NoRoom):
        session.begin({0: 61})


def test_a_fork_that_has_no_room_is_refused(session):
    """Two free pages, and users whose last page is full (0), not full (1) and not there (2)."""
    session.lengths[:2] = torch.tensor([16, 20], dtype=torch.int32)
    session.refs[:6] = 1
    for ok in (([1, 1], [0, 2]), ([0, 1, 1], [2, 1, 0]), ([0, 0], [1, 2]), ([2], [0]), ([], [])):
        session.fork(*ok)
    forks = [name for name, _ in session.calls].count("kfl_kv4_fork")
    assert forks == 5
    session.refs[6] = 2
    session.fork([1], [0])
    with pytest.raises(kv4_session.NoRoom, match="2 new pages are needed, 1 "):
        session.fork([1, 1], [0, 2])
    for bad in (([1], [3]), ([-1], [0]), ([1, 1], [0, 0]), ([1, 0], [2])):
        with pytest.raises(ValueError):
            session.fork(*bad)
    assert [name for name, _ in session.calls].count("kfl_kv4_fork") == forks + 1
