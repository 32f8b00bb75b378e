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
