"""What kfl_kv4_tree_window and its binding refuse, and which views a session's passes take, without a GPU."""
import pytest
import torch

from paper_2609_34045_gb300 import kv4, kv4_session, stage
from test_abi_cpu import lib  # noqa: F401
from test_kv4_binding_cpu import OnDevice, recorded  # noqa: F401
from test_kv4_more_cpu import P
from test_kv4_session_cpu import session  # noqa: F401


def test_refusals_of_the_library(lib):  # noqa: F811
    f = kv4.lib().kfl_kv4_tree_window
    assert f(P, P, None, 0, 0, 4, 3, P, P, None, None) == 0
    for bad in ((P, P, None, -1, 4, 4, 3, P), (P, P, None, 1, -4, 4, 3, P), (P, P, None, 1, 4, 0, 3, P), (P, P, None, 1, 4, 4, -1, P),
                (None, P, None, 1, 4, 4, 3, P), (P, P, None, 1, 4, 4, 3, None), (P, None, None, 1, 4, 4, 3, P), (P, P, None, 1, 4, 1025, 3, P)):
        assert f(*bad, P, None, None) < 0
        assert b"kfl_kv4_tree_window" in stage.kfl_last_error_detail().encode()


def test_the_bindings_call(recorded):  # noqa: F811
    parents, views = OnDevice(torch.zeros(3, dtype=torch.int32)), OnDevice(torch.zeros(3, 1, dtype=torch.int32))
    for window in (0, 5, -1):
        kv4.kfl_kv4_tree(parents, views, window=window)
    assert recorded == ["kfl_kv4_tree", "kfl_kv4_tree_window", "kfl_kv4_tree_window"]
    assert [a[6] for a in recorded.args[1:]] == [5, -1] and len(recorded.args[1]) == 11


def test_a_sessions_views(session, monkeypatch):  # noqa: F811
    """Of the window where it is shorter than a path, else those of the pass's beginning."""
    calls = session.calls
    for name in ("kfl_kv4_tree", "kfl_kv4_attend_tree"):
        monkeypatch.setattr(kv4, name, lambda *a, _name=name, **kw: calls.append((_name, (a, kw))))
    step = session.begin({0: 4, 1: 3}, {0: [-1, 0, 1, 0]})
    q, k = torch.zeros(7, 4, 64), torch.zeros(7, 2, 64)
    for window in (0, 3, 2, 100, 1):
        session.attend(0, step, q, k, k, window=window)
    trees = [a for name, a in calls if name == "kfl_kv4_tree"]
    views = [a for name, a in calls if name == "kfl_kv4_attend_tree"]
    assert [kw.get("window", 0) for _, kw in trees] == [0, 2, 1]
    assert [a[5] is step["views"] for a, _ in views] == [True, True, False, True, False]
    assert [a[5].data_ptr() for a, _ in views][2::2] == [a[1].data_ptr() for a, _ in trees[1:]]
    assert all(kw["window"] == w for (_, kw), w in zip(views, (0, 3, 2, 100, 1)))
    with pytest.raises(kv4_session.NoRoom):
        session.begin({2: 65}, {})
