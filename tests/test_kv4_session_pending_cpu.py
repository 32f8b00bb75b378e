"""Trees between their pass and their acceptance: what a session refuses meanwhile, and what it still knows them by.  Without a GPU; the
library's calls are recorded, the lengths set as their kernels would leave them."""
import pytest
import torch

from paper_2609_34045_gb300 import kv4, kv4_session
from test_kv4_more_cpu import masses  # noqa: F401
from test_kv4_session_cpu import session  # noqa: F401

TREE = [-1, 0, 0, 1]


def lengths(s, *n):
    s.lengths[:len(n)] = torch.tensor(n, dtype=torch.int32)


def done(s):
    return [name for name, _ in s.calls]


@pytest.fixture
def held(masses):  # noqa: F811
    """A session whose user 0 has 40 rows and a tree of four behind them, user 1 20 rows; the step of the tree."""
    s = masses
    lengths(s, 40, 20, 0)
    s.table[0, :3], s.table[1, :2] = torch.arange(3, dtype=torch.int32), torch.arange(3, 5, dtype=torch.int32)
    s.refs[:5] = 1
    step = s.begin({0: 4}, {0: TREE})
    lengths(s, 44, 20, 0)
    del s.calls[:]
    return s, step


def test_evictions_of_drafts_that_wait_are_refused(held):
    """The rows would stay as context for good: rejected drafts, at positions that count them."""
    s, step = held
    for users in (None, [0], [1, 0]):
        with pytest.raises(ValueError, match="accept"):
            s.evict(10, users, first=0, recent=0)
    assert done(s) == [] and s.evicted == [0, 0, 0]
    assert s.evict(10, [1], first=0, recent=0) == {1: 10}   # the others may be cut
    assert s.evict(44, [0], first=0, recent=0) == {}        # (nothing of it goes)
    s.accept(step, {0: [0, 1]})
    lengths(s, 42)
    assert s.evict(10, [0], first=0, recent=0) == {0: 32}


def test_passes_behind_drafts_that_wait_are_refused(held):
    """Their tokens would stand behind all of the tree, at positions that count its nodes."""
    s, step = held
    for counts, parents in (({0: 1}, None), ({1: 1, 0: 2}, None), ({0: 3}, {0: [-1, 0, 0]})):
        with pytest.raises(ValueError, match="accept"):
            s.begin(counts, parents)
    assert done(s) == []
    s.begin({1: 1, 0: 0})
    lengths(s, 44, 21)
    s.accept(step, {})
    lengths(s, 40)
    s.begin({0: 1})


def test_forks_of_drafts_that_wait_are_refused(held):
    s, step = held
    with pytest.raises(ValueError, match="accept"):
        s.fork([1, 0], [2, 1])
    assert done(s) == []
    s.fork([0, 1], [0, 2])  # (itself: nothing changes)
    s.accept(step, {0: [0]})
    s.fork([0], [1])


@pytest.mark.parametrize("leave", ["free", "fork"])
def test_a_user_that_left_and_grew_again_is_another(held, leave):
    """Freed, or forked over: as many rows as before, none of them the tree's."""
    s, step = held
    if leave == "free":
        s.free([0])
    else:
        s.fork([1], [0])
    lengths(s, 0 if leave == "free" else 20)
    s.begin({0: 44 if leave == "free" else 24})
    lengths(s, 44)
    del s.calls[:]
    with pytest.raises(ValueError, match="last tokens"):
        s.accept(step, {0: [0, 1]})
    assert done(s) == []


def test_the_others_of_a_pass_are_accepted_when_one_has_left(masses):  # noqa: F811
    s = masses
    step = s.begin({0: 4, 1: 2, 2: 3}, {0: TREE})
    lengths(s, 4, 2, 3)
    q, k = torch.zeros(9, 4, 64), torch.zeros(9, 2, 64)
    s.attend(0, step, q, k, k)
    s.free([1])
    lengths(s, 4, 0, 3)
    with pytest.raises(ValueError, match="last tokens"):
        s.accept(step, {0: [0, 2], 1: [0]})
    kept = []
    for name in ("kfl_kv4_keep", "kfl_kv4_weights"):
        def record(*args, _name=name, **kw):
            kept.append((_name, args, kw))
        setattr(kv4, name, record)  # (the fixture puts the real ones back)
    s.accept(step, {0: [0, 2], 2: [0, 1, 2]})
    (_, args, kw), (_, wargs, wkw) = kept
    assert args[2].tolist() == [0, 2] and args[4].tolist() == [2, 3] and kw["first"].tolist() == [0, 0]
    assert args[3][0, :, 0].tolist() == [[0, 2, -1], [0, 1, 2]]
    assert wkw["users"].tolist() == [0, 2] and wkw["q_start"].tolist() == [0, 2, 5] and wkw["max_q"] == 3 and len(wargs[3]) == 5
    with pytest.raises(ValueError, match="once"):
        s.accept(step, {})


def test_a_pass_whose_users_have_all_left(masses):  # noqa: F811
    s = masses
    step = s.begin({0: 4}, {0: TREE})
    s.free([0])
    del s.calls[:]
    s.accept(step, {})
    assert done(s) == []
