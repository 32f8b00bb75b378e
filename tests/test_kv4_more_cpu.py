"""Trees and evictions of the 4-bit cache without a GPU: what the oracle's new functions are pinned by, what the library's entry
points and their binding refuse, and what the session hands to them."""
import ctypes as C

import numpy as np
import pytest
import torch

import oracle.kv4 as ora
from paper_2609_34045_gb300 import kv4, kv4_session, stage
from test_abi_cpu import lib  # noqa: F401
from test_kv4_binding_cpu import Names, OnDevice, recorded  # noqa: F401
from test_kv4_session_cpu import CALLS, STREAM, session  # noqa: F401

OK, ARG, RANGE = 0, -1, None
P = 0x1000  # an address that no kernel sees


# ---- the oracle

def test_trees_of_the_oracle():
    seen, depth = ora.tree_seen([-1, 0, 0, 1, -1, 4])
    assert depth.tolist() == [0, 1, 1, 2, 0, 1]
    assert [np.nonzero(r)[0].tolist() for r in seen] == [[0], [0, 1], [0, 2], [0, 1, 3], [4], [4, 5]]
    words = ora.tree_words(np.tril(np.ones((34, 34), dtype=bool)), 40)
    assert words[33].tolist() == [0xFFFFFFFF, 3] and words[0].tolist() == [1, 0]


def test_keys_of_trees():
    seen, _ = ora.tree_seen([-1, 0, -1])
    assert ora.tree_keys(seen, 5).astype(int).tolist() == [[1, 1, 1, 0, 0], [1, 1, 1, 1, 0], [1, 1, 0, 0, 1]]
    assert ora.tree_keys(seen, 5, 2).astype(int).tolist() == [[0, 1, 1, 0, 0], [0, 0, 1, 1, 0], [0, 1, 0, 0, 1]]
    chain = np.tril(np.ones((4, 4), dtype=bool))
    for n, window in ((4, 0), (9, 0), (9, 4), (9, 5), (2, 0)):  # a chain is causal, windows that hold it too
        assert np.array_equal(ora.tree_keys(chain, n, window), ora.causal_keys(4, n, window))


def test_attention_and_weights_of_the_oracle():
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(n, 8, generator=g, dtype=torch.float64).numpy() for n in (3, 6, 6))
    keys = np.array([[1, 0, 1, 0, 0, 1], [0] * 6, [1] * 6], dtype=bool)
    out, _, lse = ora.attend_keys(q, k, v, keys, 0.3)
    ref = torch.nn.functional.scaled_dot_product_attention(*(torch.from_numpy(x)[None] for x in (q, k, v)),
                                                           attn_mask=torch.from_numpy(keys)[None], scale=0.3)[0].numpy()
    assert np.abs(out - ref)[[0, 2]].max() < 1e-12 and (out[1] == 0).all() and lse[1] == -np.inf
    w = ora.weights(q, k, lse, keys, 0.3)
    assert np.allclose(w.sum(1), [1, 0, 1]) and np.allclose(w @ v, out)
    causal, _, causal_lse = ora.attend(q, k, v, [3, 4, 5], 0.3, 2)
    again, _, again_lse = ora.attend_keys(q, k, v, ora.causal_keys(3, 6, 2), 0.3)
    assert np.allclose(causal, again) and np.allclose(causal_lse, again_lse)


def test_selection_of_the_oracle():
    mass = np.array([5, 1, 3, 3, 0, 3, 9, 2], dtype=np.float32)
    assert ora.select(mass, 8, 8, 0, 0).tolist() == list(range(8))
    assert ora.select(mass, 8, 3, 0, 0).tolist() == [0, 2, 6]
    assert ora.select(mass, 8, 4, 1, 2).tolist() == [0, 2, 6, 7]
    assert ora.select(mass, 5, 2, 0, 1).tolist() == [0, 4]
    mass[4] = np.nan
    assert ora.select(mass, 8, 2, 0, 0).tolist() == [4, 6]


def test_kept_pages_of_the_oracle():
    t = ora.Pages(np.array([[0, 1, 2, -1], [0, 1, 3, -1]], dtype=np.int32), np.array([40, 45], dtype=np.int32),
                  np.array([2, 2, 1, 1, 0, 0], dtype=np.int32), 16)
    old = t.keep([0, 1], [4, 45], [20, 0])  # rows move inside two shared pages; the second user loses nothing
    assert old[1] is None and old[0].tolist() == [0, 1, 2, -1]
    assert t.table.tolist() == [[4, 5, -1, -1], [0, 1, 3, -1]] and t.refs.tolist() == [1, 1, 0, 1, 1, 1] and t.lengths.tolist() == [24, 45]


# ---- the library's entry points

def a_pool(pages=P, **kw):
    return kv4.kfl_kv4_pool(pages, *{**dict(n_pages=4, page_tokens=16, n_layers=2, n_kv_heads=2, head_dim=64), **kw}.values())


def a_map(**kw):
    return kv4.kfl_kv4_map(P, P, P, kw.get("n_users", 3), kw.get("max_pages", 4))


def rows_of(n_heads=4, dtype=0, data=P):
    return kv4._pack_heads(data, n_heads * 64, 64, n_heads, dtype)


def test_the_trees_refusals(lib):  # noqa: F811
    f = kv4.lib().kfl_kv4_tree
    assert f(P, P, None, 0, 0, 4, P, P, None, None) == OK and f(P, P, None, 3, 0, 4, P, P, None, None) == OK
    for bad in ((P, P, None, -1, 4, 4, P), (P, P, None, 1, -4, 4, P), (P, P, None, 1, 4, 0, P), (None, P, None, 1, 4, 4, P),
                (P, P, None, 1, 4, 4, None), (P, None, None, 1, 4, 4, P)):
        assert f(*bad, P, None, None) < 0
        assert b"kfl_kv4_tree" in stage.kfl_last_error_detail().encode()
    assert f(P, P, None, 1, 4, 1025, P, P, None, None) < 0


def test_tree_attentions_refusals(lib):  # noqa: F811
    f, big = kv4.lib().kfl_kv4_attend_tree, 1 << 30

    def call(pool=None, q=None, out=None, views=P, n_seqs=1, n_tokens=4, max_q=4, scale=1.0, window=0, ws=P, size=big, layer=0, start=P):
        return f(C.byref(pool or a_pool()), C.byref(a_map()), layer, q or rows_of(), out or rows_of(), None, None, start, views, n_seqs,
                 n_tokens, max_q, scale, window, ws, size, None, None)

    assert call(n_seqs=0, n_tokens=0) == OK
    for bad in (dict(views=None), dict(views=P + 2), dict(max_q=1025), dict(layer=2), dict(q=rows_of(3)), dict(out=rows_of(4, 1)),
                dict(scale=float("nan")), dict(window=-1), dict(ws=None), dict(size=64), dict(pool=a_pool(head_dim=96)),
                dict(start=None), dict(q=rows_of(4, 2), out=rows_of(4, 2))):
        assert call(**bad) < 0, bad
        assert b"kfl_kv4_attend" in stage.kfl_last_error_detail().encode()


def test_the_weights_refusals(lib):  # noqa: F811
    f, big = kv4.lib().kfl_kv4_weights, 1 << 30
    mass = kv4.kfl_kv4_mass(P, 384, 128, 64)

    def call(pool=None, q=None, lse=P, mass=mass, n_seqs=1, n_tokens=4, max_q=4, scale=1.0, window=0, ws=P, size=big, layer=0, start=P,
             max_pages=4):
        return f(C.byref(pool or a_pool()), C.byref(a_map(max_pages=max_pages)), layer, q or rows_of(), lse, mass and C.byref(mass), None,
                 start, n_seqs, n_tokens, max_q, scale, window, ws, size, None, None)

    assert call(n_seqs=0, n_tokens=0) == OK
    for bad in (dict(lse=None), dict(mass=None), dict(mass=kv4.kfl_kv4_mass(None, 1, 1, 1)), dict(mass=kv4.kfl_kv4_mass(P + 2, 1, 1, 1)),
                dict(n_seqs=1025, n_tokens=1025, start=None), dict(layer=-1), dict(q=rows_of(3)), dict(q=rows_of(4, 2)), dict(ws=P + 8),
                dict(scale=float("inf")), dict(window=-1), dict(size=0), dict(start=None), dict(max_pages=(1 << 22) + 1),
                dict(pool=a_pool(pages=None)), dict(lse=P + 1)):
        assert call(**bad) < 0, bad
        assert b"kfl_kv4_" in stage.kfl_last_error_detail().encode()


def test_the_selections_refusals(lib):  # noqa: F811
    f = kv4.lib().kfl_kv4_select
    mass = kv4.kfl_kv4_mass(P, 384, 128, 64)

    def call(n=1, budget=8, first=0, recent=0, users=P, rows=P, counts=P, mass=mass, max_pages=4):
        return f(C.byref(a_pool()), C.byref(a_map(max_pages=max_pages)), mass and C.byref(mass), users, n, budget, first, recent, rows, counts,
                 None, None)

    assert call(n=0) == OK
    for bad in (dict(n=-1), dict(n=1025), dict(budget=0), dict(budget=(1 << 26) + 1), dict(first=-1), dict(recent=-1), dict(first=5, recent=4),
                dict(first=2 ** 31 - 1, recent=2 ** 31 - 1), dict(users=None), dict(rows=None), dict(counts=None), dict(mass=None),
                dict(max_pages=(1 << 22) + 1)):
        assert call(**bad) < 0, bad
        assert b"kfl_kv4_select" in stage.kfl_last_error_detail().encode()


def test_keepings_refusals(lib):  # noqa: F811
    f = kv4.lib().kfl_kv4_keep

    def call(n=1, users=P, rows=kv4.kfl_kv4_rows(P, 0, 4, 0, 4), counts=P, mass=None, ws=P, pool=None, max_pages=4):
        return f(C.byref(pool or a_pool()), C.byref(a_map(max_pages=max_pages)), users, rows and C.byref(rows), None, counts, mass and C.byref(mass),
                 n, ws, None, None)

    assert call(n=0) == OK
    for bad in (dict(n=-1), dict(n=1025), dict(users=None), dict(counts=None), dict(rows=None), dict(rows=kv4.kfl_kv4_rows(None, 0, 0, 0, 4)),
                dict(rows=kv4.kfl_kv4_rows(P, 0, 0, 0, -1)), dict(mass=kv4.kfl_kv4_mass(None, 0, 0, 0)), dict(ws=None), dict(ws=P + 4),
                dict(pool=a_pool(pages=None)), dict(pool=a_pool(page_tokens=17)), dict(max_pages=(1 << 22) + 1)):
        assert call(**bad) < 0, bad
        assert b"kfl_kv4_keep" in stage.kfl_last_error_detail().encode()


# ---- the binding

def handles(place):
    p = kv4.pool(place("pages", torch.zeros(5 * 2 * 2 * 16 * 72, dtype=torch.uint8)), 16, 2, 2, 64)
    m = kv4.page_map(place("table", torch.zeros(3, 4, dtype=torch.int32)), place("lengths", torch.zeros(3, dtype=torch.int32)),
                     place("refs", torch.zeros(5, dtype=torch.int32)))
    return p, m


def more_calls(place):
    def i32(name, *n):
        return place(name, torch.zeros(*n, dtype=torch.int32))

    def mass():
        return place("mass", torch.zeros(2, 3, 2, 64))

    def scratch():
        return place("workspace", torch.zeros(1 << 15, dtype=torch.uint8))

    def q(name):
        return place(name, torch.zeros(2, 4, 64, dtype=torch.bfloat16))

    status = i32("status", 1)
    yield lambda: kv4.kfl_kv4_tree(i32("parents", 2), i32("views", 2, 1), i32("positions", 2), q_start=i32("q_start", 2),
                                   first=i32("first", 1), max_q=2, status=status)
    yield lambda: kv4.kfl_kv4_attend_tree(*handles(place), 0, q("q"), q("out"), i32("views", 2, 1), scratch(), users=i32("users", 1),
                                          q_start=i32("q_start", 2), max_q=2, lse=place("lse", torch.zeros(2, 4)), status=status)
    yield lambda: kv4.kfl_kv4_weights(*handles(place), 1, q("q"), place("lse", torch.zeros(2, 4)), mass(), scratch(),
                                      users=i32("users", 1), q_start=i32("q_start", 2), max_q=2, status=status)
    yield lambda: kv4.kfl_kv4_select(*handles(place), mass(), i32("users", 3), 7, i32("rows", 2, 3, 2, 7), i32("counts", 3), status=status)
    yield lambda: kv4.kfl_kv4_keep(*handles(place), i32("users", 3), i32("rows", 2, 3, 2, 7), i32("counts", 3), scratch(),
                                   first=i32("first", 3), mass=mass(), status=status)


def test_host_tensors_are_refused(recorded):  # noqa: F811
    names = []
    for call in more_calls(lambda name, t: names.append(name) or OnDevice(t)):
        call()
    assert len(recorded) == 5
    for host in sorted(set(names)):
        del recorded[:]
        refused = 0
        for call in more_calls(lambda name, t: t if name == host else OnDevice(t)):  # noqa: B023
            try:
                call()
            except ValueError as e:
                assert "current CUDA device" in str(e)
                refused += 1
        assert refused > 0 and refused + len(recorded) == 5, host


def test_tensors_of_another_device_are_refused(recorded, monkeypatch):  # noqa: F811
    monkeypatch.setattr(kv4, "_several", True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in more_calls(lambda name, t: OnDevice(t, 1)):
        call()
    assert len(recorded) == 5
    for call in more_calls(lambda name, t: OnDevice(t, 0)):
        with pytest.raises(ValueError, match="current CUDA device"):
            call()


def test_wrong_shapes_and_strides_are_refused(recorded):  # noqa: F811
    """What a kernel would read or write beyond a tensor, or two rows of masses in one place."""
    p, m = handles(lambda _, t: OnDevice(t))
    good = dict(mass=torch.zeros(2, 3, 2, 64), rows=torch.zeros(2, 3, 2, 7, dtype=torch.int32), counts=torch.zeros(3, dtype=torch.int32),
                views=torch.zeros(2, 1, dtype=torch.int32), ws=torch.zeros(1 << 15, dtype=torch.uint8))
    on = {n: OnDevice(t) for n, t in good.items()}
    users, q = OnDevice(torch.zeros(3, dtype=torch.int32)), OnDevice(torch.zeros(2, 4, 64, dtype=torch.bfloat16))
    masses = [torch.zeros(2, 3, 2, 63), torch.zeros(1, 3, 2, 64), torch.zeros(2, 2, 2, 64), torch.zeros(2, 3, 1, 64), torch.zeros(3, 2, 64),
              torch.zeros(2, 3, 2, 64, dtype=torch.float64), torch.zeros(1, 3, 2, 64).expand(2, 3, 2, 64), torch.zeros(2, 3, 2, 128)[..., ::2],
              torch.zeros(2 * 3 * 2 * 64).as_strided((2, 3, 2, 64), (384, 128, 32, 1))]
    for bad in masses:
        for call in (lambda t: kv4.kfl_kv4_select(p, m, t, users, 7, on["rows"], on["counts"]),
                     lambda t: kv4.kfl_kv4_keep(p, m, users, on["rows"], on["counts"], on["ws"], mass=t),
                     lambda t: kv4.kfl_kv4_weights(p, m, 0, q, OnDevice(torch.zeros(2, 4)), t, on["ws"])):
            with pytest.raises(ValueError, match="mass"):
                call(OnDevice(bad))
    for bad in (torch.zeros(2, 3, 2, 8, dtype=torch.int32), torch.zeros(2, 2, 2, 7, dtype=torch.int32), torch.zeros(2, 3, 2, 7, dtype=torch.int64)):
        with pytest.raises(ValueError, match="rows"):
            kv4.kfl_kv4_select(p, m, on["mass"], users, 7, OnDevice(bad), on["counts"])
    for bad in (torch.zeros(1, 3, 2, 7, dtype=torch.int32), torch.zeros(2, 3, 2, 14, dtype=torch.int32)[..., ::2], torch.zeros(2, 3, 2, 7)):
        with pytest.raises(ValueError, match="rows"):
            kv4.kfl_kv4_keep(p, m, users, OnDevice(bad), on["counts"], on["ws"])
    with pytest.raises(ValueError, match="counts"):
        kv4.kfl_kv4_keep(p, m, users, on["rows"], OnDevice(torch.zeros(2, dtype=torch.int32)), on["ws"])
    with pytest.raises(ValueError, match="workspace"):
        kv4.kfl_kv4_keep(p, m, users, on["rows"], on["counts"], OnDevice(torch.zeros(64, dtype=torch.uint8)))
    for bad in (torch.zeros(2, 2, dtype=torch.int32), torch.zeros(1, 1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)):
        with pytest.raises(ValueError, match="views"):
            kv4.kfl_kv4_attend_tree(p, m, 0, q, q, OnDevice(bad), on["ws"])
        with pytest.raises(ValueError, match="views"):
            kv4.kfl_kv4_tree(OnDevice(torch.zeros(2, dtype=torch.int32)), OnDevice(bad))
    with pytest.raises(ValueError, match="lse"):
        kv4.kfl_kv4_weights(p, m, 0, q, OnDevice(torch.zeros(2, 3)), on["mass"], on["ws"])
    assert recorded == []
    # strides that keep rows apart, and lists that all layers share, are fine
    wide = torch.zeros(3, 2, 2, 70).transpose(0, 1)[..., :64]
    kv4.kfl_kv4_select(p, m, OnDevice(wide), users, 7, on["rows"], on["counts"])
    kv4.kfl_kv4_keep(p, m, users, OnDevice(torch.zeros(1, 3, 1, 7, dtype=torch.int32).expand(2, 3, 2, 7)), on["counts"], on["ws"])
    assert recorded == ["kfl_kv4_select", "kfl_kv4_keep"]


# ---- the session

@pytest.fixture
def masses(session, monkeypatch):  # noqa: F811
    """The session of test_kv4_session_cpu with masses, and the new calls recorded too."""
    for name in ("kfl_kv4_tree", "kfl_kv4_attend_tree", "kfl_kv4_weights", "kfl_kv4_select", "kfl_kv4_keep"):
        def record(*args, _name=name, **kw):
            session.calls.append((_name, kw))
        monkeypatch.setattr(kv4, name, record)
    s = kv4_session.Session(1, 4, 2, 64, n_users=3, max_ctx=64, n_pages=8, page_tokens=16, masses=True, max_positions=100)
    s.calls = session.calls
    return s


def test_new_calls_are_on_torchs_current_stream(masses):
    s = masses
    q, k = torch.zeros(5, 4, 64), torch.zeros(5, 2, 64)
    step = s.begin({0: 3, 1: 2}, {0: [-1, 0, 0]})
    s.attend(0, step, q, k, k)
    s.lengths[:2] = torch.tensor([3, 2], dtype=torch.int32)
    s.accept(step, {0: [0, 2], 1: [0]})
    s.lengths[:2] = torch.tensor([60, 1], dtype=torch.int32)
    s.table[0] = torch.arange(4, dtype=torch.int32)
    s.attend(0, s.begin({0: 3, 1: 2}), q, k, k)
    assert s.evict(32, first=1, recent=2) == {0: 28} and s.evicted == [28, 0, 0]
    names = [name for name, _ in s.calls]
    for name in ("kfl_kv4_tree", "kfl_kv4_attend_tree", "kfl_kv4_weights", "kfl_kv4_select", "kfl_kv4_keep"):
        assert name in names
    assert [name for name, kw in s.calls if kw.get("cuda_stream") != STREAM] == []
    assert names.count("kfl_kv4_weights") == 2


def test_a_cut_user_goes_on_at_its_position(masses):
    s = masses
    s.evicted, s.lengths[0] = [28, 0, 0], 32
    step = s.begin({0: 2, 1: 1})
    assert step["slots"].tolist() == [32, 33, 0] and step["positions"].tolist() == [60, 61, 0]
    s.evicted[0] = 60
    s.begin({0: 8})
    with pytest.raises(kv4_session.NoRoom, match="position"):
        s.begin({0: 9})
    s.fork([0], [2])
    assert s.evicted == [60, 0, 60]
    s.free([0])
    assert s.evicted == [0, 0, 60]


@pytest.mark.parametrize("parents", [{0: [-1, 1]}, {0: [0, -1]}, {0: [-1]}, {0: [-1, -2]}, {2: [-1]}])
def test_trees_that_are_none_are_refused(masses, parents):
    with pytest.raises(ValueError, match="parents"):
        masses.begin({0: 2, 1: 1}, parents)
    assert masses.calls[-1][0] == "kfl_rope_table"


def test_paths_that_are_none_are_refused(masses):
    s = masses
    step = s.begin({0: 4, 1: 2}, {0: [-1, 0, 0, 1]})
    s.lengths[:2] = torch.tensor([4, 2], dtype=torch.int32)
    for paths in ({0: [1]}, {0: [0, 3]}, {0: [0, 1, 2]}, {0: [0, 4]}, {0: [-1]}, {1: [1]}, {2: [0]}):
        with pytest.raises(ValueError, match="paths"):
            s.accept(step, paths)
    with pytest.raises(ValueError, match="once"):
        s.accept(s.begin({0: 1}), {})
    s.lengths[0] = 5
    with pytest.raises(ValueError, match="last tokens"):
        s.accept(step, {0: [0]})
    s.lengths[0] = 4
    s.accept(step, {0: [0, 1, 3]})
    with pytest.raises(ValueError, match="once"):
        s.accept(step, {})
    assert [name for name, _ in s.calls].count("kfl_kv4_keep") == 1


def test_evictions_that_cannot_be_are_refused(masses, session):  # noqa: F811
    for bad in (dict(budget=0), dict(budget=4, first=3, recent=2), dict(budget=4, first=-1), dict(budget=4, recent=-1)):
        with pytest.raises(ValueError, match="budget"):
            masses.evict(**{**dict(first=0, recent=0), **bad})
    with pytest.raises(ValueError, match="masses"):
        session.evict(10)
    for users in ([0, 0], [-1], [3]):
        with pytest.raises(ValueError, match="users"):
            masses.evict(10, users, first=0, recent=0)
    masses.lengths[:2] = torch.tensor([60, 64], dtype=torch.int32)
    masses.table[:2] = torch.arange(4, dtype=torch.int32)
    masses.refs[:] = 1
    masses.refs[:4] = 2
    with pytest.raises(kv4_session.NoRoom):  # three pages of each are another's too, and none is free
        masses.evict(40, first=1, recent=2)
    assert masses.evicted == [0, 0, 0] and masses.calls[-1][0] == "kfl_rope_table"


def test_a_pass_of_trees_without_tokens(masses):
    s = masses
    step = s.begin({0: 0, 1: 0}, {})
    s.accept(step, {})
    assert "kfl_kv4_tree" not in [name for name, _ in s.calls] and "kfl_kv4_weights" not in [name for name, _ in s.calls]
