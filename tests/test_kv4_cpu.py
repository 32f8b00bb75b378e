"""The 4-bit cache's host side and its oracle, without a GPU: refusals before any launch, sizes, and the oracle's pins."""
import ctypes as C
import os

import numpy as np
import pytest
import torch

import oracle.kv4 as ora
from paper_2609_34045_gb300 import kv4
from paper_2609_34045_gb300 import stage as K


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(K.LIB_PATH):
        from paper_2609_34045_gb300.build import build
        build()
    return kv4.lib()


AT = 1 << 20  # an address that is never read


def heads(n=4, dtype=0, data=AT):
    return kv4.kfl_heads(data, 4 * 64, 64, n, dtype)


def pool(**kw):
    f = dict(pages=AT, n_pages=10, page_tokens=16, n_layers=2, n_kv_heads=2, head_dim=64)
    f.update(kw)
    return kv4.kfl_kv4_pool(f["pages"], f["n_pages"], f["page_tokens"], f["n_layers"], f["n_kv_heads"], f["head_dim"])


def page_map(**kw):
    f = dict(table=AT, lengths=AT, refs=AT, n_users=3, max_pages=4)
    f.update(kw)
    return kv4.kfl_kv4_map(f["table"], f["lengths"], f["refs"], f["n_users"], f["max_pages"])


def ref(x):
    return None if x is None else C.byref(x)


BAD_POOLS = [dict(page_tokens=0), dict(page_tokens=48), dict(page_tokens=256), dict(head_dim=96), dict(n_kv_heads=0),
             dict(n_kv_heads=257), dict(n_layers=0), dict(n_pages=0), dict(n_pages=(1 << 20) + 1)]


@pytest.mark.parametrize("bad", BAD_POOLS + [dict(pages=None), dict(pages=AT + 8)])
def test_bad_pools(lib, bad):
    p, m, h, out = pool(**bad), page_map(), heads(2), C.c_size_t(0)
    calls = [lib.kfl_kv4_append(ref(p), ref(m), 0, ref(h), ref(h), AT, AT, 1, None, None, None),
             lib.kfl_kv4_read(ref(p), ref(m), 0, AT, AT, 1, ref(h), ref(h), None, None),
             lib.kfl_kv4_attend(ref(p), ref(m), 0, ref(h), ref(h), None, None, None, 1, 1, 1, 1.0, 0, AT, 1 << 40, None, None),
             lib.kfl_kv4_fork(ref(p), ref(m), AT, AT, 1, AT, None, None),
             lib.kfl_kv4_compact(ref(p), ref(m), AT, AT, None, AT, None, None),
             lib.kfl_kv4_copy_pages(ref(p), AT, AT, 1, None, None)]
    if "pages" not in bad:  # calls that touch no bytes
        calls += [lib.kfl_kv4_page_bytes(ref(p), C.byref(out)), lib.kfl_kv4_reserve(ref(p), ref(m), AT, AT, 1, AT, None, None),
                  lib.kfl_kv4_free(ref(p), ref(m), AT, 1, None, None), lib.kfl_kv4_pages_workspace_bytes(ref(p), C.byref(out)),
                  lib.kfl_kv4_attend_workspace_bytes(ref(p), 2, 1, 1, 1, C.byref(out))]
    assert set(calls) == {K.KFL_ERR_ARG}


@pytest.mark.parametrize("bad", [dict(table=None), dict(lengths=None), dict(refs=None), dict(n_users=0), dict(max_pages=0),
                                 dict(n_users=1 << 20, max_pages=1 << 12)])
def test_bad_maps(lib, bad):
    p, m, h = pool(), page_map(**bad), heads(2)
    assert lib.kfl_kv4_append(ref(p), ref(m), 0, ref(h), ref(h), AT, AT, 1, None, None, None) == K.KFL_ERR_ARG
    assert lib.kfl_kv4_reserve(ref(p), ref(m), AT, AT, 1, AT, None, None) == K.KFL_ERR_ARG
    assert lib.kfl_kv4_free(ref(p), ref(m), AT, 1, None, None) == K.KFL_ERR_ARG


def test_refused_rows(lib):
    p, m, h = pool(), page_map(), heads(2)
    append = lambda layer=0, k=h, v=h, pos=AT, n=1, rope=None: lib.kfl_kv4_append(  # noqa: E731
        ref(p), ref(m), layer, ref(k), ref(v), AT, pos, n, ref(rope), None, None)
    assert append(layer=2) == append(layer=-1) == K.KFL_ERR_RANGE
    assert "layer" in K.kfl_last_error_detail()
    for bad in (dict(k=None), dict(v=heads(3)), dict(v=heads(2, 1)), dict(k=heads(2, 3)), dict(k=heads(2, 0, None)),
                dict(k=heads(2, 0, AT + 1)), dict(pos=None), dict(n=-1), dict(rope=kv4.kfl_rope_plan(AT, 10, 66, 0)),
                dict(rope=kv4.kfl_rope_plan(None, 10, 64, 0)), dict(rope=kv4.kfl_rope_plan(AT, 10, 64, 2)),
                dict(rope=kv4.kfl_rope_plan(AT + 8, 10, 64, 0))):
        assert append(**bad) == K.KFL_ERR_ARG, bad
    assert append(n=0, pos=None) == K.KFL_OK  # nothing to do


def test_refused_attention(lib):
    p, m = pool(), page_map()

    def attend(q=heads(4), out=heads(4), layer=0, q_start=AT, n_seqs=1, n=4, max_q=4, scale=1.0, window=0, ws=AT, size=1 << 40, mm=m):
        return lib.kfl_kv4_attend(ref(p), ref(mm), layer, ref(q), ref(out), None, None, q_start, n_seqs, n, max_q, scale, window,
                                  ws, size, None, None)

    assert attend(layer=5) == K.KFL_ERR_RANGE
    for bad in (dict(q=heads(3), out=heads(3)), dict(out=heads(2)), dict(out=heads(4, 1)), dict(q=heads(4, 2), out=heads(4, 2)),
                dict(q=heads(258), out=heads(258)), dict(q=None), dict(max_q=0), dict(n=-1), dict(n_seqs=-1), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(window=-1), dict(q_start=None, n=2), dict(ws=None), dict(ws=AT + 4), dict(size=100),
                dict(mm=page_map(max_pages=1 << 23))):
        assert attend(**bad) == K.KFL_ERR_ARG, bad


def test_refused_rotations(lib):
    plan, q = kv4.kfl_rope_plan(AT, 10, 64, 0), heads(4)

    def rope(plan=plan, q=q, q_out=heads(4), k=None, k_out=None, pos=AT, n=1, hd=64):
        return lib.kfl_rope(ref(plan), ref(q), ref(q_out), ref(k), ref(k_out), pos, n, hd, 0, None, None)

    for bad in (dict(plan=None), dict(plan=kv4.kfl_rope_plan(AT, 0, 64, 0)), dict(plan=kv4.kfl_rope_plan(AT, 10, 63, 0)),
                dict(plan=kv4.kfl_rope_plan(AT, 10, 514, 0), hd=514), dict(q=None), dict(q_out=heads(3)), dict(q_out=heads(4, 1)),
                dict(k=heads(2)), dict(k_out=heads(2)), dict(k=heads(2), k_out=heads(1)), dict(k=heads(2, 1), k_out=heads(2, 1)),
                dict(pos=None), dict(n=-1), dict(hd=62), dict(hd=65), dict(hd=514)):
        assert rope(**bad) == K.KFL_ERR_ARG, bad
    assert rope(n=0, pos=None) == K.KFL_OK

    def table(n=10, out=AT, **kw):
        f = dict(rope_dim=64, scaling=0, theta=1e4, factor=1.0, low=0.0, high=0.0, original_ctx=0.0, magnitude=0.0)
        f.update(kw)
        return lib.kfl_rope_table(C.byref(kv4.kfl_rope_cfg(*f.values())), n, out, None)

    for bad in (dict(rope_dim=63), dict(rope_dim=0), dict(rope_dim=514), dict(theta=1.0), dict(theta=float("inf")), dict(scaling=5),
                dict(scaling=1, factor=0.5), dict(scaling=2, factor=2.0, rope_dim=2), dict(scaling=3, factor=2.0),
                dict(scaling=4, factor=2.0, low=2.0, high=1.0, original_ctx=100.0), dict(magnitude=-1.0), dict(n=0), dict(out=None)):
        assert table(**bad) == K.KFL_ERR_ARG, bad


def test_refused_lists(lib):
    p, m = pool(), page_map()
    assert lib.kfl_kv4_reserve(ref(p), ref(m), AT, AT, 1025, AT, None, None) == K.KFL_ERR_RANGE
    assert lib.kfl_kv4_fork(ref(p), ref(m), AT, AT, 1025, AT, None, None) == K.KFL_ERR_RANGE
    assert lib.kfl_kv4_free(ref(p), ref(m), AT, 1025, None, None) == K.KFL_ERR_RANGE
    for call in (lib.kfl_kv4_reserve, lib.kfl_kv4_fork):
        assert call(ref(p), ref(m), None, AT, 1, AT, None, None) == K.KFL_ERR_ARG
        assert call(ref(p), ref(m), AT, None, 1, AT, None, None) == K.KFL_ERR_ARG
        assert call(ref(p), ref(m), AT, AT, 1, None, None, None) == K.KFL_ERR_ARG
        assert call(ref(p), ref(m), AT, AT, 1, AT + 4, None, None) == K.KFL_ERR_ARG
        assert call(ref(p), ref(m), AT, AT, 0, AT, None, None) == K.KFL_OK
    assert lib.kfl_kv4_compact(ref(p), ref(m), None, AT, None, AT, None, None) == K.KFL_ERR_ARG
    assert lib.kfl_kv4_copy_pages(ref(p), None, AT, 1, None, None) == K.KFL_ERR_ARG
    assert lib.kfl_kv4_copy_pages(ref(p), AT, AT, 0, None, None) == K.KFL_OK


def test_sizes(lib):
    p = kv4.pool(None, 64, 14, 4, 128, n_pages=100)
    assert kv4.kfl_kv4_page_bytes(p) == 14 * 4 * 64 * 128 * 9 // 8
    few, many = (kv4.kfl_kv4_attend_workspace_bytes(p, 28, 4, 4 * n, n) for n in (1, 100))
    assert 0 < few < many  # the larger calls' workspace covers the smaller ones
    assert kv4.kfl_kv4_attend_workspace_bytes(p, 28, 8, 8, 2) <= many


def test_the_binding_refuses_what_it_can_see(lib):
    t = torch.zeros(2, 3, 64, dtype=torch.bfloat16)
    for bad in (t.double(), t[..., ::2], t[0]):
        with pytest.raises(ValueError):
            kv4._heads(bad, "q")
    with pytest.raises(ValueError):
        kv4.pool(torch.zeros(100, dtype=torch.uint8), 16, 1, 1, 64)
    with pytest.raises(ValueError):
        kv4.rope_plan(torch.zeros(4, 4))
    with pytest.raises(KeyError):
        kv4.rope_plan(torch.zeros(4, 4, 2), "other")
    with pytest.raises(ValueError):
        kv4._int32(torch.zeros(3, dtype=torch.int64), "users")
    with pytest.raises(ValueError):
        kv4._int32(torch.zeros(3, dtype=torch.int32), "users", 4)


# ---- the oracle's pins

def test_oracle_format_by_hand():
    x = np.zeros((1, 64), dtype=np.float32)
    x[0, :16] = np.arange(16)  # lo 0, hi 15: a step of one, the centre at code 8
    codes, par = ora.quantise(x)
    assert par[0, 0].tolist() == [1.0, 8.0]
    assert codes[0, :16].tolist() == list(range(16))
    assert np.array_equal(ora.values(codes, par), x.astype(np.float64))


def test_oracle_error_is_half_a_step():
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((200, 128)) * 10 ** rng.uniform(-3, 3, (200, 1))).astype(np.float32)
    codes, par = ora.quantise(x)
    assert codes.max() == 15 and codes.min() == 0
    off = np.abs(ora.values(codes, par) - x).reshape(200, 2, 64).max(-1)
    spread = np.ptp(x.reshape(200, 2, 64), -1)
    assert (off <= spread / 30 + 2.0 ** -11 * (spread + np.abs(x).reshape(200, 2, 64).max(-1)) + 2.0 ** -24).all()


def test_oracle_unpacks_low_nibbles_first():
    block = np.zeros(16 * 64 * 9 // 8, dtype=np.uint8)
    block[0], block[16 * 32 + 31] = 0x21, 0x43
    block[2 * 16 * 32:2 * 16 * 32 + 4] = np.array([0.5, 3.0], dtype=np.float16).view(np.uint8)
    kc, vc, kp, vp = ora.unpack(block, 16, 64)
    assert kc[0, :2].tolist() == [1, 2] and vc[0, -2:].tolist() == [3, 4]
    assert kp[0, 0].tolist() == [0.5, 3.0] and (vp == 0).all()


def test_oracle_attention_against_torch():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((5, 16)), rng.standard_normal((9, 16)), rng.standard_normal((9, 16))
    pos = np.arange(4, 9)
    mask = torch.from_numpy(np.arange(9)[None, :] <= pos[:, None])
    want = torch.nn.functional.scaled_dot_product_attention(*(torch.from_numpy(x)[None] for x in (q, k, v)), attn_mask=mask[None])
    got, size, lse = ora.attend(q, k, v, pos, 0.25)
    assert np.abs(got - want[0].numpy()).max() < 1e-12 and (size >= np.abs(got) - 1e-12).all()
    one, _, _ = ora.attend(q, k, v, pos, 0.25, window=1)
    assert np.array_equal(one, v[pos])
    none, _, lse = ora.attend(q[:1], k, v, [-1], 0.25)
    assert (none == 0).all() and np.isneginf(lse).all()


def test_oracle_rotation_keeps_lengths_and_differences():
    rng = np.random.default_rng(2)
    x, y = rng.standard_normal((1, 1, 24)), rng.standard_normal((1, 1, 24))
    f = 1e4 ** (-np.arange(0, 16, 2) / 16)
    for inter in (False, True):
        turn = lambda a, n: ora.rotate(a, n * f[None], inter)[0, 0]  # noqa: E731,B023
        assert np.isclose(np.linalg.norm(turn(x, 7)), np.linalg.norm(x))
        assert np.isclose(turn(x, 9) @ turn(y, 4), turn(x, 5) @ turn(y, 0))
        assert np.array_equal(turn(x, 3)[16:], x[0, 0, 16:])


def test_oracle_pages_by_hand():
    p = ora.Pages(np.full((3, 3), -1, dtype=np.int32), np.zeros(3, dtype=np.int32), np.zeros(6, dtype=np.int32), 4)
    p.reserve([0, 1], [6, 4])
    assert p.table.tolist() == [[0, 1, -1], [2, -1, -1], [-1, -1, -1]] and p.refs.tolist() == [1, 1, 1, 0, 0, 0]
    assert p.fork([0], [2]) == [(1, 3)]
    assert p.table[2].tolist() == [0, 3, -1] and p.refs.tolist() == [2, 1, 1, 1, 0, 0]
    p.free([0])
    assert p.refs.tolist() == [1, 0, 1, 1, 0, 0]
    assert p.compact() == ([(3, 1)], 3) and p.table[2].tolist() == [0, 1, -1] and p.refs.tolist() == [1, 1, 1, 0, 0, 0]
