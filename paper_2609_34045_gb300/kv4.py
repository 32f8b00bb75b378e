"""Python binding of ``include/kafila_rope.h``, ``include/kafila_kv4.h``, ``include/kafila_kv4_tree.h`` and
``include/kafila_kv4_evict.h``: rotary positions, the 4-bit paged KV cache, trees of drafted tokens over it and rows that leave
it (argument marshalling only, as in ``stage``).

Functions named ``kfl_*`` call the C entry point of that name on CUDA tensors.  ``rope_plan``, ``pool`` and
``page_map`` describe buffers that the caller keeps; ``attend_workspace`` and ``pages_workspace`` allocate the
scratch that those calls want.  Rows of heads are tensors ``[token][head][head_dim]`` of any strides whose last
is 1.  Every tensor lies in the memory of the current device; others are refused.
"""
from __future__ import annotations

import ctypes as C
import math
import struct

import torch

from . import stage
from .stage import KflError  # noqa: F401

KFL_BAD_POSITION, KFL_BAD_USER, KFL_BAD_PAGE, KFL_NO_PAGES, KFL_TIMED_OUT = 1, 2, 4, 8, 16
LAYOUTS = {"half": 0, "interleaved": 1}
SCALINGS = {"plain": 0, "linear": 1, "base": 2, "bands": 3, "ramp": 4}
_DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}


class kfl_heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64),
                ("n_heads", C.c_int), ("dtype", C.c_int)]


# the same as packed bytes, in a third of a ctypes structure's time: a decode step's kernel is over in less than its
# arguments take
_pack_heads = struct.Struct("@Pqqii").pack
_pack_mass = struct.Struct("@Pqqq").pack
_pack_rows = struct.Struct("@Pqqqi4x").pack


class kfl_rope_cfg(C.Structure):
    _fields_ = [("rope_dim", C.c_int), ("scaling", C.c_int), ("theta", C.c_double), ("factor", C.c_double),
                ("low", C.c_double), ("high", C.c_double), ("original_ctx", C.c_double), ("magnitude", C.c_double)]


class kfl_rope_plan(C.Structure):
    _fields_ = [("cos_sin", C.c_void_p), ("n_pos", C.c_int), ("rope_dim", C.c_int), ("layout", C.c_int)]


class kfl_kv4_pool(C.Structure):
    _fields_ = [("pages", C.c_void_p)] + [(n, C.c_int) for n in ("n_pages", "page_tokens", "n_layers", "n_kv_heads",
                                                                 "head_dim")]


class kfl_kv4_map(C.Structure):
    _fields_ = [("table", C.c_void_p), ("lengths", C.c_void_p), ("refs", C.c_void_p), ("n_users", C.c_int),
                ("max_pages", C.c_int)]


class kfl_kv4_mass(C.Structure):
    _fields_ = [("data", C.c_void_p)] + [(n, C.c_int64) for n in ("layer_stride", "user_stride", "head_stride")]


class kfl_kv4_rows(C.Structure):
    _fields_ = [("data", C.c_void_p)] + [(n, C.c_int64) for n in ("layer_stride", "seq_stride", "head_stride")] + [
        ("most", C.c_int)]


_lib = _signed = None
_several = True  # whether a tensor may be another device's (until the library is loaded: perhaps)


def lib() -> C.CDLL:
    """The library of ``stage.lib()`` with the signatures of these entry points."""
    global _lib, _signed, _several
    L = stage.lib()
    if _signed is not L:
        vp, i, f, P = C.c_void_p, C.c_int, C.c_float, C.POINTER
        heads, plan, pl, mp, sz = vp, P(kfl_rope_plan), P(kfl_kv4_pool), P(kfl_kv4_map), P(C.c_size_t)
        mass = rows = vp
        for name, args in {
            "kfl_rope_table": [P(kfl_rope_cfg), i, vp, vp],
            "kfl_rope": [plan, heads, heads, heads, heads, vp, i, i, i, vp, vp],
            "kfl_kv4_page_bytes": [pl, sz],
            "kfl_kv4_append": [pl, mp, i, heads, heads, vp, vp, i, plan, vp, vp],
            "kfl_kv4_append_at": [pl, mp, i, heads, heads, vp, vp, vp, i, plan, vp, vp],
            "kfl_kv4_read": [pl, mp, i, vp, vp, i, heads, heads, vp, vp],
            "kfl_kv4_attend": [pl, mp, i, heads, heads, vp, vp, vp, i, i, i, f, i, vp, C.c_size_t, vp, vp],
            "kfl_kv4_attend_workspace_bytes": [pl, i, i, i, i, sz],
            "kfl_kv4_pages_workspace_bytes": [pl, sz],
            "kfl_kv4_reserve": [pl, mp, vp, vp, i, vp, vp, vp],
            "kfl_kv4_fork": [pl, mp, vp, vp, i, vp, vp, vp],
            "kfl_kv4_free": [pl, mp, vp, i, vp, vp],
            "kfl_kv4_compact": [pl, mp, vp, vp, vp, vp, vp, vp],
            "kfl_kv4_copy_pages": [pl, vp, vp, i, vp, vp],
            "kfl_kv4_tree": [vp, vp, vp, i, i, i, vp, vp, vp, vp],
            "kfl_kv4_tree_window": [vp, vp, vp, i, i, i, i, vp, vp, vp, vp],
            "kfl_kv4_attend_tree": [pl, mp, i, heads, heads, vp, vp, vp, vp, i, i, i, f, i, vp, C.c_size_t, vp, vp],
            "kfl_kv4_weights": [pl, mp, i, heads, vp, mass, vp, vp, i, i, i, f, i, vp, C.c_size_t, vp, vp],
            "kfl_kv4_select": [pl, mp, mass, vp, i, i, i, i, vp, vp, vp, vp],
            "kfl_kv4_keep": [pl, mp, vp, rows, vp, vp, mass, i, vp, vp, vp],
        }.items():
            fn = getattr(L, name)
            fn.argtypes, fn.restype = args, i
        _lib = _signed = L
        _several = torch.cuda.device_count() > 1
    return L


def _check(rc: int, where: str) -> None:
    if rc < 0:
        detail = stage.kfl_last_error_detail()
        raise KflError(rc, detail if detail.startswith(where) else where)


def _at(t, where):
    """Address of a tensor in the memory of the current device, which is where the calls run (None: NULL)."""
    if t is None:
        return None
    if not t.is_cuda or _several and t.get_device() != torch.cuda.current_device():
        raise ValueError(f"{where} is not in the memory of the current CUDA device")
    return t.data_ptr()


def _handle(h):
    """A description whose buffers are the current device's."""
    if _several and getattr(h, "device", None) not in (None, torch.cuda.current_device()):
        raise ValueError(f"the buffers of a {type(h).__name__} are not in the memory of the current CUDA device")
    return C.byref(h)


def _int32(t, where, n=None):
    if t is None:
        return None
    if t.dtype != torch.int32 or not t.is_contiguous() or (n is not None and t.numel() < n):
        raise ValueError(f"{where} is a contiguous int32 tensor" + (f" of {n}" if n is not None else ""))
    return t.data_ptr() if t.is_cuda and not _several else _at(t, where)  # (a step's call has six of them: no call more)


def _heads(t, where, n_tokens=None, head_dim=None):
    """kfl_heads of a tensor [token][head][head_dim]."""
    if t is None:
        return None
    if t.dim() != 3:
        raise ValueError(f"{where} is [token][head][head_dim]")
    n, n_heads, hd = t.shape
    per_token, per_head, one = t.stride()
    if (n != n_tokens and n_tokens is not None) or (hd != head_dim and head_dim is not None) or (one != 1 and hd != 1):
        raise ValueError(f"{where} has contiguous channels, and as many tokens and channels as the others")
    dtype = _DTYPES.get(t.dtype)
    if dtype is None:
        raise ValueError(f"{where} is bf16, fp16 or fp32")
    return _pack_heads(t.data_ptr() if t.is_cuda and not _several else _at(t, where), per_token, per_head, n_heads, dtype)


# ---- rotary positions ----------------------------------------------------------------------------

def kfl_rope_table(n_pos: int, rope_dim: int, theta: float, scaling: str = "plain", factor: float = 1.0,
                   low: float = 0.0, high: float = 0.0, original_ctx: float = 0.0, magnitude: float = 0.0, out=None,
                   cuda_stream: int | None = None):
    """cos and sin of positions [0, n_pos): fp32 [n_pos][rope_dim / 2][2] (``out``, or a new tensor)."""
    if out is None:
        out = torch.empty(max(n_pos, 0), max(rope_dim // 2, 0), 2, dtype=torch.float32, device="cuda")
    elif out.dtype != torch.float32 or not out.is_contiguous() or out.numel() < n_pos * rope_dim:
        raise ValueError("out is a contiguous fp32 [n_pos][rope_dim / 2][2]")
    cfg = kfl_rope_cfg(rope_dim, SCALINGS[scaling], theta, factor, low, high, original_ctx, magnitude)
    _check(lib().kfl_rope_table(C.byref(cfg), n_pos, _at(out, "out"), cuda_stream), "kfl_rope_table")
    return out


def rope_plan(table, layout: str = "half") -> kfl_rope_plan:
    """A rotation by a table of kfl_rope_table; keeps the tensor alive."""
    if table.dtype != torch.float32 or not table.is_contiguous() or table.dim() != 3 or table.shape[2] != 2:
        raise ValueError("a rotation's table is a contiguous fp32 [n_pos][rope_dim / 2][2]")
    code = LAYOUTS[layout]
    plan = kfl_rope_plan(_at(table, "the table"), table.shape[0], 2 * table.shape[1], code)
    plan.table, plan.device = table, table.get_device()
    return plan


def kfl_rope(plan: kfl_rope_plan, q, q_out, k, k_out, positions, inverse: bool = False, status=None,
             cuda_stream: int | None = None) -> None:
    """Rotates q into q_out and k into k_out ([token][head][head_dim]; k and k_out may be None; an output may be
    its input) by int32 positions [token].  Asynchronous."""
    n, _, hd = q.shape
    _check(lib().kfl_rope(_handle(plan), _heads(q, "q", n, hd), _heads(q_out, "q_out", n, hd), _heads(k, "k", n, hd),
                          _heads(k_out, "k_out", n, hd), _int32(positions, "positions", n), n, hd, int(inverse), _int32(status, "status", 1),
                          cuda_stream), "kfl_rope")


# ---- the cache -----------------------------------------------------------------------------------

def pool(pages, page_tokens: int, n_layers: int, n_kv_heads: int, head_dim: int, n_pages: int | None = None):
    """A pool in the uint8 tensor ``pages`` (or, for the calls that move no bytes, ``n_pages`` of none)."""
    page_bytes = n_layers * n_kv_heads * (page_tokens * head_dim * 9 // 8)
    if pages is not None:
        if pages.dtype != torch.uint8 or not pages.is_contiguous() or page_bytes < 1 or pages.numel() % page_bytes:
            raise ValueError(f"the pages are a contiguous uint8 tensor of whole pages ({page_bytes} bytes)")
        n_pages = pages.numel() // page_bytes
    p = kfl_kv4_pool(_at(pages, "the pool"), n_pages, page_tokens, n_layers, n_kv_heads, head_dim)
    p.tensor, p.device = pages, None if pages is None else pages.get_device()
    return p


def page_map(table, lengths, refs) -> kfl_kv4_map:
    """Who holds which pages: int32 table [n_users][max_pages], lengths [n_users], refs [n_pages]."""
    m = kfl_kv4_map(_int32(table, "table"), _int32(lengths, "lengths", table.shape[0]), _int32(refs, "refs"),
                    table.shape[0], table.shape[1])
    m.tensors, m.device = (table, lengths, refs), table.get_device()
    return m


def _covers(p, m):
    if m.tensors[2].numel() < p.n_pages:
        raise ValueError(f"refs is a contiguous int32 tensor of {p.n_pages}")
    return _handle(p), _handle(m)


def kfl_kv4_page_bytes(p) -> int:
    out = C.c_size_t(0)
    _check(lib().kfl_kv4_page_bytes(C.byref(p), C.byref(out)), "kfl_kv4_page_bytes")
    return out.value


def kfl_kv4_append(p, m, layer: int, k, v, users, positions, rope=None, status=None,
                   cuda_stream: int | None = None, rope_positions=None) -> None:
    """Rows of k and v ([token][KV head][head_dim]) of one layer into the users' pages at int32 positions [token];
    k rotated first where ``rope`` is a rope_plan: by the same positions, or (kfl_kv4_append_at) by ``rope_positions`` (int32
    [token]) where a row's place is not its position.  users None: row t is user t's.  Asynchronous."""
    n = k.shape[0]
    a, b = _heads(k, "k", n, p.head_dim), _heads(v, "v", n, p.head_dim)
    if rope_positions is not None:
        _check(lib().kfl_kv4_append_at(_handle(p), _handle(m), layer, a, b, _int32(users, "users", n), _int32(positions, "positions", n),
                                       _int32(rope_positions, "rope_positions", n), n, rope and _handle(rope),
                                       _int32(status, "status", 1), cuda_stream), "kfl_kv4_append_at")
        return
    _check(lib().kfl_kv4_append(_handle(p), _handle(m), layer, a, b, _int32(users, "users", n),
                                _int32(positions, "positions", n), n, rope and _handle(rope),
                                _int32(status, "status", 1), cuda_stream), "kfl_kv4_append")


def kfl_kv4_read(p, m, layer: int, users, positions, k_out, v_out, status=None, cuda_stream: int | None = None) -> None:
    """The values that the cache holds for rows (users[t], positions[t]) of one layer.  Asynchronous."""
    n = k_out.shape[0]
    a, b = _heads(k_out, "k_out", n, p.head_dim), _heads(v_out, "v_out", n, p.head_dim)
    _check(lib().kfl_kv4_read(_handle(p), _handle(m), layer, _int32(users, "users", n),
                              _int32(positions, "positions", n), n, a, b,
                              _int32(status, "status", 1), cuda_stream), "kfl_kv4_read")


def kfl_kv4_attend_workspace_bytes(p, n_heads: int, n_seqs: int, n_tokens: int, max_q: int) -> int:
    out = C.c_size_t(0)
    _check(lib().kfl_kv4_attend_workspace_bytes(C.byref(p), n_heads, n_seqs, n_tokens, max_q, C.byref(out)),
           "kfl_kv4_attend_workspace_bytes")
    return out.value


def attend_workspace(p, n_heads: int, n_seqs: int, n_tokens: int, max_q: int = 1):
    """The zeroed workspace of kfl_kv4_attend for these sizes."""
    return torch.zeros(kfl_kv4_attend_workspace_bytes(p, n_heads, n_seqs, n_tokens, max_q), dtype=torch.uint8,
                       device="cuda")


def _sequences(m, q, users, q_start, lse, workspace):
    """How many sequences a call's rows are."""
    n = q.shape[0]
    n_seqs = users.numel() if users is not None else q_start.numel() - 1 if q_start is not None else n
    if users is None and n_seqs > m.n_users:
        raise ValueError("more sequences than users")
    if lse is not None and (lse.dtype != torch.float32 or not lse.is_contiguous() or lse.numel() < n * q.shape[1]):
        raise ValueError("lse is a contiguous fp32 [token][query head]")
    if not workspace.is_contiguous():
        raise ValueError("the workspace is contiguous")
    return n_seqs


def kfl_kv4_attend(p, m, layer: int, q, out, workspace, users=None, q_start=None, max_q: int = 1, scale=None,
                   window: int = 0, lse=None, status=None, cuda_stream: int | None = None) -> None:
    """Attention of q's rows over the users' cached rows of one layer, into out (bf16 or fp16
    [token][query head][head_dim]).  Without q_start (int32 [sequence + 1]) every row is a sequence; without users
    (int32 [sequence]) sequence s is user s.  lse: fp32 [token][query head].  Asynchronous."""
    n, _, hd = q.shape
    n_seqs = _sequences(m, q, users, q_start, lse, workspace)
    a, b = _heads(q, "q", n, p.head_dim), _heads(out, "out", n, p.head_dim)
    _check(lib().kfl_kv4_attend(_handle(p), _handle(m), layer, a, b, _at(lse, "lse"),
                                _int32(users, "users"), _int32(q_start, "q_start", n_seqs + 1), n_seqs, n, max_q,
                                1.0 / math.sqrt(hd) if scale is None else scale, window, _at(workspace, "the workspace"),
                                workspace.numel() * workspace.element_size(), _int32(status, "status", 1), cuda_stream), "kfl_kv4_attend")


# ---- trees of drafted tokens ---------------------------------------------------------------------

def _views(views, n, max_q, where="views"):
    words = -(-max_q // 32)
    if views.dim() != 2 or views.shape[0] < n or views.shape[1] != words:
        raise ValueError(f"{where} is a contiguous int32 [token][{words}]")
    return _int32(views, where)


def kfl_kv4_tree(parents, views, positions=None, q_start=None, first=None, max_q: int = 1, status=None,
                 cuda_stream: int | None = None, window: int = 0) -> None:
    """Which of their sequence's nodes the nodes of drafted trees see, into views (int32 [token][ceil(max_q / 32)], a bit a
    node), and their positions, first (int32 [sequence], None: 0) + ancestors, into positions (int32 [token], may be
    None).  parents: int32 [token], counted within the sequence, -1 for none; q_start as in kfl_kv4_attend.  With a window
    (kfl_kv4_tree_window) a node sees that many of its path at most, the nearest.  Asynchronous."""
    n = parents.numel()
    n_seqs = q_start.numel() - 1 if q_start is not None else n
    trees = (_int32(parents, "parents"), _int32(q_start, "q_start"), _int32(first, "first", n_seqs), n_seqs, n, max_q)
    rest = (_views(views, n, max_q), _int32(positions, "positions", n), _int32(status, "status", 1), cuda_stream)
    if window:
        _check(lib().kfl_kv4_tree_window(*trees, window, *rest), "kfl_kv4_tree_window")
    else:
        _check(lib().kfl_kv4_tree(*trees, *rest), "kfl_kv4_tree")


def kfl_kv4_attend_tree(p, m, layer: int, q, out, views, workspace, users=None, q_start=None, max_q: int = 1, scale=None,
                        window: int = 0, lse=None, status=None, cuda_stream: int | None = None) -> None:
    """kfl_kv4_attend of the nodes of trees: of its sequence's last tokens each sees those of its row of views
    (kfl_kv4_tree).  Asynchronous."""
    n, _, hd = q.shape
    n_seqs = _sequences(m, q, users, q_start, lse, workspace)
    a, b = _heads(q, "q", n, p.head_dim), _heads(out, "out", n, p.head_dim)
    _check(lib().kfl_kv4_attend_tree(_handle(p), _handle(m), layer, a, b, _at(lse, "lse"), _int32(users, "users"),
                                     _int32(q_start, "q_start", n_seqs + 1), _views(views, n, max_q), n_seqs, n, max_q,
                                     1.0 / math.sqrt(hd) if scale is None else scale, window, _at(workspace, "the workspace"),
                                     workspace.numel() * workspace.element_size(), _int32(status, "status", 1), cuda_stream),
           "kfl_kv4_attend_tree")


# ---- rows that leave the cache -------------------------------------------------------------------

def _mass(mass, p, m):
    """kfl_kv4_mass of a tensor [layer][user][KV head][slot] whose slots are neighbours and whose rows do not overlap."""
    if mass is None:
        return None
    shape = mass.shape
    if mass.dtype != torch.float32 or len(shape) != 4 or shape[0] != p.n_layers or shape[1] < m.n_users \
            or shape[2] != p.n_kv_heads or shape[3] < m.max_pages * p.page_tokens:
        raise ValueError("mass is fp32 [layer][user][KV head][slot] of "
                         f"{[p.n_layers, m.n_users, p.n_kv_heads, m.max_pages * p.page_tokens]}")
    a, b, c, one = mass.stride()
    if one != 1 or c < shape[3] or b < c * shape[2] or a < b * shape[1]:  # not in this order, with room between
        span = 1
        for size, stride in sorted(zip(shape, (a, b, c, one)), key=lambda v: v[1]):
            if size > 1 and stride < span:
                raise ValueError("the rows of mass do not overlap")
            span += (size - 1) * stride
        if one != 1:
            raise ValueError("the slots of mass are neighbours")
    return _pack_mass(_at(mass, "mass"), a, b, c)


def kfl_kv4_weights(p, m, layer: int, q, lse, mass, workspace, users=None, q_start=None, max_q: int = 1, scale=None,
                    window: int = 0, status=None, cuda_stream: int | None = None) -> None:
    """Adds to mass (fp32 [layer][user][KV head][slot]) of one layer the weight that q's rows give every cached row, with the
    lse that kfl_kv4_attend or kfl_kv4_attend_tree wrote for them; the other arguments as theirs.  Asynchronous."""
    n, _, hd = q.shape
    n_seqs = _sequences(m, q, users, q_start, lse, workspace)
    a = _heads(q, "q", n, p.head_dim)
    _check(lib().kfl_kv4_weights(_handle(p), _handle(m), layer, a, _at(lse, "lse"), _mass(mass, p, m), _int32(users, "users"),
                                 _int32(q_start, "q_start", n_seqs + 1), n_seqs, n, max_q,
                                 1.0 / math.sqrt(hd) if scale is None else scale, window, _at(workspace, "the workspace"),
                                 workspace.numel() * workspace.element_size(), _int32(status, "status", 1), cuda_stream),
           "kfl_kv4_weights")


def kfl_kv4_select(p, m, mass, users, budget: int, rows, counts, first: int = 0, recent: int = 0, status=None,
                   cuda_stream: int | None = None) -> None:
    """The rows that stay of the users (int32) cut to `budget`: the first, the most recent, and of the others those with the
    greatest mass; slots into rows (int32 [layer][user of the list][KV head][budget], -1 behind the last), how many into
    counts (int32 [user of the list]).  Asynchronous."""
    n = users.numel()
    if tuple(rows.shape) != (p.n_layers, n, p.n_kv_heads, budget):
        raise ValueError(f"rows is int32 [layer][user of the list][KV head][budget], {[p.n_layers, n, p.n_kv_heads, budget]}")
    _check(lib().kfl_kv4_select(_handle(p), _handle(m), _mass(mass, p, m), _int32(users, "users"), n, budget, first, recent,
                                _int32(rows, "rows"), _int32(counts, "counts", n), _int32(status, "status", 1), cuda_stream),
           "kfl_kv4_select")


def kfl_kv4_keep(p, m, users, rows, counts, workspace, first=None, mass=None, status=None,
                 cuda_stream: int | None = None) -> None:
    """Cuts the users (int32) to their rows below first (int32 [user of the list], None: 0) and the counts (int32) rows of
    their lists: rows is int32 [layer][user of the list][KV head][most], of any strides whose last is 1 (expanded where
    layers or heads are alike).  mass moves with the rows.  Asynchronous."""
    n = users.numel()
    shape, strides = rows.shape, rows.stride()
    if rows.dtype != torch.int32 or len(shape) != 4 or shape[0] != p.n_layers or shape[1] != n or shape[2] != p.n_kv_heads \
            or strides[3] != 1 and shape[3] > 1:
        raise ValueError(f"rows is int32 [layer][user of the list][KV head][most], {[p.n_layers, n, p.n_kv_heads]}, its last stride 1")
    a, b = _covers(p, m)
    r = _pack_rows(_at(rows, "rows"), strides[0], strides[1], strides[2], shape[3])
    _check(lib().kfl_kv4_keep(a, b, _int32(users, "users"), r, _int32(first, "first", n), _int32(counts, "counts", n),
                              _mass(mass, p, m), n, _scratch(p, workspace), _int32(status, "status", 1), cuda_stream),
           "kfl_kv4_keep")


# ---- pages ---------------------------------------------------------------------------------------

def kfl_kv4_pages_workspace_bytes(p) -> int:
    out = C.c_size_t(0)
    _check(lib().kfl_kv4_pages_workspace_bytes(C.byref(p), C.byref(out)), "kfl_kv4_pages_workspace_bytes")
    return out.value


def pages_workspace(p):
    """Scratch of the calls that hand out or move pages."""
    return torch.empty(kfl_kv4_pages_workspace_bytes(p), dtype=torch.uint8, device="cuda")


def _scratch(p, workspace):
    """Address of a workspace that covers the pool's pages: as many bytes as the library asks for, which the pool's
    description keeps for the next call's check."""
    n_pages, need = getattr(p, "scratch", (None, 0))
    if n_pages != p.n_pages:
        need = kfl_kv4_pages_workspace_bytes(p)
        p.scratch = (p.n_pages, need)
    if not workspace.is_contiguous() or workspace.numel() * workspace.element_size() < need:
        raise ValueError(f"the workspace is one of pages_workspace for this pool ({need} bytes)")
    return _at(workspace, "the workspace")


def kfl_kv4_reserve(p, m, users, n_new, workspace, status=None, cuda_stream: int | None = None) -> None:
    """Room for n_new[i] more tokens of user users[i] (int32): pages and lengths.  Asynchronous."""
    n = users.numel()
    a, b = _covers(p, m)
    _check(lib().kfl_kv4_reserve(a, b, _int32(users, "users"), _int32(n_new, "n_new", n), n, _scratch(p, workspace),
                                 _int32(status, "status", 1), cuda_stream), "kfl_kv4_reserve")


def kfl_kv4_fork(p, m, src, dst, workspace, status=None, cuda_stream: int | None = None) -> None:
    """User dst[i] goes on from where src[i] is (int32), all at once.  Asynchronous."""
    n = dst.numel()
    a, b = _covers(p, m)
    _check(lib().kfl_kv4_fork(a, b, _int32(src, "src", n), _int32(dst, "dst"), n, _scratch(p, workspace),
                              _int32(status, "status", 1), cuda_stream), "kfl_kv4_fork")


def kfl_kv4_free(p, m, users, status=None, cuda_stream: int | None = None) -> None:
    """Gives back the pages of the users (int32).  Asynchronous."""
    a, b = _covers(p, m)
    _check(lib().kfl_kv4_free(a, b, _int32(users, "users"), users.numel(), _int32(status, "status", 1), cuda_stream),
           "kfl_kv4_free")


def kfl_kv4_compact(p, m, table_out, refs_out, n_live, workspace, status=None, cuda_stream: int | None = None) -> None:
    """Live pages to the lowest numbers; the new table and references into table_out and refs_out (the map's own
    tensors or others), the number of live pages into n_live (int32, may be None).  Asynchronous."""
    a, b = _covers(p, m)
    _check(lib().kfl_kv4_compact(a, b, _int32(table_out, "table_out", m.n_users * m.max_pages),
                                 _int32(refs_out, "refs_out", p.n_pages), _int32(n_live, "n_live", 1),
                                 _scratch(p, workspace), _int32(status, "status", 1), cuda_stream), "kfl_kv4_compact")


def kfl_kv4_copy_pages(p, src, dst, status=None, cuda_stream: int | None = None) -> None:
    """Copies page src[i] to page dst[i] (int32).  Asynchronous."""
    n = src.numel()
    _check(lib().kfl_kv4_copy_pages(_handle(p), _int32(src, "src"), _int32(dst, "dst", n), n,
                                    _int32(status, "status", 1), cuda_stream), "kfl_kv4_copy_pages")
