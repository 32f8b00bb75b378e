"""Operators for drafted trees and for full caches, over the 4-bit paged KV cache, as cases that can be
timed and compared.

A case is one pass through an operator as a serving loop calls it:

* ``tree``: what a step has to know of its users' trees of drafted tokens: which nodes each node sees,
  and its position;
* ``attend``: attention of the nodes over the users' cached rows and their own ancestors;
* ``weights``: the attention weight that every cached row got in a pass, added to what it had;
* ``select``: the rows that stay of a cache that is cut to a budget: the first, the last, and those with
  the greatest weight so far;
* ``keep``: the rows of a list brought together in place, the pages behind them given back, and room
  for the next rows reserved (accepted drafts, or a cache that has been cut).

``run`` computes a pass in plain torch in 32 bits, or with ``own`` set calls the library.  ``exact``
recomputes the floating outputs in 64 bits.

The page layout that both share.  A pool is ``[pages][layers][KV heads]`` blocks; a block holds
``page`` tokens of one head: K codes ``[token][head_dim / 2]`` bytes, V codes, K parameters
``[token][head_dim / 64]`` pairs of fp16 (scale, centre), V parameters.  A byte holds two channels,
the even one in its low half.  A value is ``centre + (code - 8) * scale``.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
GROUP = 64  # channels that share a scale and a centre


def _tree(name, tokens, spread):
    return {"name": name, "op": "tree", "tokens": _text(tokens), "spread": spread}


def _attend(name, lengths, tokens, spread, q_heads, kv_heads, head_dim, dtype, page, window=0, layers=1):
    return {"name": name, "op": "attend", "lengths": _text(lengths), "tokens": _text(tokens), "spread": spread,
            "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype, "page": page,
            "window": window, "layers": layers}


def _weights(name, lengths, tokens, q_heads, kv_heads, head_dim, dtype, page, window=0, layers=1):
    return {"name": name, "op": "weights", "lengths": _text(lengths), "tokens": _text(tokens), "q_heads": q_heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype, "page": page, "window": window,
            "layers": layers}


def _select(name, lengths, layers, kv_heads, budget, first, recent, page):
    return {"name": name, "op": "select", "lengths": _text(lengths), "layers": layers, "kv_heads": kv_heads,
            "budget": budget, "first": first, "recent": recent, "page": page, "head_dim": 64}


def _keep(name, lengths, kept, tokens, layers, kv_heads, head_dim, page, per_head, shared=0):
    """tokens: how many rows at each user's end are in question (all of them: 0), kept: how many of those stay."""
    return {"name": name, "op": "keep", "lengths": _text(lengths), "kept": _text(kept), "tokens": _text(tokens),
            "layers": layers, "kv_heads": kv_heads, "head_dim": head_dim, "page": page, "per_head": per_head,
            "shared": shared}


def _text(values):
    return ",".join(str(int(v)) for v in values)


def _list(text):
    return [int(v) for v in text.split(",")]


RAGGED_32 = [8192 - 251 * i for i in range(32)]


def listed():
    return [
        # four users' small trees of one step: nothing but latency
        _tree("tree-b4x8", [8, 8, 6, 7], 3),
        # a full house: 64 users' trees of up to 128 nodes, long chains among them
        _tree("tree-b64x128", [128 - i for i in range(64)], 6),
        # the tiny model's user with a handful of drafts: the smallest tree there is to check
        _attend("attend-tiny-b1x5", [141], [5], 2, 8, 2, 64, "bf16", 16),
        # a few drafts for each of 32 users at ragged contexts: the cache streams from HBM
        _attend("attend-b32x4-ragged", RAGGED_32, [4] * 32, 3, 28, 4, 128, "bf16", 64),
        # wide trees of eight users at long contexts: matrix products
        _attend("attend-b8x63-8192", [8192 + 63] * 8, [63] * 8, 12, 64, 8, 128, "bf16", 64),
        # a decode step of 32 users at ragged contexts: what each cached row was looked at
        _weights("weights-step-b32-ragged", RAGGED_32, [1] * 32, 64, 8, 128, "bf16", 64),
        # a prompt's last 2048 tokens over 8192
        _weights("weights-prompt-2048-at-6144", [8192], [2048], 64, 8, 128, "bf16", 64),
        # one user of a small model over its budget
        _select("select-b1-4096-to-1024", [4096], 1, 4, 1024, 4, 64, 64),
        # the users of a 7B-shaped stage at once, down to a quarter
        _select("select-b16-8192-to-2048", [8192 - 131 * i for i in range(16)], 14, 4, 2048, 4, 256, 64),
        # one user at a very long context: few rows to choose in, all of them long
        _select("select-b1-131072-to-16384", [131072], 1, 8, 16384, 4, 1024, 64),
        # accepted paths of four users' trees of 16 drafts, and room for the next trees
        _keep("keep-accept-b4x16", [3000, 512, 1777, 2305], [5, 1, 3, 4], [16, 16, 16, 16], 14, 4, 128, 32, False),
        # eight users of a 7B-shaped stage cut to half, each layer and head to rows of its own
        _keep("keep-evict-b8-8192-to-4096", [8192 - 61 * i for i in range(8)], [4096] * 8, [0] * 8, 14, 4, 128, 64, True,
              shared=2),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Another case of the same ranges: 1 to 64 users, 1 to 131072 cached rows, trees of 1 to 128 nodes, one
    token to 2048, heads of 64 and 128 in groups of 1 to 12, pages of 16 to 128 tokens, both types, windows."""
    op = rng.choice(["tree", "attend", "attend", "attend", "weights", "weights", "weights", "select", "select", "keep",
                     "keep"])
    head_dim = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 3, 4, 5, 7, 8, 8, 12])
    page = rng.choice([16, 32, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "fp16"])
    window = rng.choice([0, 0, 0, _log_int(rng, 1, 4096)])
    if op == "tree":
        n = _log_int(rng, 1, 63)
        c = _tree("", [_log_int(rng, 1, 90) for _ in range(n)], rng.randint(1, 12))
    elif op == "attend":
        n = _log_int(rng, 1, 16)
        tokens = [_log_int(rng, 1, max(2, 128 // n)) for _ in range(n)]
        long = 12 if max(tokens) <= 8 else 1  # (short trees also over the longest contexts)
        lengths = [t + _log_int(rng, 1, min(131000, long * 10000 // n)) - 1 for t in tokens]
        c = _attend("", lengths, tokens, rng.randint(1, 12), kv_heads * group, kv_heads, head_dim, dtype, page, window)
    elif op == "weights":
        if rng.random() < 0.6:
            n = _log_int(rng, 1, 64)
            tokens = [1] * n if rng.random() < 0.6 else [rng.randint(1, 12) for _ in range(n)]
            lengths = [t + _log_int(rng, 1, min(131000, 130000 // n)) - 1 for t in tokens]
        else:
            n = rng.randint(1, 3)
            tokens = [_log_int(rng, 13, 2048 // n) for _ in range(n)]
            lengths = [t + _log_int(rng, 1, 6000 // n) - 1 for t in tokens]
            group = min(group, 8)
        c = _weights("", lengths, tokens, kv_heads * group, kv_heads, head_dim, dtype, page, window)
    elif op == "select":
        n = _log_int(rng, 1, 16)
        layers = _log_int(rng, 1, 14)
        lengths = [_log_int(rng, 1, max(2, min(131072, 900000 // (n * layers * kv_heads)))) for _ in range(n)]
        budget = _log_int(rng, 1, max(lengths))
        first = rng.randint(0, min(8, budget))
        c = _select("", lengths, layers, kv_heads, budget, first, rng.randint(0, budget - first), page)
    else:
        n = _log_int(rng, 1, 16)
        layers = _log_int(rng, 1, 14)
        if rng.random() < 0.5:
            tokens = [_log_int(rng, 1, 64) for _ in range(n)]
            kept = [rng.randint(1, min(t, 12)) for t in tokens]
            lengths = [t + _log_int(rng, 1, 4000) - 1 for t in tokens]
            c = _keep("", lengths, kept, tokens, layers, kv_heads, head_dim, page, False, rng.choice([0, 0, 1, n // 2]))
        else:
            lengths = [_log_int(rng, 1, 60000 // n) for _ in range(n)]
            kept = [rng.randint(1, v) for v in lengths]
            c = _keep("", lengths, kept, [0] * n, layers, kv_heads, head_dim, page, rng.random() < 0.7,
                      rng.choice([0, 0, 1, n // 2]))
    del c["name"]
    return c


# ------------------------------------------------------------------------------------- inputs

def _gen(seed, *tag):
    key = seed & 0xFFFFFFFF
    for t in tag:
        key = (key * 1000003 + t + 1) & 0x3FFFFFFFFFFFFFF
    return torch.Generator(device="cuda").manual_seed(key)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _block_bytes(case):
    return case["page"] * case["head_dim"] // 8 * 9


def _starts(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def _parents(counts, spread, seed):
    """Trees in the order in which they were drafted: a node hangs on one of the `spread` before it, the first on the
    last cached token, and now and then another one too."""
    rng = random.Random(seed * 7919 + 13)
    return [rng.randint(max(-1, i - spread), i - 1) if i else -1 for c in counts for i in range(c)]


def _tables(lengths, page, n_pages, spare, g, shared=0):
    """Every user's pages, scattered over the pool, and how many users hold each.  Users 1 to `shared` hold the full
    pages of user 0 as far as their own go: they went on from it."""
    need = [-(-n // page) for n in lengths]
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    table = torch.full((len(lengths), max(need) + spare), -1, dtype=torch.int32, device="cuda")
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        common = min(lengths[0] // page, lengths[i] // page) if 0 < i <= shared else 0
        table[i, :common] = table[0, :common]
        table[i, common:n] = order[at:at + n - common]
        at += n - common
    held = table[table >= 0].long()
    refs.index_add_(0, held, torch.ones_like(held, dtype=torch.int32))
    return table, refs


def prepare(case, seed):
    g = _gen(seed, 11)
    op = case["op"]
    s = {"case": dict(case)}
    if op == "tree":
        tokens = _list(case["tokens"])
        s["parents"], s["q_start"] = _int32(_parents(tokens, case["spread"], seed)), _int32(_starts(tokens))
        s["first"] = torch.randint(0, 100000, (len(tokens),), dtype=torch.int32, generator=g, device="cuda")
        s["max_q"] = max(tokens)
        s["views"] = torch.empty(sum(tokens), -(-s["max_q"] // 32), dtype=torch.int32, device="cuda")
        s["positions"] = torch.empty(sum(tokens), dtype=torch.int32, device="cuda")
    elif op in ("attend", "weights"):
        lengths, tokens = _list(case["lengths"]), _list(case["tokens"])
        n_pages = sum(-(-v // case["page"]) for v in lengths) + 3
        s["table"], s["refs"] = _tables(lengths, case["page"], n_pages, 1, g)
        s["lengths"] = _int32(lengths)
        s["pool"] = _filled_pool(case, n_pages, s["table"], s["lengths"], g)
        x = torch.randn(sum(tokens), case["q_heads"], case["head_dim"], generator=g, device="cuda")
        s["q"] = x.to(DTYPES[case["dtype"]])
        s["q_start"] = None if max(tokens) == min(tokens) == 1 else _int32(_starts(tokens))
        s["max_q"], s["max_len"] = max(tokens), max(lengths)
        if op == "attend":
            s["out"] = torch.empty_like(s["q"])
            parents = _int32(_parents(tokens, case["spread"], seed))
            starts = _int32(_starts(tokens))
            s["views"] = _tree_views(parents, starts, s["max_q"])[0]
        else:
            # what attention left of its softmax, and the weights that the rows have had so far
            s["lse"] = _scores_lse(s)
            shape = (case["layers"], len(lengths), case["kv_heads"], s["table"].shape[1] * case["page"])
            # (a few such passes' worth, most of it on few rows)
            s["mass"] = torch.rand(shape, generator=g, device="cuda").pow_(6)
            s["mass"] *= 20 * case["q_heads"] / case["kv_heads"] * sum(tokens) / sum(lengths)
            s["mass"] *= torch.arange(shape[3], device="cuda") < s["lengths"][:, None, None]
    elif op == "select":
        lengths = _list(case["lengths"])
        page = case["page"]
        s["table"], s["refs"] = _tables(lengths, page, sum(-(-v // page) for v in lengths) + 1, 1, g)
        s["lengths"] = _int32(lengths)
        s["users"] = torch.randperm(len(lengths), generator=g, device="cuda").int()
        shape = (case["layers"], len(lengths), case["kv_heads"], s["table"].shape[1] * page)
        # a few rows with most of the weight, many with next to none, some that nothing has looked at: equal
        s["mass"] = torch.randn(shape, generator=g, device="cuda").mul_(3).exp_()
        s["mass"] *= torch.rand(shape, generator=g, device="cuda") > 0.05
        s["rows"] = torch.empty(case["layers"], len(lengths), case["kv_heads"], case["budget"], dtype=torch.int32,
                                device="cuda")
        s["counts"] = torch.empty(len(lengths), dtype=torch.int32, device="cuda")
    else:
        lengths, kept, tokens = (_list(case[n]) for n in ("lengths", "kept", "tokens"))
        page, n = case["page"], len(lengths)
        need = sum(-(-v // page) for v in lengths)
        s["table"], s["refs"] = _tables(lengths, page, 2 * need + 5, 1, g, case["shared"])
        s["lengths"] = _int32(lengths)
        shape = (2 * need + 5, case["layers"], case["kv_heads"], _block_bytes(case))
        s["pool"] = torch.randint(0, 256, shape, dtype=torch.uint8, generator=g, device="cuda")
        s["users"] = torch.randperm(n, generator=g, device="cuda").int()
        order = s["users"].tolist()
        lists = (case["layers"] if case["per_head"] else 1, n, case["kv_heads"] if case["per_head"] else 1)
        s["rows"] = torch.full(lists + (max(kept),), -1, dtype=torch.int32, device="cuda")
        for i, u in enumerate(order):
            m = tokens[u] or lengths[u]
            pick = torch.rand(lists[0], lists[2], m, generator=g, device="cuda").argsort(-1)[..., :kept[u]]
            s["rows"][:, i, :, :kept[u]] = (pick.sort(-1).values + lengths[u] - m).int()
        s["rows"] = s["rows"].expand(case["layers"], n, case["kv_heads"], max(kept))
        s["first"] = _int32([lengths[u] - (tokens[u] or lengths[u]) for u in order])
        s["counts"] = _int32([kept[u] for u in order])
        s["n_new"] = _int32([(tokens[u] or lengths[u]) - kept[u] for u in order])
        s["mass"] = torch.rand(case["layers"], n, case["kv_heads"], s["table"].shape[1] * page, generator=g,
                               device="cuda")
        s["mass"] *= torch.arange(s["mass"].shape[3], device="cuda") < s["lengths"][:, None, None]
        s["max_len"] = max(lengths)
    if own:
        _handles(s)
    return s


def _filled_pool(case, n_pages, table, lengths, g):
    """A pool whose cached tokens hold quantised normal values, and whose other slots were never written."""
    page, hd, h = case["page"], case["head_dim"], case["kv_heads"]
    pool = torch.full((n_pages, case["layers"], h, _block_bytes(case)), 255, dtype=torch.uint8, device="cuda")
    outlier = 4 * (torch.rand(h, 1, hd, generator=g, device="cuda") < 0.05).float()
    kv = [torch.empty(n_pages, h, page, hd // 2, dtype=torch.uint8, device="cuda") for _ in range(2)]
    pv = [torch.empty(n_pages, h, page, hd // GROUP, 2, dtype=torch.float16, device="cuda") for _ in range(2)]
    for a in range(0, n_pages, 512):  # (a slab at a time: 32-bit values take seven times the pages' bytes)
        b = min(n_pages, a + 512)
        for i in range(2):
            x = torch.randn(b - a, h, page, hd, generator=g, device="cuda") + (outlier if i == 0 else 0)
            kv[i][a:b], pv[i][a:b] = _quantise(x)
    # slots behind a user's last token: parameters of a memory that nobody has written
    slot = torch.arange(table.shape[1] * page, device="cuda").view(table.shape[1], page)
    unused = (slot >= lengths[:, None, None]) & (table >= 0)[:, :, None]
    at = unused.nonzero()
    for i in range(2):
        pv[i][table[at[:, 0], at[:, 1]].long(), :, at[:, 2]] = float("nan")
    parts = _parts(pool, case)
    l = case["layers"] - 1
    for i in range(2):
        parts[i][:, l] = kv[i]
        parts[2 + i][:, l] = pv[i]
    return pool


def _scores_lse(s):
    """The log of the sum of exp(scores) of every row, as the pass's attention gives it: [token][query head]."""
    case = s["case"]
    n, h = len(_list(case["lengths"])), case["kv_heads"]
    group = case["q_heads"] // h
    out = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda")
    token, user, i = _rows_of(s)
    for head in range(h):
        p = _head_scores(s, head)  # user, [token, group], key
        lse = p.logsumexp(-1).view(n, s["max_q"], group)
        out[:, head * group:(head + 1) * group] = lse[user, i]
    return out


# ------------------------------------------------------------------- the operators in plain torch

def _parts(pool, case):
    """K codes, V codes, K parameters and V parameters of a pool, as views."""
    page, hd = case["page"], case["head_dim"]
    n, m = page * hd // 2, page * hd // 16
    codes = [pool[..., i * n:(i + 1) * n].unflatten(-1, (page, hd // 2)) for i in range(2)]
    params = [pool[..., 2 * n + i * m:2 * n + (i + 1) * m].view(torch.float16).unflatten(-1, (page, hd // GROUP, 2))
              for i in range(2)]
    return codes + params


def _quantise(x):
    """Codes (two channels a byte) and parameters of fp32 rows [..., head_dim]."""
    x = x.unflatten(-1, (-1, GROUP))
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    scale = ((hi - lo) / torch.full_like(hi, 15.0)).half()
    centre = (lo + 8 * scale.float()).half()
    inv = torch.where(scale > 0, 1 / scale.float(), 0.0)
    u = (((x - centre.float()) * inv).round() + 8).clamp(0, 15).to(torch.uint8).flatten(-2)
    return u[..., 0::2] | (u[..., 1::2] << 4), torch.cat([scale, centre], -1)


def _values(codes, params):
    u = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float() - 8
    p = params.float()
    return (u.unflatten(-1, (-1, GROUP)) * p[..., :1] + p[..., 1:]).flatten(-2)


def _rows_of(s):
    """Each row's number, user, and place among the user's."""
    n = len(_list(s["case"]["lengths"] if "lengths" in s["case"] else s["case"]["tokens"]))
    device = s["parents"].device if "parents" in s else s["q"].device
    start = torch.arange(n + 1, device=device) if s["q_start"] is None else s["q_start"].long()
    total = s["parents"].shape[0] if "parents" in s else s["q"].shape[0]
    token = torch.arange(total, device=device)
    user = torch.searchsorted(start, token, right=True) - 1
    return token, user, token - start[user]


def _ancestors(parents, start, m):
    """Who sees whom, [user][node][node] as 0 and 1: ancestors by doubling of the steps upwards."""
    row = torch.arange(m, device=parents.device)
    count = (start[1:] - start[:-1]).long()
    at = (start[:-1, None].long() + row).clamp(max=parents.numel() - 1)
    up = torch.where(row < count[:, None], parents.long()[at], -1)
    seen = torch.eye(m, device=parents.device) + (up[..., None] == row)
    steps = 1
    while steps < m:
        seen = (torch.matmul(seen, seen) > 0).float()
        steps *= 2
    return seen * (row < count[:, None])[..., None]


def _tree_views(parents, start, m):
    """The views as bits, 32 nodes a word, and how many nodes each node sees."""
    seen = _ancestors(parents, start, m)
    words = -(-m // 32)
    bits = torch.zeros(*seen.shape[:2], words * 32, dtype=torch.int64, device=parents.device)
    bits[..., :m] = seen.long()
    weight = torch.tensor([1 << i if i < 31 else -(1 << 31) for i in range(32)], device=parents.device)
    packed = (bits.view(*seen.shape[:2], words, 32) * weight).sum(-1).int()
    token = torch.arange(parents.numel(), device=parents.device)
    user = torch.searchsorted(start.long(), token, right=True) - 1
    at = token - start.long()[user]
    return packed[user, at], seen.sum(-1).int()[user, at], user


def _plain_tree(s):
    views, n, user = _tree_views(s["parents"], s["q_start"], s["max_q"])
    return {"views": views, "positions": s["first"][user] + n - 1}


def _cached(s, i):
    """32-bit K (i = 0) or V (1) of every user, [user][KV head][key][channel], 0 where nothing is cached."""
    case = s["case"]
    page, layer = case["page"], case["layers"] - 1
    parts = _parts(s["pool"], case)
    pages = s["table"][:, :-(-s["max_len"] // page)].long().clamp(min=0)
    key = torch.arange(pages.shape[1] * page, device=pages.device)
    there = (key < s["lengths"][:, None])[:, None, :, None]
    return torch.where(there, _values(parts[i][pages, layer], parts[2 + i][pages, layer]).transpose(1, 2).flatten(2, 3), 0.0)


def _padded_queries(s):
    """32-bit q as [user][KV head][token, group][channel], and each user's first row."""
    case, q = s["case"], s["q"]
    n, h, m = len(s["lengths"]), case["kv_heads"], s["max_q"]
    group = case["q_heads"] // h
    start = torch.arange(n + 1, device=q.device) if s["q_start"] is None else s["q_start"].long()
    at = (start[:-1, None] + torch.arange(m, device=q.device)).clamp(max=q.shape[0] - 1)
    return q.float()[at].view(n, m, h, group, case["head_dim"]).transpose(1, 2).flatten(2, 3), start


def _causal(s, keys):
    """Who sees which key, [user][token][key], and which tokens there are."""
    case, m = s["case"], s["max_q"]
    lengths = s["lengths"].long()
    start = torch.arange(len(lengths) + 1, device=lengths.device) if s["q_start"] is None else s["q_start"].long()
    count = start[1:] - start[:-1]
    row, key = torch.arange(m, device=lengths.device), torch.arange(keys, device=lengths.device)
    pos = ((lengths - count)[:, None] + row)[..., None]
    seen = (key <= pos) & (key < lengths[:, None, None])
    if case["window"]:
        seen &= key > pos - case["window"]
    return seen & (row < count[:, None])[..., None]


def _head_scores(s, head):
    """One KV head's scores, [user][token, group][key], -inf where nothing is seen."""
    case = s["case"]
    page, layer = case["page"], case["layers"] - 1
    parts = _parts(s["pool"], case)
    pages = s["table"][:, :-(-s["max_len"] // page)].long().clamp(min=0)
    k = _values(parts[0][pages, layer, head], parts[2][pages, layer, head]).flatten(1, 2)
    k = torch.where((torch.arange(k.shape[1], device=k.device) < s["lengths"][:, None])[..., None], k, 0.0)
    x = _padded_queries(s)[0][:, head]
    p = torch.matmul(x, k.transpose(-1, -2)) * (1 / math.sqrt(case["head_dim"]))
    group = case["q_heads"] // case["kv_heads"]
    seen = _causal(s, k.shape[1])[:, :, None, :].expand(-1, -1, group, -1).flatten(1, 2)
    return p.masked_fill_(~seen, -math.inf)


def _plain_attend(s):
    case = s["case"]
    hd, h, q, m = case["head_dim"], case["kv_heads"], s["q"], s["max_q"]
    n, group, lengths = len(s["lengths"]), case["q_heads"] // case["kv_heads"], s["lengths"].long()
    kv = [_cached(s, i) for i in range(2)]
    x, start = _padded_queries(s)
    p = torch.matmul(x, kv[0].transpose(-1, -2)) * (1 / math.sqrt(hd))
    # the context, as far as the window's rest, and the nodes of the view
    keys = p.shape[-1]
    key, row = torch.arange(keys, device=q.device), torch.arange(m, device=q.device)
    base = lengths - (start[1:] - start[:-1])
    node = key - base[:, None]  # user, key
    at = (start[:-1, None] + row).clamp(max=q.shape[0] - 1)
    words = s["views"].long()[at]  # user, token, word
    bit = words.gather(2, (node.clamp(0, m - 1) >> 5)[:, None, :].expand(-1, m, -1)) >> (node.clamp(0, m - 1) & 31)[:, None, :]
    seen = torch.where((node < 0)[:, None], True, (bit & 1 != 0) & (node < m)[:, None] & (key < lengths[:, None])[:, None])
    if case["window"]:
        shifts = torch.arange(32, device=q.device)
        nodes = (words[..., None] >> shifts & 1).sum((-1, -2))
        begin = base[:, None] - (case["window"] - nodes).clamp(min=0)
        seen &= (node >= 0)[:, None] | (key >= begin[..., None])
    seen = seen[:, None, :, None, :].expand(n, 1, m, group, keys).flatten(2, 3)
    p = p.masked_fill_(~seen, -math.inf)
    top = p.amax(-1, keepdim=True)
    p = p.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, kv[1]) / torch.where(total == 0, 1.0, total)
    o = o.view(n, h, m, group, hd).transpose(1, 2).reshape(n, m, h * group, hd)
    token, user, i = _rows_of(s)
    return {"out": o[user, i].to(q.dtype)}


def _plain_weights(s):
    case = s["case"]
    h, m, n = case["kv_heads"], s["max_q"], len(s["lengths"])
    group = case["q_heads"] // h
    x, start = _padded_queries(s)
    p = torch.matmul(x, _cached(s, 0).transpose(-1, -2)) * (1 / math.sqrt(case["head_dim"]))
    keys = p.shape[-1]
    at = (start[:-1, None] + torch.arange(m, device=x.device)).clamp(max=s["q"].shape[0] - 1)
    lse = s["lse"][at].view(n, m, h, group).transpose(1, 2).flatten(2, 3)
    seen = _causal(s, keys)[:, None, :, None, :].expand(n, 1, m, group, keys).flatten(2, 3)
    p = p.sub_(lse[..., None]).exp_().masked_fill_(~seen, 0.0).sum(2)
    mass = s["mass"][case["layers"] - 1]
    mass[..., :keys] += p
    return {"mass": s["mass"]}


def _plain_select(s):
    case = s["case"]
    users, lengths = s["users"].long(), s["lengths"][s["users"].long()].long()
    budget, device = case["budget"], users.device
    mass = s["mass"][:, users]  # layer, user, head, row
    row = torch.arange(mass.shape[3], device=device)
    n = lengths[:, None, None]
    kept = (row < case["first"]) | (row >= n - case["recent"])
    rank = torch.where(row >= n, -1.0, torch.where(kept, math.inf, mass))
    pick = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :budget]
    if pick.shape[-1] < budget:
        pick = torch.cat([pick, torch.full((*pick.shape[:-1], budget - pick.shape[-1]), mass.shape[3], device=device)], -1)
    pick = torch.where(pick < n, pick, 1 << 30).sort(-1).values
    return {"rows": torch.where(pick < 1 << 30, pick, -1).int(), "counts": lengths.clamp(max=budget).int()}


def _lowest_free(refs, count):
    return torch.argsort((refs != 0).to(torch.uint8), stable=True)[:count]


def _plain_keep(s):
    case = s["case"]
    page, table, refs, lengths = case["page"], s["table"], s["refs"], s["lengths"]
    users, first, counts = s["users"].long(), s["first"].long(), s["counts"].long()
    n_old = lengths[users].long()
    n_new = first + counts
    changes = n_new < n_old
    begin, need, held = first // page, (n_new + page - 1) // page, (n_old + page - 1) // page
    column = torch.arange(table.shape[1], device=table.device)
    old = table[users]
    # pages that rows move into and that others hold too: new ones
    moved = (column >= begin[:, None]) & (column < need[:, None]) & changes[:, None]
    fresh = moved & (refs[old.clamp(min=0).long()] > 1)
    free = _lowest_free(refs, fresh.numel())
    rank = (fresh.flatten().long().cumsum(0) - 1).clamp(0, free.numel() - 1).view(fresh.shape)
    new = torch.where(fresh, free[rank].int(), torch.where(changes[:, None] & (column >= need[:, None]), -1, old))
    # the rows, from the first moved page's start on (what stands before the first one goes along into a new page)
    most = s["max_len"]
    place = begin[:, None] * page + torch.arange(most, device=table.device)  # user, j
    there = (place < n_new[:, None]) & changes[:, None]
    j = (place - first[:, None]).clamp(0, s["rows"].shape[3] - 1)
    layers, n, heads = s["rows"].shape[:3]
    row = s["rows"].long().gather(3, j[None, :, None].expand(layers, n, heads, most))
    row = torch.where((place < first[:, None])[None, :, None], place[None, :, None], row)
    l, i, h, t = torch.nonzero(there[None, :, None].expand(layers, n, heads, most), as_tuple=True)
    source, place = row[l, i, h, t], place[i, t]
    from_page, to_page = old[i, source // page].long(), new[i, place // page].long()
    for part in _parts(s["pool"], case):
        part[to_page, l, h, place % page] = part[from_page, l, h, source % page]
    s["mass"][l, users[i], h, place] = s["mass"][l, users[i], h, source]
    key = torch.arange(s["mass"].shape[3], device=table.device)
    gone = (key >= n_new[:, None]) & changes[:, None]
    s["mass"][:, users] = torch.where(gone[None, :, None], 0.0, s["mass"][:, users])
    for pages, by in ((torch.where(old != new, old, -1), -1), (torch.where(old != new, new, -1), 1)):
        refs.index_add_(0, pages.clamp(min=0).flatten().long(), ((pages >= 0) * by).flatten().int())
    # room for the next rows
    held = need
    total = (n_new + s["n_new"].long() + page - 1) // page
    wanted = (column >= held[:, None]) & (column < total[:, None])
    free = _lowest_free(refs, wanted.numel())
    rank = (wanted.flatten().long().cumsum(0) - 1).clamp(0, free.numel() - 1).view(wanted.shape)
    rows = torch.where(wanted, free[rank].int(), new)
    refs.index_add_(0, torch.where(wanted, rows, 0).flatten().long(), wanted.flatten().int())
    table[users] = rows
    lengths[users] = (n_new + s["n_new"].long()).int()
    return {"table": table, "refs": refs, "lengths": lengths, "pool": s["pool"], "mass": s["mass"]}


# ------------------------------------------------------------------------------ the library's calls

def _handles(s):
    """What a program keeps beside its buffers: the descriptions of pool and tables, and the workspaces."""
    from paper_2609_34045_gb300 import kv4

    s["lib"], case = kv4, s["case"]
    if case["op"] == "tree":
        return
    if "pool" in s:
        s["pages"] = kv4.pool(s["pool"], case["page"], case["layers"], case["kv_heads"], case["head_dim"])
    else:
        s["pages"] = kv4.pool(None, case["page"], case["layers"], case["kv_heads"], case["head_dim"],
                              n_pages=s["refs"].numel())
    s["map"] = kv4.page_map(s["table"], s["lengths"], s["refs"])
    if case["op"] in ("attend", "weights"):
        s["workspace"] = kv4.attend_workspace(s["pages"], case["q_heads"], len(_list(case["lengths"])),
                                              s["q"].shape[0], s["max_q"])
    elif case["op"] == "keep":
        s["workspace"] = kv4.pages_workspace(s["pages"])


def _own(s):
    kv4, case = s["lib"], s["case"]
    stream = torch.cuda.current_stream().cuda_stream
    op, layer = case["op"], case.get("layers", 1) - 1
    if op == "tree":
        kv4.kfl_kv4_tree(s["parents"], s["views"], s["positions"], q_start=s["q_start"], first=s["first"],
                         max_q=s["max_q"], cuda_stream=stream)
        return {"views": s["views"], "positions": s["positions"]}
    if op == "attend":
        kv4.kfl_kv4_attend_tree(s["pages"], s["map"], layer, s["q"], s["out"], s["views"], s["workspace"],
                                q_start=s["q_start"], max_q=s["max_q"], window=case["window"], cuda_stream=stream)
        return {"out": s["out"]}
    if op == "weights":
        kv4.kfl_kv4_weights(s["pages"], s["map"], layer, s["q"], s["lse"], s["mass"], s["workspace"],
                            q_start=s["q_start"], max_q=s["max_q"], window=case["window"], cuda_stream=stream)
        return {"mass": s["mass"]}
    if op == "select":
        kv4.kfl_kv4_select(s["pages"], s["map"], s["mass"], s["users"], case["budget"], s["rows"], s["counts"],
                           first=case["first"], recent=case["recent"], cuda_stream=stream)
        return {"rows": s["rows"], "counts": s["counts"]}
    kv4.kfl_kv4_keep(s["pages"], s["map"], s["users"], s["rows"], s["counts"], s["workspace"], first=s["first"],
                     mass=s["mass"], cuda_stream=stream)
    kv4.kfl_kv4_reserve(s["pages"], s["map"], s["users"], s["n_new"], s["workspace"], cuda_stream=stream)
    return {"table": s["table"], "refs": s["refs"], "lengths": s["lengths"], "pool": s["pool"], "mass": s["mass"]}


PLAIN = {"tree": _plain_tree, "attend": _plain_attend, "weights": _plain_weights, "select": _plain_select,
         "keep": _plain_keep}


def run(state):
    return _own(state) if own else PLAIN[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------- what it has to do

def work(case):
    op, hd = case["op"], case.get("head_dim", 0)
    if op == "tree":
        tokens = _list(case["tokens"])
        return {"bytes": sum(tokens) * (8 + 4 * -(-max(tokens) // 32)) + 8 * len(tokens), "flops": 0}
    lengths = _list(case["lengths"])
    if op in ("attend", "weights"):
        heads, kv_heads = case["q_heads"], case["kv_heads"]
        row = kv_heads * hd * 9 / 16  # a cached token of one layer, k or v
        pairs = rows = 0
        for n, t in zip(lengths, _list(case["tokens"])):
            w = case["window"] or n + 1
            if op == "attend":  # (a node sees itself and some four more)
                pairs += t * min(n - t + min(t, 5), w)
                rows += min(n, w + t)
            else:
                pairs += sum(min(p + 1, w) for p in range(max(0, n - t), n))
                rows += min(n, w + min(n, t) - 1)
        values = sum(_list(case["tokens"])) * heads * hd * 2
        if op == "attend":
            return {"bytes": 2 * rows * row + 2 * values, "flops": 4 * heads * hd * pairs}
        return {"bytes": rows * (row + 8 * kv_heads) + values + sum(_list(case["tokens"])) * heads * 4,
                "flops": 2 * heads * hd * pairs}
    if op == "select":
        lists = case["layers"] * case["kv_heads"]
        return {"bytes": 4 * lists * sum(n + case["budget"] for n in lengths), "flops": 0}
    lists = case["layers"] * case["kv_heads"]
    kept = _list(case["kept"])
    entries = sum(kept) * (lists if case["per_head"] else 1)
    return {"bytes": 2 * lists * sum(kept) * (hd * 9 // 8 + 4) + 4 * entries, "flops": 0}


# ---------------------------------------------------------------------------- outputs in 64 bits

def _exact_values(byte, params):
    """Codes and parameters as 64-bit values, through a table of a byte's two codes."""
    lut = torch.tensor([[(b & 15) - 8, (b >> 4) - 8] for b in range(256)], dtype=torch.float64, device=byte.device)
    v = lut[byte.long()].flatten(-2)
    p = params.double().repeat_interleave(GROUP, dim=-2)
    return p[..., 1] + v * p[..., 0]


def exact(case, seed):
    op = case["op"]
    if op not in ("attend", "weights"):
        # whole numbers, copied bytes, and weights that move as they are
        return None
    if work(case)["flops"] > 4e12:
        return None
    s = prepare(case, seed)
    lengths, tokens = _list(case["lengths"]), _list(case["tokens"])
    hd, group, page, layer = case["head_dim"], case["q_heads"] // case["kv_heads"], case["page"], case["layers"] - 1
    n_codes = page * hd // 2
    parents = _parents(tokens, case["spread"], seed) if op == "attend" else None
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda") if op == "attend" else s["mass"].double()
    at = 0
    for u, (n, t) in enumerate(zip(lengths, tokens)):
        block = s["pool"][s["table"][u, :-(-n // page)].long(), layer]  # page, head, bytes
        codes = block[..., :2 * n_codes].unflatten(-1, (2, page, hd // 2))
        params = block[..., 2 * n_codes:].contiguous().view(torch.float16).unflatten(-1, (2, page, hd // GROUP, 2))
        if op == "attend":
            hidden = torch.ones(t, n, dtype=torch.bool)
            for i in range(t):
                line = [i]
                while parents[at + line[-1]] >= 0:
                    line.append(parents[at + line[-1]])
                hidden[i, [n - t + j for j in line]] = False
                w = case["window"]
                hidden[i, max(0, n - t - max(0, w - len(line))) if w else 0:n - t] = False
            hidden = hidden.cuda()
        else:
            pos, key = torch.arange(n - t, n, device="cuda")[:, None], torch.arange(n, device="cuda")
            hidden = key > pos
            if case["window"]:
                hidden = hidden | (pos - key >= case["window"])
        for h in range(case["kv_heads"]):
            k = _exact_values(codes[:, h, 0], params[:, h, 0]).flatten(0, 1)[:n]
            q = s["q"][at:at + t, h * group:(h + 1) * group].double()
            score = torch.einsum("tgc,kc->gtk", q, k) / math.sqrt(hd)
            if op == "attend":
                score.masked_fill_(hidden, -math.inf)
                v = _exact_values(codes[:, h, 1], params[:, h, 1]).flatten(0, 1)[:n]
                weight = torch.nan_to_num(torch.softmax(score, -1), nan=0.0)
                out[at:at + t, h * group:(h + 1) * group] = torch.einsum("gtk,kc->tgc", weight, v)
            else:
                lse = s["lse"][at:at + t, h * group:(h + 1) * group].double().t()[..., None]
                out[layer, u, h, :n] += (score - lse).exp().masked_fill(hidden, 0.0).sum((0, 1))
        at += t
    return {"out": out} if op == "attend" else {"mass": out}
