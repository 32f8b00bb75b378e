"""The operators of the 4-bit paged KV cache, as cases that can be timed and compared.

A case is one pass through an operator as a serving loop calls it:

* ``rope``: rotary positions of a pass's q and k heads, out of one fused Q/K/V projection;
* ``append``: a pass's k (rotated) and v into the cache's pages in 4 bits, and the rows that the
  cache then stands for read back;
* ``attend``: attention of one or more tokens per user over the user's pages;
* ``fork``, ``turnover``, ``compact``: the pages themselves: beams that go on from one another, users
  that leave and users that come, live pages moved together.

``run`` computes a pass in plain torch in 32 bits, or with ``own`` set calls the library.  ``exact``
recomputes the floating outputs in 64 bits.

The page layout that both share.  A pool is ``[pages][layers][KV heads]`` blocks; a block holds
``page`` tokens of one head: K codes ``[token][head_dim / 2]`` bytes, V codes, K parameters
``[token][head_dim / 64]`` pairs of fp16 (scale, centre), V parameters.  A byte holds two channels,
the even one in its low half.  A value is ``centre + (code - 8) * scale``.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
GROUP = 64       # channels that share a scale and a centre
LIMIT = 32768.0  # a group with a larger magnitude reads as NaN
THETA = 1e6


def _rope(name, tokens, q_heads, kv_heads, head_dim, rope_dim, layout, dtype, start=0):
    return {"name": name, "op": "rope", "tokens": tokens, "q_heads": q_heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "rope_dim": rope_dim, "layout": layout, "dtype": dtype, "start": start}


def _append(name, starts, tokens, kv_heads, head_dim, rope_dim, layout, dtype, page, layers=1):
    return {"name": name, "op": "append", "starts": _text(starts), "tokens": _text(tokens), "kv_heads": kv_heads,
            "head_dim": head_dim, "rope_dim": rope_dim, "layout": layout, "dtype": dtype, "page": page,
            "layers": layers}


def _attend(name, lengths, tokens, q_heads, kv_heads, head_dim, dtype, page, window=0, layers=1):
    return {"name": name, "op": "attend", "lengths": _text(lengths), "tokens": _text(tokens), "q_heads": q_heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype, "page": page, "window": window,
            "layers": layers}


def _pages(name, op, lengths, layers, kv_heads, head_dim, page, n_pages, n_moved):
    return {"name": name, "op": op, "lengths": _text(lengths), "layers": layers, "kv_heads": kv_heads,
            "head_dim": head_dim, "page": page, "n_pages": n_pages, "n_moved": n_moved}


def _text(values):
    return ",".join(str(int(v)) for v in values)


def _list(text):
    return [int(v) for v in text.split(",")]


RAGGED_32 = [8192 - 251 * i for i in range(32)]


def listed():
    return [
        # four users' next tokens in one step of a 32B-shaped block: nothing but latency
        _rope("rope-step-b4", 4, 64, 8, 128, 128, "half", "bf16", start=4096),
        # a long prompt's rows of a block whose heads rotate in their first half only, pairs interleaved
        _rope("rope-prompt-partial", 8192, 28, 4, 128, 64, "interleaved", "fp16"),
        # one step's rows of 32 users into their pages
        _append("append-step-b32", [4096 - 97 * i for i in range(32)], [1] * 32, 8, 128, 128, "half", "bf16", 64),
        # several prompts' rows at once, from places inside a page
        _append("append-prompts-16k", [0, 700, 33, 4096], [8192, 1000, 2047, 5145], 8, 128, 128, "half", "bf16", 64),
        # the tiny model's step with one user: the smallest attention there is to do
        _attend("attend-tiny-b1", [136], [1], 8, 2, 64, "bf16", 16),
        # a step of 32 users at ragged contexts: the cache streams from HBM
        _attend("attend-step-b32-ragged", RAGGED_32, [1] * 32, 64, 8, 128, "bf16", 64),
        # one user at a very long context: one token's work split over the whole GPU
        _attend("attend-step-131072", [131072], [1], 64, 8, 128, "bf16", 64),
        # drafted tokens checked in one step: five tokens for each of four users of a 7B-shaped block
        _attend("attend-draft-b4x5", [3000, 512, 1777, 2305], [5, 5, 5, 5], 28, 4, 128, "fp16", 32, layers=2),
        # a prompt's last 2048 tokens over 8192: matrix products
        _attend("attend-prompt-2048-at-6144", [8192], [2048], 64, 8, 128, "bf16", 64),
        # eight beams of a 7B-shaped stage go on from one another: shared pages, copied ends
        _pages("fork-beams-b8", "fork", [1000 + 37 * i for i in range(8)], 14, 4, 128, 64, 320, 8),
        # 24 of 64 users leave and as many come: tables and counts only
        _pages("turnover-24-of-64", "turnover", [300 + 111 * i for i in range(64)], 1, 4, 128, 64, 8192, 24),
        # a third of the users left: their holes are filled from the pool's end, so that the rest of it can go
        _pages("compact-2048", "compact", [1500 + 61 * i for i in range(24)], 14, 4, 128, 64, 2048, 8),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """Another case of the same ranges: 1 to 64 users, 1 to 131072 positions, one token to prompts of
    2048, heads of 64 and 128 in groups of 1 to 12, pages of 16 to 128 tokens, both 16-bit types (fp32
    too where there are no products), windows."""
    op = rng.choice(["rope", "append", "attend", "attend", "attend", "attend", "fork", "turnover", "compact"])
    head_dim = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 3, 4, 5, 7, 8, 8, 12])
    page = rng.choice([16, 32, 64, 128])
    layout = rng.choice(["half", "interleaved"])
    if op == "rope":
        c = _rope("", _log_int(rng, 1, 1800), kv_heads * min(group, 8), kv_heads, head_dim,
                  rng.choice([head_dim, head_dim // 2, 32]), layout, rng.choice(["bf16", "fp16", "fp32"]),
                  start=rng.randrange(0, 100000))
    elif op == "append":
        n = _log_int(rng, 1, 40)
        long = rng.random() < 0.5
        tokens = [_log_int(rng, 1, 10000 // n) if long else rng.randint(1, 4) for _ in range(n)]
        c = _append("", [rng.randrange(0, 4000) for _ in range(n)], tokens, kv_heads, head_dim,
                    rng.choice([0, head_dim, head_dim // 2]), layout, rng.choice(["bf16", "fp16", "fp32"]), page)
    elif op == "attend":
        kind = rng.choice(["step", "step", "draft", "prompt"])
        dtype = rng.choice(["bf16", "bf16", "fp16"])
        if kind == "step":
            n = _log_int(rng, 1, 64)
            lengths = [_log_int(rng, 1, min(131072, 130000 // n)) for _ in range(n)]
            tokens = [1] * n
        elif kind == "draft":
            n = _log_int(rng, 1, 16)
            lengths = [_log_int(rng, 1, min(16384, 120000 // n)) for _ in range(n)]
            tokens = [rng.randint(1, 12) for _ in range(n)]
        else:
            n = rng.randint(1, 3)
            tokens = [_log_int(rng, 13, 2048 // n) for _ in range(n)]
            lengths = [t + _log_int(rng, 1, 6000 // n) - 1 for t in tokens]
        window = rng.choice([0, 0, 0, _log_int(rng, 1, 4096)])
        c = _attend("", lengths, tokens, kv_heads * min(group, 8 if kind == "prompt" else 12), kv_heads, head_dim,
                    dtype, page, window=window)
    else:
        n = _log_int(rng, 2, 24)
        lengths = [_log_int(rng, 1, 2000) for _ in range(n)]
        pages = sum(-(-v // page) for v in lengths)
        c = _pages("", op, lengths, rng.randint(1, 8), kv_heads, head_dim, page,
                   pages + 2 * n + 8 + rng.randrange(0, 300), rng.randint(1, n))
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


def _rope_table(n_pos, rope_dim, start=0):
    """cos and sin of every position's angles, [n_pos][rope_dim / 2][2], computed in 64 bits."""
    freq = THETA ** (-torch.arange(0, rope_dim, 2, dtype=torch.float64, device="cuda") / rope_dim)
    angle = torch.arange(start, start + n_pos, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.stack([angle.cos(), angle.sin()], -1).float()


def _tables(lengths, page, n_pages, spare, g):
    """Every user's pages, scattered over the pool, and how many users hold each."""
    need = [-(-n // page) for n in lengths]
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    table = torch.full((len(lengths), max(need) + spare), -1, dtype=torch.int32, device="cuda")
    refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    refs[order[:at].long()] = 1
    return table, refs


def _starts(counts):
    out = [0]
    for n in counts:
        out.append(out[-1] + n)
    return out


def prepare(case, seed):
    g = _gen(seed, 7)
    op = case["op"]
    s = {"case": dict(case)}
    if op == "rope":
        n, hd, r = case["tokens"], case["head_dim"], case["rope_dim"]
        rows = case["q_heads"] + 2 * case["kv_heads"]
        # q, k and v as the fused projection leaves them: strided views of one buffer
        x = torch.randn(n, rows, hd, generator=g, device="cuda").to(DTYPES[case["dtype"]])
        s["q"], s["k"] = x[:, :case["q_heads"]], x[:, case["q_heads"]:case["q_heads"] + case["kv_heads"]]
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]).contiguous(), torch.empty_like(s["k"]).contiguous()
        s["table"] = _rope_table(case["start"] + n, r)
        s["positions"] = _int32(range(case["start"], case["start"] + n))
    elif op == "append":
        starts, tokens = _list(case["starts"]), _list(case["tokens"])
        n, hd, h = sum(tokens), case["head_dim"], case["kv_heads"]
        lengths = [a + t for a, t in zip(starts, tokens)]
        n_pages = sum(-(-v // case["page"]) for v in lengths) + 5
        s["table"], s["refs"] = _tables(lengths, case["page"], n_pages, 1, g)
        s["lengths"] = _int32(lengths)
        s["pool"] = torch.full((n_pages, case["layers"], h, _block_bytes(case)), 255, dtype=torch.uint8, device="cuda")
        x = torch.randn(n, 2 * h, hd, generator=g, device="cuda")
        # keys with the few large channels that models have
        x[:, :h] += 4 * (torch.rand(h, hd, generator=g, device="cuda") < 0.05).float()
        x = x.to(DTYPES[case["dtype"]])
        s["k"], s["v"] = x[:, :h], x[:, h:]
        s["k_out"], s["v_out"] = torch.empty_like(s["k"]).contiguous(), torch.empty_like(s["v"]).contiguous()
        s["users"] = _int32([u for u, t in enumerate(tokens) for _ in range(t)])
        s["positions"] = _int32([a + i for a, t in zip(starts, tokens) for i in range(t)])
        s["rope"] = _rope_table(max(lengths), case["rope_dim"]) if case["rope_dim"] else None
    elif op == "attend":
        lengths, tokens = _list(case["lengths"]), _list(case["tokens"])
        n_pages = sum(-(-v // case["page"]) for v in lengths) + 3
        s["table"], s["refs"] = _tables(lengths, case["page"], n_pages, 1, g)
        s["lengths"] = _int32(lengths)
        s["pool"] = _filled_pool(case, n_pages, s["table"], s["lengths"], g)
        x = torch.randn(sum(tokens), case["q_heads"], case["head_dim"], generator=g, device="cuda")
        s["q"] = x.to(DTYPES[case["dtype"]])
        s["out"] = torch.empty_like(s["q"])
        s["q_start"] = None if max(tokens) == min(tokens) == 1 else _int32(_starts(tokens))
        s["max_q"], s["max_len"] = max(tokens), max(lengths)
    else:
        lengths = _list(case["lengths"])
        page, n_pages, m = case["page"], case["n_pages"], case["n_moved"]
        s["table"], s["refs"] = _tables(lengths, page, n_pages, 2, g)
        s["lengths"] = _int32(lengths)
        perm = torch.randperm(len(lengths), generator=g, device="cuda").int()
        if op == "turnover":
            s["users"] = perm[:m].clone()
            s["n_new"] = s["lengths"][perm[:m].long()].flip(0).clone()
        else:
            shape = (n_pages, case["layers"], case["kv_heads"], _block_bytes(case))
            s["pool"] = torch.randint(0, 256, shape, dtype=torch.uint8, generator=g, device="cuda")
        if op == "fork":
            s["src"] = torch.randint(0, len(lengths), (m,), generator=g, device="cuda").int()
            s["dst"] = perm[:m].clone()
        if op == "compact":
            gone = perm[:m].long()
            held = s["table"][gone]
            s["refs"].index_add_(0, held[held >= 0].long(), torch.full_like(held[held >= 0], -1))
            s["table"][gone] = -1
            s["lengths"][gone] = 0
            s["table_out"], s["refs_out"] = torch.empty_like(s["table"]), torch.empty_like(s["refs"])
            s["n_live"] = torch.zeros(1, dtype=torch.int32, device="cuda")
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
    ok = (hi <= LIMIT) & (lo >= -LIMIT)
    scale = torch.where(ok, (hi - lo) / torch.full_like(hi, 15.0), math.nan).half()
    centre = (lo + 8 * scale.float()).half()
    inv = torch.where(scale > 0, 1 / scale.float(), 0.0)
    u = torch.where(ok, (((x - centre.float()) * inv).round() + 8).clamp(0, 15), 8.0).to(torch.uint8).flatten(-2)
    params = torch.where(ok, torch.cat([scale, centre], -1), math.nan)
    return u[..., 0::2] | (u[..., 1::2] << 4), params


def _values(codes, params):
    u = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).float() - 8
    p = params.float()
    return (u.unflatten(-1, (-1, GROUP)) * p[..., :1] + p[..., 1:]).flatten(-2)


def _rotate(x, table, positions, layout):
    """fp32 [token][head][channel], rotated in its first channels by the positions' angles."""
    r = 2 * table.shape[1]
    cs = table[positions.long()][:, None]
    c, s = cs[..., 0], cs[..., 1]
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if layout == "half" else (x[..., 0:r:2], x[..., 1:r:2])
    y, z = a * c - b * s, b * c + a * s
    both = torch.cat([y, z], -1) if layout == "half" else torch.stack([y, z], -1).flatten(-2)
    return torch.cat([both, x[..., r:]], -1)


def _plain_rope(s):
    out = {}
    for n in ("q", "k"):
        y = _rotate(s[n].float(), s["table"], s["positions"], s["case"]["layout"])
        out[n] = y.to(s[n].dtype)
    return out


def _plain_append(s):
    case = s["case"]
    k, v = s["k"].float(), s["v"].float()
    if s["rope"] is not None:
        k = _rotate(k, s["rope"], s["positions"], case["layout"])
    pos = s["positions"].long()
    page = s["table"][s["users"].long(), pos // case["page"]].long()
    slot, layer = pos % case["page"], case["layers"] - 1
    parts = _parts(s["pool"], case)
    out = {}
    for i, (n, x) in enumerate((("k", k), ("v", v))):
        parts[i][page, layer, :, slot], parts[2 + i][page, layer, :, slot] = _quantise(x)
        out[n] = _values(parts[i][page, layer, :, slot], parts[2 + i][page, layer, :, slot]).to(s[n].dtype)
    return out


def _plain_attend(s):
    case = s["case"]
    page, hd, h = case["page"], case["head_dim"], case["kv_heads"]
    q, lengths = s["q"], s["lengths"].long()
    n, group, m = len(lengths), case["q_heads"] // h, s["max_q"]
    parts = _parts(s["pool"], case)
    pages = s["table"][:, :-(-s["max_len"] // page)].long().clamp(min=0)
    key = torch.arange(pages.shape[1] * page, device=q.device)
    cached = (key < lengths[:, None])[:, None, :, None]  # user, head, key, channel
    kv = [torch.where(cached, _values(parts[i][pages, case["layers"] - 1], parts[2 + i][pages, case["layers"] - 1])
                      .transpose(1, 2).flatten(2, 3), 0.0) for i in range(2)]
    # queries padded to [user][KV head][token, group]
    start = torch.arange(n + 1, device=q.device) if s["q_start"] is None else s["q_start"].long()
    count = start[1:] - start[:-1]
    row = torch.arange(m, device=q.device)
    at = (start[:-1, None] + row).clamp(max=q.shape[0] - 1)
    x = q.float()[at].view(n, m, h, group, hd).transpose(1, 2).flatten(2, 3)
    p = torch.matmul(x, kv[0].transpose(-1, -2)) * (1 / math.sqrt(hd))
    pos = (lengths - count)[:, None] + row  # each token's own position
    seen = (key <= pos[..., None]) & (key < lengths[:, None, None])
    if case["window"]:
        seen &= key > pos[..., None] - case["window"]
    seen = seen[:, None, :, None, :].expand(n, 1, m, group, len(key)).flatten(2, 3)
    p = p.masked_fill_(~seen, -math.inf)
    top = p.amax(-1, keepdim=True)
    p = p.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, kv[1]) / torch.where(total == 0, 1.0, total)
    o = o.view(n, h, m, group, hd).transpose(1, 2).reshape(n, m, h * group, hd)
    token = torch.arange(q.shape[0], device=q.device)
    user = torch.searchsorted(start, token, right=True) - 1
    return {"out": o[user, token - start[user]].to(q.dtype)}


def _lowest_free(refs, count):
    return torch.argsort((refs != 0).to(torch.uint8), stable=True)[:count]


def _plain_fork(s):
    case = s["case"]
    page, table, refs, lengths, pool = case["page"], s["table"], s["refs"], s["lengths"], s["pool"]
    src, dst = s["src"].long(), s["dst"].long()
    other = src != dst
    n_src = lengths[src].long()
    full = n_src // page
    ends = (n_src % page > 0) & other
    free = _lowest_free(refs, len(src))
    new = free[(ends.long().cumsum(0) - 1).clamp(min=0)]
    column = torch.arange(table.shape[1], device=table.device)
    rows = torch.where(column < full[:, None], table[src], -1)
    last = (column == full[:, None]) & ends[:, None]
    # (a pair without an end to copy writes a page that it reads, live and so no pair's new one, onto itself)
    old_end = table[src, torch.where(ends, full, 0)].long()
    rows = torch.where(last, new[:, None].int(), rows)
    before = table[dst]
    for held, by in ((torch.where(other[:, None], rows, -1), 1), (torch.where(other[:, None], before, -1), -1)):
        refs.index_add_(0, held.clamp(min=0).flatten().long(), ((held >= 0) * by).flatten().int())
    pool[torch.where(ends, new, old_end)] = pool[old_end]
    table[dst] = torch.where(other[:, None], rows, before)
    lengths[dst] = n_src.int()
    return {"table": table, "refs": refs, "lengths": lengths, "pool": pool}


def _plain_turnover(s):
    page, table, refs, lengths = s["case"]["page"], s["table"], s["refs"], s["lengths"]
    users = s["users"].long()
    held = table[users]
    refs.index_add_(0, held.clamp(min=0).flatten().long(), -(held >= 0).flatten().int())
    need = (s["n_new"].long() + page - 1) // page
    column = torch.arange(table.shape[1], device=table.device)
    wanted = column < need[:, None]
    free = _lowest_free(refs, users.numel() * table.shape[1])
    rank = (wanted.flatten().long().cumsum(0) - 1).clamp(min=0).view(wanted.shape)
    rows = torch.where(wanted, free[rank.clamp(max=free.numel() - 1)].int(), -1)
    refs.index_add_(0, rows.clamp(min=0).flatten().long(), (rows >= 0).flatten().int())
    table[users] = rows
    lengths[users] = s["n_new"]
    return {"table": table, "refs": refs, "lengths": lengths}


def _plain_compact(s):
    refs, table, pool = s["refs"], s["table"], s["pool"]
    page = torch.arange(refs.numel(), device=refs.device)
    live = refs != 0
    n_live = live.sum()
    source, hole = page[live & (page >= n_live)], page[~live & (page < n_live)]
    pool[hole] = pool[source]
    to = page.scatter(0, source, hole).int()
    s["table_out"].copy_(torch.where(table >= 0, to[table.clamp(min=0).long()], -1))
    s["refs_out"].copy_(refs.scatter(0, hole, refs[source]) * (page < n_live))
    s["n_live"].copy_(n_live.int().view(1))
    return {"table": s["table_out"], "refs": s["refs_out"], "n_live": s["n_live"], "pool": pool}


# ------------------------------------------------------------------------------ the library's calls

def _handles(s):
    """What a program keeps beside its buffers: the descriptions of pool, tables and rotation, and the
    attention's workspace."""
    from paper_2609_34045_gb300 import kv4

    s["lib"], case = kv4, s["case"]
    if case["op"] == "rope" or s.get("rope") is not None:
        s["plan"] = kv4.rope_plan(s["table"] if case["op"] == "rope" else s["rope"], case["layout"])
    if case["op"] == "rope":
        return
    if "pool" in s:
        s["pages"] = kv4.pool(s["pool"], case["page"], case["layers"], case["kv_heads"], case["head_dim"])
    else:
        s["pages"] = kv4.pool(None, case["page"], case["layers"], case["kv_heads"], case["head_dim"],
                              n_pages=case["n_pages"])
    s["map"] = kv4.page_map(s["table"], s["lengths"], s["refs"])
    if case["op"] == "attend":
        s["workspace"] = kv4.attend_workspace(s["pages"], case["q_heads"], len(_list(case["lengths"])),
                                              s["q"].shape[0], s["max_q"])
    elif case["op"] != "append":
        s["workspace"] = kv4.pages_workspace(s["pages"])


def _own(s):
    kv4, case = s["lib"], s["case"]
    stream = torch.cuda.current_stream().cuda_stream
    op = case["op"]
    if op == "rope":
        kv4.kfl_rope(s["plan"], s["q"], s["q_out"], s["k"], s["k_out"], s["positions"], cuda_stream=stream)
        return {"q": s["q_out"], "k": s["k_out"]}
    layer = case.get("layers", 1) - 1
    if op == "append":
        kv4.kfl_kv4_append(s["pages"], s["map"], layer, s["k"], s["v"], s["users"], s["positions"],
                           rope=s.get("plan"), cuda_stream=stream)
        kv4.kfl_kv4_read(s["pages"], s["map"], layer, s["users"], s["positions"], s["k_out"], s["v_out"],
                         cuda_stream=stream)
        return {"k": s["k_out"], "v": s["v_out"]}
    if op == "attend":
        kv4.kfl_kv4_attend(s["pages"], s["map"], layer, s["q"], s["out"], s["workspace"], q_start=s["q_start"],
                           max_q=s["max_q"], window=case["window"], cuda_stream=stream)
        return {"out": s["out"]}
    if op == "fork":
        kv4.kfl_kv4_fork(s["pages"], s["map"], s["src"], s["dst"], s["workspace"], cuda_stream=stream)
        return {"table": s["table"], "refs": s["refs"], "lengths": s["lengths"], "pool": s["pool"]}
    if op == "turnover":
        kv4.kfl_kv4_free(s["pages"], s["map"], s["users"], cuda_stream=stream)
        kv4.kfl_kv4_reserve(s["pages"], s["map"], s["users"], s["n_new"], s["workspace"], cuda_stream=stream)
        return {"table": s["table"], "refs": s["refs"], "lengths": s["lengths"]}
    kv4.kfl_kv4_compact(s["pages"], s["map"], s["table_out"], s["refs_out"], s["n_live"], s["workspace"],
                        cuda_stream=stream)
    return {"table": s["table_out"], "refs": s["refs_out"], "n_live": s["n_live"], "pool": s["pool"]}


PLAIN = {"rope": _plain_rope, "append": _plain_append, "attend": _plain_attend, "fork": _plain_fork,
         "turnover": _plain_turnover, "compact": _plain_compact}


def run(state):
    return _own(state) if own else PLAIN[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------- what it has to do

def _size(case):
    return DTYPES[case["dtype"]].itemsize


def work(case):
    op, hd = case["op"], case["head_dim"]
    if op == "rope":
        n, heads = case["tokens"], case["q_heads"] + case["kv_heads"]
        return {"bytes": n * (heads * hd * 2 * _size(case) + case["rope_dim"] * 4 + 4),
                "flops": n * heads * case["rope_dim"] * 3}
    row = case["kv_heads"] * hd * 2 * 9 / 16  # a cached token of one layer, k and v
    if op == "append":
        n = sum(_list(case["tokens"]))
        values = case["kv_heads"] * hd * 2 * _size(case)
        # read k, v and the angles, write the rows; read the rows, write the values
        return {"bytes": n * (2 * values + 2 * row + case["rope_dim"] * 4 + 16),
                "flops": n * case["kv_heads"] * hd * 2 * 8}
    if op == "attend":
        pairs = rows = 0
        for n, t in zip(_list(case["lengths"]), _list(case["tokens"])):
            w = case["window"] or n + 1
            pairs += sum(min(p + 1, w) for p in range(max(0, n - t), n))
            rows += min(n, w + min(n, t) - 1)
        values = sum(_list(case["tokens"])) * case["q_heads"] * hd * 2 * _size(case)
        return {"bytes": rows * row + values, "flops": 4 * case["q_heads"] * hd * pairs}
    lengths, page = _list(case["lengths"]), case["page"]
    width = max(-(-n // page) for n in lengths) + 2
    page_bytes = case["layers"] * case["kv_heads"] * _block_bytes(case)
    if op == "fork":  # the copied ends, and the rows of both sides
        return {"bytes": case["n_moved"] * (2 * page_bytes + 3 * 4 * width), "flops": 0}
    if op == "turnover":
        return {"bytes": case["n_moved"] * 3 * 4 * width + 4 * case["n_pages"], "flops": 0}
    pages = sum(-(-n // page) for n in lengths) * (1 - case["n_moved"] / len(lengths))
    moved = pages * max(0.0, 1 - pages / case["n_pages"])  # live pages, scattered evenly, behind the last place
    return {"bytes": moved * 2 * page_bytes + 2 * 4 * (width * len(lengths) + case["n_pages"]), "flops": 0}


# ---------------------------------------------------------------------------- outputs in 64 bits

def _exact_rotate(x, start_angles, layout):
    """Rotation as a product of complex numbers."""
    r = 2 * start_angles.shape[-1]
    turn = start_angles[:, None]
    z = (torch.complex(x[..., :r // 2].contiguous(), x[..., r // 2:r].contiguous()) if layout == "half"
         else torch.view_as_complex(x[..., :r].unflatten(-1, (-1, 2)).contiguous())) * turn
    y = x.clone()
    if layout == "half":
        y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
    else:
        y[..., :r] = torch.view_as_real(z).flatten(-2)
    return y


def _exact_values(byte, params):
    """Codes and parameters as 64-bit values, through a table of a byte's two codes."""
    lut = torch.tensor([[(b & 15) - 8, (b >> 4) - 8] for b in range(256)], dtype=torch.float64, device=byte.device)
    v = lut[byte.long()].flatten(-2)
    p = params.double().repeat_interleave(GROUP, dim=-2)
    return p[..., 1] + v * p[..., 0]


def exact(case, seed):
    op = case["op"]
    if op in ("fork", "turnover", "compact"):
        return None  # whole numbers and copied bytes
    s = prepare(case, seed)
    if op == "rope":
        turn = torch.view_as_complex(s["table"].double())[s["positions"].long()]
        return {n: _exact_rotate(s[n].double(), turn, case["layout"]) for n in ("q", "k")}
    if op == "append":
        k, v = s["k"].double(), s["v"].double()
        if s["rope"] is not None:
            k = _exact_rotate(k, torch.view_as_complex(s["rope"].double())[s["positions"].long()], case["layout"])
        out = {}
        for n, x in (("k", k), ("v", v)):
            x = x.unflatten(-1, (-1, GROUP))
            lo, hi = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values
            scale = ((hi - lo) / 15).half().double()
            centre = (lo + 8 * scale).half().double()
            code = torch.where(scale > 0, ((x - centre) / scale).round(), 0.0).clamp(-8, 7)
            out[n] = (centre + code * scale).flatten(-2)
        return out
    lengths, tokens = _list(case["lengths"]), _list(case["tokens"])
    if work(case)["flops"] > 4e12:
        return None
    hd, group, page = case["head_dim"], case["q_heads"] // case["kv_heads"], case["page"]
    n_codes, n_params = page * hd // 2, page * hd // 16
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for u, (n, t) in enumerate(zip(lengths, tokens)):
        block = s["pool"][s["table"][u, :-(-n // page)].long(), case["layers"] - 1]  # page, head, bytes
        codes = block[..., :2 * n_codes].unflatten(-1, (2, page, hd // 2))
        params = block[..., 2 * n_codes:].contiguous().view(torch.float16).unflatten(-1, (2, page, hd // GROUP, 2))
        assert params.numel() * 2 == block.shape[0] * block.shape[1] * 2 * n_params
        pos = torch.arange(n - t, n, device="cuda")[:, None]
        key = torch.arange(n, device="cuda")
        hidden = key > pos
        if case["window"]:
            hidden = hidden | (pos - key >= case["window"])
        for h in range(case["kv_heads"]):
            k, v = (_exact_values(codes[:, h, i], params[:, h, i]).flatten(0, 1)[:n] for i in range(2))
            q = s["q"][at:at + t, h * group:(h + 1) * group].double()
            score = torch.einsum("tgc,kc->gtk", q, k) / math.sqrt(hd)
            score.masked_fill_(hidden, -math.inf)
            weight = torch.nan_to_num(torch.softmax(score, -1), nan=0.0)  # a token that sees nothing
            out[at:at + t, h * group:(h + 1) * group] = torch.einsum("gtk,kc->tgc", weight, v)
        at += t
    return {"out": out}
