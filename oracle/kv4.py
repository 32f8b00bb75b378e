"""Rotary positions and the 4-bit paged KV cache in numpy, 64 bits, from their definitions: test infrastructure only.

``quantise`` / ``values`` are the format of include/kafila_kv4.h (Section V-C and V-D of the paper bound a session by
the bytes of its cache; the paper has no 4-bit cache of its own), ``rotate`` the rotation of include/kafila_rope.h,
``attend`` softmax attention over a user's rows, ``Pages`` the tables.  Nothing here is shared with the CUDA path.
"""
from __future__ import annotations

import numpy as np

GROUP, LIMIT = 64, 32768.0


def quantise(x):
    """Codes 0..15 [..., hd] and (scale, centre) fp16 [..., hd / 64, 2] of rows [..., hd] (fp32 or fp64)."""
    x = np.asarray(x)
    g = x.reshape(*x.shape[:-1], -1, GROUP).astype(np.float32)
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        ok = (np.abs(g) <= LIMIT).all(-1, keepdims=True)
        lo, hi = g.min(-1, keepdims=True), g.max(-1, keepdims=True)
        scale = ((hi - lo) / np.float32(15)).astype(np.float16)
        centre = (lo + np.float32(8) * scale.astype(np.float32)).astype(np.float16)
        inv = np.where(scale > 0, np.float32(1) / scale.astype(np.float32), np.float32(0)).astype(np.float32)
        u = np.clip(np.rint((g - centre.astype(np.float32)) * inv) + 8, 0, 15)
    u = np.where(ok, u, 8).astype(np.uint8).reshape(x.shape)
    params = np.concatenate([scale, centre], -1)
    return u, np.where(ok, params, np.float16(np.nan)).astype(np.float16)


def values(codes, params):
    """fp64 values of codes [..., hd] and (scale, centre) [..., hd / 64, 2]."""
    p = np.repeat(params.astype(np.float64), GROUP, axis=-2)
    return p[..., 1] + (codes.astype(np.float64) - 8) * p[..., 0]


def unpack(block, page, hd):
    """K codes, V codes [page][hd] and K, V parameters [page][hd / 64][2] of one block's bytes."""
    n, m = page * hd // 2, page * hd // 16
    out = []
    for i in range(2):
        b = block[i * n:(i + 1) * n].reshape(page, hd // 2)
        out.append(np.stack([b & 15, b >> 4], -1).reshape(page, hd))
    for i in range(2):
        out.append(block[2 * n + i * m:2 * n + (i + 1) * m].copy().view(np.float16).reshape(page, hd // GROUP, 2))
    return out


def rows(pool, table_row, layer, head, n, page, hd):
    """fp64 K and V of a user's first n rows; pool [pages][layers][heads][bytes]."""
    k, v = np.zeros((n, hd)), np.zeros((n, hd))
    for j in range(-(-n // page)):
        kc, vc, kp, vp = unpack(pool[table_row[j], layer, head], page, hd)
        m = min(page, n - j * page)
        k[j * page:j * page + m] = values(kc, kp)[:m]
        v[j * page:j * page + m] = values(vc, vp)[:m]
    return k, v


def rotate(x, angles, interleaved, magnitude=1.0):
    """x [token][head][hd] turned by angles [token][rope_dim / 2] (fp64)."""
    r = 2 * angles.shape[-1]
    y = np.array(x, dtype=np.float64)
    c, s = magnitude * np.cos(angles)[:, None], magnitude * np.sin(angles)[:, None]
    a, b = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    u, v = y[..., a].copy(), y[..., b].copy()
    y[..., a], y[..., b] = u * c - v * s, v * c + u * s
    return y


def attend(q, k, v, positions, scale, window=0):
    """Tokens q [t][hd] at `positions` over rows k, v [n][hd]: output, the weighted mean of |v|, and the log of the
    sum of exponentials."""
    out, size, lse = np.zeros(q.shape), np.zeros(q.shape), np.full(len(q), -np.inf)
    for i, pos in enumerate(positions):
        a = max(0, pos - window + 1) if window else 0
        if pos < a:
            continue
        x = k[a:pos + 1] @ q[i].astype(np.float64) * scale
        m = x.max()
        w = np.exp(x - m)
        out[i], size[i] = w @ v[a:pos + 1] / w.sum(), w @ np.abs(v[a:pos + 1]) / w.sum()
        lse[i] = m + np.log(w.sum())
    return out, size, lse


def tree_seen(parents):
    """Which nodes each node of a tree sees [node][node], and how many ancestors it has."""
    seen = np.zeros((len(parents), len(parents)), dtype=bool)
    for i, up in enumerate(parents):
        if up >= 0:
            seen[i] = seen[up]
        seen[i, i] = True
    return seen, seen.sum(1) - 1


def tree_words(seen, max_q):
    """Rows of `seen` as 32-bit words, node j in bit j % 32 of word j / 32."""
    out = np.zeros((len(seen), -(-max_q // 32)), dtype=np.uint32)
    for i, j in zip(*np.nonzero(seen)):
        out[i, j // 32] |= np.uint32(1 << (j % 32))
    return out


def tree_keys(seen, n, window=0):
    """Which of n cached rows, the last of which are the nodes, each node sees."""
    c = len(seen)
    keys = np.zeros((c, n), dtype=bool)
    for i in range(c):
        begin = n - c - max(0, window - int(seen[i].sum())) if window else 0
        keys[i, max(0, begin):max(0, n - c)] = True
        for j in range(c):
            if seen[i, j] and n - c + j >= 0:
                keys[i, n - c + j] = True
    return keys


def causal_keys(count, n, window=0):
    """The same of tokens that see the rows up to their own."""
    pos, key = np.arange(n - count, n)[:, None], np.arange(n)
    return (key <= pos) & ((key > pos - window) if window else True)


def attend_keys(q, k, v, seen, scale):
    """attend over the keys that `seen` [t][n] says."""
    out, size, lse = np.zeros(q.shape), np.zeros(q.shape), np.full(len(q), -np.inf)
    for i in range(len(q)):
        if seen[i].any():
            x = k[seen[i]] @ q[i].astype(np.float64) * scale
            w = np.exp(x - x.max())
            out[i], size[i] = w @ v[seen[i]] / w.sum(), w @ np.abs(v[seen[i]]) / w.sum()
            lse[i] = x.max() + np.log(w.sum())
    return out, size, lse


def weights(q, k, lse, seen, scale):
    """exp(scale q k - lse) [t][n] where seen, else 0."""
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.exp(q.astype(np.float64) @ k.T * scale - lse.astype(np.float64)[:, None])
    return np.where(seen & (lse != -np.inf)[:, None], w, 0.0)


def select(mass, n, budget, first, recent):
    """The slots that stay of n, ascending."""
    if n <= budget:
        return np.arange(n)
    middle = np.arange(first, n - recent)
    order = sorted(middle, key=lambda t: (0 if np.isnan(mass[t]) else 1, 0.0 if np.isnan(mass[t]) else -mass[t], t))
    return np.array(sorted([*range(first), *order[:budget - first - recent], *range(n - recent, n)]))


def keep_bytes(pool, table_row, new_row, layer, head, lists, first, page, hd):
    """One block's rows of kfl_kv4_keep: slots first + j from lists[j], and what stands before them in a new page, into a
    copy of the pool."""
    n, m = page * hd // 2, page * hd // 16
    src = pool.copy()
    begin = first // page * page if new_row[first // page] != table_row[first // page] else first
    for s in range(begin, first + len(lists)):
        e = s if s < first else int(lists[s - first])
        a, b = src[table_row[e // page], layer, head], pool[new_row[s // page], layer, head]
        for at, size in ((0, hd // 2), (n, hd // 2), (2 * n, hd // 16), (2 * n + m, hd // 16)):
            b[at + s % page * size:at + (s % page + 1) * size] = a[at + e % page * size:at + (e % page + 1) * size]


class Pages:
    """Tables of users' pages, as kfl_kv4_reserve, _fork, _free and _compact leave them."""

    def __init__(self, table, lengths, refs, page):
        self.table, self.lengths, self.refs, self.page = table.copy(), lengths.copy(), refs.copy(), page

    def _free_pages(self):
        return [int(i) for i in np.nonzero(self.refs == 0)[0]]

    def reserve(self, users, n_new):
        free, full = self._free_pages(), False
        for u, n in zip(users, n_new):
            held, to = -(-int(self.lengths[u]) // self.page), -(-(int(self.lengths[u]) + int(n)) // self.page)
            if to > self.table.shape[1]:
                continue
            full = full or to - held > len(free)
            if full and to > held:
                continue
            for j in range(held, to):
                self.table[u, j] = free.pop(0)
                self.refs[self.table[u, j]] = 1
            self.lengths[u] += n

    def free(self, users):
        for u in users:
            for page in self.table[u][self.table[u] >= 0]:
                self.refs[page] -= 1
            self.table[u], self.lengths[u] = -1, 0

    def fork(self, src, dst):
        """Returns the (source, destination) pages to copy."""
        free, old, lengths, copies = self._free_pages(), self.table.copy(), self.lengths.copy(), []
        for a, b in zip(src, dst):
            if a == b:
                continue
            full, end = divmod(int(lengths[a]), self.page)
            if end and not free:
                continue
            row = np.full_like(old[b], -1)
            row[:full] = old[a, :full]
            self.refs[old[a, :full]] += 1
            if end:
                row[full] = free.pop(0)
                self.refs[row[full]] = 1
                copies.append((int(old[a, full]), int(row[full])))
            for page in old[b][old[b] >= 0]:
                self.refs[page] -= 1
            self.table[b], self.lengths[b] = row, lengths[a]
        return copies

    def keep(self, users, first, counts):
        """The users' old rows of the table (None: not touched)."""
        free, old, refs, gone = self._free_pages(), [], self.refs.copy(), []
        used = 0
        for u, f, c in zip(users, first, counts):
            n = int(self.lengths[u])
            if f + c == n:
                old.append(None)
                continue
            row, need, held = self.table[u].copy(), -(-(f + c) // self.page), -(-n // self.page)
            shared = [j for j in range(f // self.page, need) if refs[row[j]] > 1]
            used += len(shared)
            if shared and used > len(free):
                old.append(None)
                continue
            for r, j in enumerate(shared):
                new = free[used - len(shared) + r]
                gone.append(row[j])
                self.table[u, j], self.refs[new] = new, 1
            gone += [int(p) for p in row[need:held]]
            self.table[u, need:held] = -1
            self.lengths[u] = f + c
            old.append(row)
        for p in gone:
            self.refs[p] -= 1
        return old

    def compact(self):
        live = np.nonzero(self.refs)[0]
        n = len(live)
        moves = list(zip(live[live >= n], [i for i in range(n) if self.refs[i] == 0]))
        for a, b in moves:
            self.refs[b], self.refs[a] = self.refs[a], 0
            self.table[self.table == a] = b
        return moves, n
