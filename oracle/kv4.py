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

    def compact(self):
        live = np.nonzero(self.refs)[0]
        n = len(live)
        moves = list(zip(live[live >= n], [i for i in range(n) if self.refs[i] == 0]))
        for a, b in moves:
            self.refs[b], self.refs[a] = self.refs[a], 0
            self.table[self.table == a] = b
        return moves, n
