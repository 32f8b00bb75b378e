"""The operators of the 4-bit paged KV cache as a serving loop uses them.

``Session`` keeps the buffers (pool, tables, workspaces, rotation) of a stage's layers for a number of users and
runs the passes of one layer's attention: reserve room, rotate q, append k and v, attend, and for beams and leaving
users fork, free and compact.  Everything is enqueued on torch's current stream, that of its own tensors.

    python -m paper_2609_34045_gb300.kv4_session

runs a small stage's attention: users with prompts of different lengths, decode steps, beams that fork and change
places, users that leave, and a compaction, with the times of each.
"""
from __future__ import annotations

import argparse

import torch

from . import kv4


class NoRoom(RuntimeError):
    """The pool or a user's row of the table has no room for a pass or a fork; nothing was changed."""


class Session:
    """Buffers of a stage's 4-bit cache: ``n_users`` users of up to ``max_ctx`` tokens sharing ``n_pages`` pages.

    ``status`` collects the bits that kernels raise (0: nothing went wrong); reading it waits for the device."""

    def __init__(self, n_layers, n_heads, n_kv_heads, head_dim, n_users, max_ctx, n_pages, page_tokens=64,
                 dtype=torch.bfloat16, theta=1e6, rope_dim=None, layout="half", max_tokens=2048):
        self.n_heads, self.head_dim, self.dtype, self.n_users = n_heads, head_dim, dtype, n_users
        self.max_ctx, self.page_tokens = max_ctx, page_tokens
        page_bytes = n_layers * n_kv_heads * (page_tokens * head_dim * 9 // 8)
        int32 = dict(dtype=torch.int32, device="cuda")
        self.pages = torch.empty(n_pages * page_bytes, dtype=torch.uint8, device="cuda")
        self.table = torch.full((n_users, -(-max_ctx // page_tokens)), -1, **int32)
        self.lengths, self.refs = torch.zeros(n_users, **int32), torch.zeros(n_pages, **int32)
        self.status, self.n_live = torch.zeros(1, **int32), torch.zeros(1, **int32)
        self.pool = kv4.pool(self.pages, page_tokens, n_layers, n_kv_heads, head_dim)
        self.map = kv4.page_map(self.table, self.lengths, self.refs)
        self.rope = kv4.rope_plan(kv4.kfl_rope_table(max_ctx, rope_dim or head_dim, theta, cuda_stream=self._stream()), layout)
        self.scratch = kv4.pages_workspace(self.pool)
        # attention of one token per user, and of prompts
        self.workspace = kv4.attend_workspace(self.pool, n_heads, n_users, max(max_tokens, n_users), max_tokens)

    @staticmethod
    def _int32(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    @staticmethod
    def _stream():
        """torch's current stream: the inputs, the lists made here and the outputs' memory are ordered on it, and on no other."""
        return torch.cuda.current_stream().cuda_stream

    def _room(self, pages):
        if pages > 0:
            free = int((self.refs == 0).sum())
            if pages > free:
                raise NoRoom(f"{pages} new pages are needed, {free} of {self.refs.numel()} are free")

    def begin(self, counts: dict) -> dict:
        """Room for counts[user] more tokens of each user, and what the layers of the pass need to know of them.  Waits for
        the device once, to read the lengths, and once more in passes that need new pages, to count the free ones: the
        operators themselves only report a full pool in `status`, by which time a pass that goes on has attended at the
        wrong positions.  Raises NoRoom before anything is changed."""
        users, n = list(counts), [counts[u] for u in counts]
        if any(not 0 <= u < self.n_users for u in users) or any(c < 0 for c in n):
            raise ValueError(f"counts of users below {self.n_users}, none negative")
        before = self.lengths.tolist()
        for u, c in zip(users, n):
            if before[u] + c > self.max_ctx:
                raise NoRoom(f"user {u} has {before[u]} tokens and takes {c} more, of {self.max_ctx}")
        pages = [-(-(before[u] + c) // self.page_tokens) - -(-before[u] // self.page_tokens) for u, c in zip(users, n)]
        self._room(sum(pages))
        ids = self._int32(users)
        kv4.kfl_kv4_reserve(self.pool, self.map, ids, self._int32(n), self.scratch, status=self.status,
                            cuda_stream=self._stream())
        start = [0]
        for c in n:
            start.append(start[-1] + c)
        return {"users": ids, "max_q": max(n), "q_start": None if max(n) == min(n) == 1 else self._int32(start),
                "row_users": self._int32([u for u in users for _ in range(counts[u])]),
                "positions": self._int32([before[u] + i for u in users for i in range(counts[u])])}

    def attend(self, layer: int, step: dict, q, k, v, window: int = 0):
        """One layer's attention of a pass: q [token][query head][head_dim] rotated, k and v appended, the users' rows
        attended to."""
        turned, out, stream = torch.empty_like(q), torch.empty_like(q), self._stream()
        kv4.kfl_rope(self.rope, q, turned, None, None, step["positions"], status=self.status, cuda_stream=stream)
        kv4.kfl_kv4_append(self.pool, self.map, layer, k, v, step["row_users"], step["positions"], rope=self.rope,
                           status=self.status, cuda_stream=stream)
        kv4.kfl_kv4_attend(self.pool, self.map, layer, turned, out, self.workspace, users=step["users"],
                           q_start=step["q_start"], max_q=step["max_q"], window=window, status=self.status,
                           cuda_stream=stream)
        return out

    def fork(self, src, dst):
        """User dst[i] goes on from where src[i] is, all at once.  Waits for the device, to read the lengths: raises
        NoRoom where the pool has no page for a copied end (the operator would leave that user as it was)."""
        src, dst = list(src), list(dst)
        if len(src) != len(dst) or len(set(dst)) != len(dst) or any(not 0 <= u < self.n_users for u in src + dst):
            raise ValueError(f"as many users below {self.n_users} in src and dst, in dst none twice")
        lengths = self.lengths.tolist()
        self._room(sum(a != b and lengths[a] % self.page_tokens != 0 for a, b in zip(src, dst)))
        kv4.kfl_kv4_fork(self.pool, self.map, self._int32(src), self._int32(dst), self.scratch, status=self.status,
                         cuda_stream=self._stream())

    def free(self, users):
        kv4.kfl_kv4_free(self.pool, self.map, self._int32(users), status=self.status, cuda_stream=self._stream())

    def compact(self):
        """Live pages to the lowest numbers; returns how many there are (on the device)."""
        kv4.kfl_kv4_compact(self.pool, self.map, self.table, self.refs, self.n_live, self.scratch, status=self.status,
                            cuda_stream=self._stream())
        return self.n_live


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--layers", type=int, default=14)
    ap.add_argument("--steps", type=int, default=32)
    a = ap.parse_args()
    heads, kv_heads, hd = 28, 4, 128  # a 7B-shaped block
    s = Session(a.layers, heads, kv_heads, hd, n_users=8, max_ctx=4096, n_pages=400)
    g = torch.Generator(device="cuda").manual_seed(1)

    def pass_over(name, counts):
        n = sum(counts.values())
        x = torch.randn(a.layers, n, heads + 2 * kv_heads, hd, generator=g, device="cuda").to(s.dtype)
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        step = s.begin(counts)
        begin.record()
        for layer in range(a.layers):
            q, k, v = x[layer].split([heads, kv_heads, kv_heads], dim=1)  # the fused projection's parts, where they are
            s.attend(layer, step, q, k, v)
        end.record()
        torch.cuda.synchronize()
        print(f"{name:32s} {n:6d} tokens x {a.layers} layers: {1e3 * begin.elapsed_time(end):9.1f} us")

    pass_over("prompts of three users", {0: 700, 1: 43, 2: 1500})
    pass_over("prompts of three users, again", {3: 700, 4: 43, 5: 1500})
    for i in range(a.steps):
        pass_over(f"decode step {i}", {u: 1 for u in range(6)}) if i % 8 == 0 else [
            s.attend(layer, step, *(torch.randn(6, h, hd, generator=g, device="cuda").to(s.dtype) for h in (heads, kv_heads, kv_heads)))
            for step in [s.begin({u: 1 for u in range(6)})] for layer in range(a.layers)]
    s.fork([0, 0], [6, 7])           # two beams go on from user 0, its full pages shared
    pass_over("decode step of three beams", {0: 1, 6: 1, 7: 1})
    s.fork([7, 6], [6, 7])           # and change places
    pass_over("drafted tokens checked", {0: 4, 6: 3, 7: 2})
    s.free([1, 2, 3])
    live = s.compact()
    pass_over("decode step after compaction", {0: 1, 4: 1, 5: 1, 6: 1, 7: 1})
    print(f"live pages {live.item()} of {s.refs.numel()}, lengths {s.lengths.tolist()}, status {s.status.item()}")


if __name__ == "__main__":
    main()
