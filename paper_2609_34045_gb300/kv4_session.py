"""The operators of the 4-bit paged KV cache as a serving loop uses them.

``Session`` keeps the buffers (pool, tables, workspaces, rotation) of a stage's layers for a number of users and
runs the passes of one layer's attention: reserve room, rotate q, append k and v, attend, and for beams and leaving
users fork, free and compact.  A pass may be of trees of drafted tokens, of which ``accept`` keeps a path each; with ``masses``
the weight that every cached row gets is summed up, by which ``evict`` cuts users to a budget of rows.  Everything is enqueued
on torch's current stream, that of its own tensors.

    python -m paper_2609_34045_gb300.kv4_session

runs a small stage's attention: users with prompts of different lengths, decode steps, beams that fork and change
places, trees of drafts, users that are cut and that leave, and a compaction, with the times of each.
"""
from __future__ import annotations

import argparse

import torch

from . import kv4


class NoRoom(RuntimeError):
    """The pool or a user's row of the table has no room for a pass or a fork; nothing was changed."""


class Session:
    """Buffers of a stage's 4-bit cache: ``n_users`` users of up to ``max_ctx`` tokens sharing ``n_pages`` pages.

    ``status`` collects the bits that kernels raise (0: nothing went wrong); reading it waits for the device.  ``masses``: keep
    the attention weight that every row has had, which ``evict`` goes by.  ``max_positions``: of the rotation, for users
    that go on beyond max_ctx by evicting rows (default: max_ctx)."""

    def __init__(self, n_layers, n_heads, n_kv_heads, head_dim, n_users, max_ctx, n_pages, page_tokens=64,
                 dtype=torch.bfloat16, theta=1e6, rope_dim=None, layout="half", max_tokens=2048, masses=False,
                 max_positions=None):
        self.n_heads, self.head_dim, self.dtype, self.n_users = n_heads, head_dim, dtype, n_users
        self.n_layers, self.n_kv_heads = n_layers, n_kv_heads
        self.max_ctx, self.page_tokens, self.max_positions = max_ctx, page_tokens, max_positions or max_ctx
        self.evicted = [0] * n_users  # rows that a user has lost: its next token's position is its length and these
        self.drafts = [None] * n_users  # the pass whose tree a user's last rows are, until it is accepted
        page_bytes = n_layers * n_kv_heads * (page_tokens * head_dim * 9 // 8)
        int32 = dict(dtype=torch.int32, device="cuda")
        self.pages = torch.empty(n_pages * page_bytes, dtype=torch.uint8, device="cuda")
        self.table = torch.full((n_users, -(-max_ctx // page_tokens)), -1, **int32)
        self.lengths, self.refs = torch.zeros(n_users, **int32), torch.zeros(n_pages, **int32)
        self.status, self.n_live = torch.zeros(1, **int32), torch.zeros(1, **int32)
        self.pool = kv4.pool(self.pages, page_tokens, n_layers, n_kv_heads, head_dim)
        self.map = kv4.page_map(self.table, self.lengths, self.refs)
        self.rope = kv4.rope_plan(kv4.kfl_rope_table(self.max_positions, rope_dim or head_dim, theta, cuda_stream=self._stream()), layout)
        self.scratch = kv4.pages_workspace(self.pool)
        # attention of one token per user, and of prompts
        self.workspace = kv4.attend_workspace(self.pool, n_heads, n_users, max(max_tokens, n_users), max_tokens)
        self.mass = None
        if masses:
            self.mass = torch.zeros(n_layers, n_users, n_kv_heads, self.table.shape[1] * page_tokens, dtype=torch.float32,
                                    device="cuda")

    @staticmethod
    def _int32(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    @staticmethod
    def _stream():
        """torch's current stream: the inputs, the lists made here and the outputs' memory are ordered on it, and on no other."""
        return torch.cuda.current_stream().cuda_stream

    def _no_drafts(self, users):
        waiting = [u for u in users if self.drafts[u] is not None]
        if waiting:
            raise ValueError(f"a tree of users {waiting} waits: accept it, once, or free them")

    def _room(self, pages):
        if pages > 0:
            free = int((self.refs == 0).sum())
            if pages > free:
                raise NoRoom(f"{pages} new pages are needed, {free} of {self.refs.numel()} are free")

    def begin(self, counts: dict, parents: dict | None = None) -> dict:
        """Room for counts[user] more tokens of each user, and what the layers of the pass need to know of them.  With
        parents they are the nodes of trees: parents[user][i] is the parent of the user's token i among them, an earlier one
        or -1 (a user without an entry drafts a chain).  Waits for
        the device once, to read the lengths, and once more in passes that need new pages, to count the free ones: the
        operators themselves only report a full pool in `status`, by which time a pass that goes on has attended at the
        wrong positions.  Raises NoRoom before anything is changed.  A user whose tree has not been accepted takes no other pass."""
        users, n = list(counts), [counts[u] for u in counts]
        if any(not 0 <= u < self.n_users for u in users) or any(c < 0 for c in n):
            raise ValueError(f"counts of users below {self.n_users}, none negative")
        self._no_drafts([u for u in users if counts[u] > 0])
        trees = None
        if parents is not None:
            trees = [list(parents.get(u, range(-1, c - 1))) for u, c in zip(users, n)]
            if set(parents) - set(users) or any(len(t) != c or any(not -1 <= p < i for i, p in enumerate(t)) for t, c in zip(trees, n)):
                raise ValueError("parents are those of the pass's users: for each of a user's tokens an earlier one, or -1")
            if max(n, default=0) > 1024:
                raise ValueError("a tree has at most 1024 nodes")
        before = self.lengths.tolist()
        for u, c in zip(users, n):
            if before[u] + c > self.max_ctx:
                raise NoRoom(f"user {u} has {before[u]} tokens and takes {c} more, of {self.max_ctx}")
            if before[u] + self.evicted[u] + c > self.max_positions:
                raise NoRoom(f"user {u} is at position {before[u] + self.evicted[u]} and takes {c} more, of {self.max_positions}")
        pages = [-(-(before[u] + c) // self.page_tokens) - -(-before[u] // self.page_tokens) for u, c in zip(users, n)]
        self._room(sum(pages))
        ids = self._int32(users)
        kv4.kfl_kv4_reserve(self.pool, self.map, ids, self._int32(n), self.scratch, status=self.status,
                            cuda_stream=self._stream())
        start = [0]
        for c in n:
            start.append(start[-1] + c)
        slots = self._int32([before[u] + i for u in users for i in range(counts[u])])
        step = {"users": ids, "max_q": max(n), "q_start": None if max(n) == min(n) == 1 else self._int32(start),
                "row_users": self._int32([u for u in users for _ in range(counts[u])]), "slots": slots, "positions": slots}
        if any(self.evicted[u] for u in users):
            step["positions"] = self._int32([before[u] + self.evicted[u] + i for u in users for i in range(counts[u])])
        if trees is not None:
            deepest = 0
            for t in trees:
                depth = []
                for p in t:
                    depth.append(1 + (depth[p] if p >= 0 else 0))
                deepest = max([deepest, *depth])
            mark = object()
            for u, c in zip(users, n):
                if c > 0:
                    self.drafts[u] = mark
            step.update(mark=mark, trees=dict(zip(users, trees)), before={u: before[u] for u in users}, start=start, rows={}, deepest=deepest,
                        views=torch.empty(start[-1], -(-step["max_q"] // 32), dtype=torch.int32, device="cuda"),
                        positions=torch.empty(start[-1], dtype=torch.int32, device="cuda"))
            if start[-1] > 0:
                step["parents"] = self._int32([p for t in trees for p in t])
                kv4.kfl_kv4_tree(step["parents"], step["views"], step["positions"],
                                 q_start=step["q_start"], first=self._int32([before[u] + self.evicted[u] for u in users]),
                                 max_q=step["max_q"], status=self.status, cuda_stream=self._stream())
        return step

    def _views(self, step, window):
        """What the nodes of a pass see of their trees: their paths, or with a window that is shorter than one, its nodes."""
        if not 0 < window < step["deepest"]:
            return step["views"]
        views = torch.empty_like(step["views"])
        kv4.kfl_kv4_tree(step["parents"], views, q_start=step["q_start"], max_q=step["max_q"], window=window, status=self.status,
                         cuda_stream=self._stream())
        return views

    def attend(self, layer: int, step: dict, q, k, v, window: int = 0):
        """One layer's attention of a pass: q [token][query head][head_dim] rotated, k and v appended, the users' rows
        attended to, with a window the last `window` of them that a token would see behind its path alone.  With masses their weights
        are added up, of trees by `accept`; a window shorter than the longest path is refused there."""
        if "trees" in step and self.mass is not None and 0 < window < step["deepest"]:
            raise ValueError(f"a path of {step['deepest']} nodes is longer than the window of {window}")
        turned, out, stream = torch.empty_like(q), torch.empty_like(q), self._stream()
        places = dict(status=self.status, cuda_stream=stream)
        kv4.kfl_rope(self.rope, q, turned, None, None, step["positions"], **places)
        kv4.kfl_kv4_append(self.pool, self.map, layer, k, v, step["row_users"], step["slots"], rope=self.rope,
                           rope_positions=None if step["positions"] is step["slots"] else step["positions"], **places)
        lse = None if self.mass is None else torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
        rows = dict(users=step["users"], q_start=step["q_start"], max_q=step["max_q"], window=window, **places)
        if "views" in step:
            kv4.kfl_kv4_attend_tree(self.pool, self.map, layer, turned, out, self._views(step, window), self.workspace, lse=lse, **rows)
            if lse is not None:
                step["rows"][layer] = (turned, lse, window)
        elif lse is not None:
            kv4.kfl_kv4_attend(self.pool, self.map, layer, turned, out, self.workspace, lse=lse, **rows)
            kv4.kfl_kv4_weights(self.pool, self.map, layer, turned, lse, self.mass, self.workspace, **rows)
        else:
            kv4.kfl_kv4_attend(self.pool, self.map, layer, turned, out, self.workspace, **rows)
        return out

    def _unshared(self, users, first, stop):
        """Room for the pages that rows move in and that others hold too (first, stop: slots)."""
        table, refs = self.table.tolist(), self.refs.tolist()
        self._room(sum(refs[table[u][j]] > 1 for u, a, b in zip(users, first, stop)
                       for j in range(a // self.page_tokens, -(-b // self.page_tokens))))

    def accept(self, step: dict, paths: dict):
        """Of the trees of a pass each user's nodes paths[user] stay, from a root down, each the child of the one before it
        (none, and users that are not named: nothing of the tree stays); the others' rows go.  With masses, the weights that
        the accepted tokens gave are added up.  Once for a pass, before its users' next one: until then its users take no other
        pass and are neither cut nor forked from, but may leave (be freed, or forked over).  Waits for the device, to look for
        pages that others hold too, and raises NoRoom where there are none to be had in their place."""
        if "trees" not in step or "accepted" in step:
            raise ValueError("a pass of trees is accepted, once")
        users = [u for u in step["trees"] if self.drafts[u] is step["mark"]]
        kept = [list(paths.get(u, [])) for u in users]
        if any(u in step["trees"] and u not in users and list(paths[u]) for u in paths):
            raise ValueError("the trees are no longer their users' last tokens")
        if set(paths) - set(step["trees"]) or any(not 0 <= j < len(step["trees"][u]) or step["trees"][u][j] != up
                                                  for u, path in zip(users, kept) for j, up in zip(path, [-1] + path)):
            raise ValueError("paths are of the pass's users, each node the child of the one before it")
        lengths = self.lengths.tolist()
        if any(lengths[u] != step["before"][u] + len(step["trees"][u]) for u in users):
            raise ValueError("the trees are no longer their users' last tokens")
        first = [step["before"][u] for u in users]
        counts = [len(path) for path in kept]
        self._unshared(users, first, [a + c for a, c in zip(first, counts)])
        step["accepted"] = True
        for u in users:
            self.drafts[u] = None
        if not users:
            return
        ids = self._int32(users)
        most = max([1, *counts])
        rows = self._int32([[a + j for j in path] + [-1] * (most - len(path)) for a, path in zip(first, kept)])
        kv4.kfl_kv4_keep(self.pool, self.map, ids, rows[None, :, None].expand(self.n_layers, len(users), self.n_kv_heads, most),
                         self._int32(counts), self.scratch, first=self._int32(first), mass=self.mass, status=self.status,
                         cuda_stream=self._stream())
        if self.mass is None or sum(counts) == 0:
            return
        start = dict(zip(step["trees"], step["start"]))
        at = [start[u] + j for u, path in zip(users, kept) for j in path]
        pick = torch.tensor(at, device="cuda")
        start = [sum(counts[:i]) for i in range(len(counts) + 1)]
        for layer, (q, lse, window) in step["rows"].items():
            kv4.kfl_kv4_weights(self.pool, self.map, layer, q[pick], lse[pick], self.mass, self.workspace, users=ids,
                                q_start=self._int32(start), max_q=max(counts), window=window, status=self.status,
                                cuda_stream=self._stream())

    def evict(self, budget: int, users=None, first: int = 4, recent: int = 64):
        """Users (None: all) with more than `budget` rows are cut to it, in each layer and KV head on its own: the `first`
        rows stay, the `recent` last ones, and of the others those with the greatest mass.  Returns how many rows each lost.  Waits
        for the device; raises NoRoom where pages that others hold too cannot be replaced."""
        if self.mass is None:
            raise ValueError("a session with masses evicts")
        if budget < 1 or first < 0 or recent < 0 or first + recent > budget:
            raise ValueError("first and recent are not negative and together at most the budget")
        users = list(range(self.n_users) if users is None else users)
        if len(set(users)) != len(users) or any(not 0 <= u < self.n_users for u in users):
            raise ValueError(f"users below {self.n_users}, none twice")
        lengths = self.lengths.tolist()
        users = [u for u in users if lengths[u] > budget]
        if not users:
            return {}
        self._no_drafts(users)
        self._unshared(users, [0] * len(users), [budget] * len(users))
        ids, stream = self._int32(users), self._stream()
        rows = torch.empty(self.n_layers, len(users), self.n_kv_heads, budget, dtype=torch.int32, device="cuda")
        counts = torch.empty(len(users), dtype=torch.int32, device="cuda")
        kv4.kfl_kv4_select(self.pool, self.map, self.mass, ids, budget, rows, counts, first=first, recent=recent,
                           status=self.status, cuda_stream=stream)
        kv4.kfl_kv4_keep(self.pool, self.map, ids, rows, counts, self.scratch, mass=self.mass, status=self.status,
                         cuda_stream=stream)
        lost = {u: lengths[u] - budget for u in users}
        for u in users:
            self.evicted[u] += lost[u]
        return lost

    def fork(self, src, dst):
        """User dst[i] goes on from where src[i] is, all at once.  Waits for the device, to read the lengths: raises
        NoRoom where the pool has no page for a copied end (the operator would leave that user as it was)."""
        src, dst = list(src), list(dst)
        if len(src) != len(dst) or len(set(dst)) != len(dst) or any(not 0 <= u < self.n_users for u in src + dst):
            raise ValueError(f"as many users below {self.n_users} in src and dst, in dst none twice")
        self._no_drafts([a for a, b in zip(src, dst) if a != b])
        lengths = self.lengths.tolist()
        self._room(sum(a != b and lengths[a] % self.page_tokens != 0 for a, b in zip(src, dst)))
        kv4.kfl_kv4_fork(self.pool, self.map, self._int32(src), self._int32(dst), self.scratch, status=self.status,
                         cuda_stream=self._stream())
        if self.mass is not None:
            self.mass[:, dst] = self.mass[:, src]
        evicted = [self.evicted[u] for u in src]
        for a, u, n in zip(src, dst, evicted):
            self.evicted[u] = n
            if a != u:
                self.drafts[u] = None

    def free(self, users):
        users = list(users)
        kv4.kfl_kv4_free(self.pool, self.map, self._int32(users), status=self.status, cuda_stream=self._stream())
        users = [u for u in users if 0 <= u < self.n_users]  # (the others are reported in `status`)
        if self.mass is not None and users:
            self.mass[:, users] = 0
        for u in users:
            self.evicted[u], self.drafts[u] = 0, None

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
    s = Session(a.layers, heads, kv_heads, hd, n_users=8, max_ctx=4096, n_pages=400, masses=True, max_positions=8192)
    g = torch.Generator(device="cuda").manual_seed(1)

    def pass_over(name, counts, parents=None):
        n = sum(counts.values())
        x = torch.randn(a.layers, n, heads + 2 * kv_heads, hd, generator=g, device="cuda").to(s.dtype)
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        step = s.begin(counts, parents)
        begin.record()
        for layer in range(a.layers):
            q, k, v = x[layer].split([heads, kv_heads, kv_heads], dim=1)  # the fused projection's parts, where they are
            s.attend(layer, step, q, k, v)
        end.record()
        torch.cuda.synchronize()
        print(f"{name:32s} {n:6d} tokens x {a.layers} layers: {1e3 * begin.elapsed_time(end):9.1f} us")
        return step

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
    tree = [-1, 0, 0, 1, 1, 2, 3, 4]  # two drafts behind the first, and so on
    step = pass_over("trees of drafted tokens", {0: 8, 6: 8, 7: 8}, {0: tree, 6: tree, 7: tree})
    s.accept(step, {0: [0, 1, 3, 6], 6: [0, 2], 7: [0]})
    print(f"rows that users lost beyond 512: {s.evict(512, [0, 2, 5])}")
    pass_over("decode step of users that were cut", {0: 1, 2: 1, 5: 1, 6: 1})
    s.free([1, 2, 3])
    live = s.compact()
    pass_over("decode step after compaction", {0: 1, 4: 1, 5: 1, 6: 1, 7: 1})
    print(f"live pages {live.item()} of {s.refs.numel()}, lengths {s.lengths.tolist()}, status {s.status.item()}")


if __name__ == "__main__":
    main()
