"""Plain models of the operators on a paged key/value cache: block bookkeeping on
host lists, attention in 64 bits. They share nothing with the library."""
from __future__ import annotations

import numpy as np

BS = 16


class Pages:
    """Block table, lengths and counts of a cache, and a tag per block that stands for its contents."""

    def __init__(self, table, ctx, refs):
        self.table, self.ctx, self.refs = np.array(table), np.array(ctx), np.array(refs)
        self.tag = np.arange(len(self.refs))
        self.short = False

    def _free(self):
        free = np.nonzero(self.refs == 0)[0]
        return [int(b) for b in free]

    def release(self, rows, window=0, sinks=0):
        for r in rows:
            n = int(self.ctx[r])
            for j in range(self.table.shape[1]):
                b = self.table[r, j]
                # the next query stands at position n and sees n - window + 1 onward, and the sinks
                hidden = not window or (j * BS >= sinks and (j + 1) * BS <= n - window + 1)
                if b >= 0 and hidden:
                    self.refs[b] -= 1
                    self.table[r, j] = -1
            if not window:
                self.ctx[r] = 0

    def reserve(self, rows, new):
        free = self._free()
        for r, m in zip(rows, new):
            for j in range(-(-int(self.ctx[r]) // BS), -(-(int(self.ctx[r]) + int(m)) // BS)):
                if self.table[r, j] < 0:
                    if not free:
                        self.short = True
                        continue
                    b = free.pop(0)
                    self.table[r, j] = b
                    self.refs[b] = 1

    def fork(self, src, dst):
        old, lens = self.table.copy(), self.ctx.copy()
        pairs = [(int(s), int(d)) for s, d in zip(src, dst) if s != d]
        held = set()
        for s, d in pairs:
            for b in old[d]:
                if b >= 0:
                    self.refs[b] -= 1
            n = int(lens[s])
            row = np.full(old.shape[1], -1)
            row[:n // BS] = old[s, :n // BS]
            for b in row:
                if b >= 0:
                    self.refs[b] += 1
            self.table[d], self.ctx[d] = row, n
            if n % BS:
                held.add(int(old[s, n // BS]))
        free = [b for b in self._free() if b not in held]
        for s, d in pairs:
            n = int(lens[s])
            if n % BS:
                if not free:
                    self.short = True
                    self.ctx[d] = n // BS * BS
                    continue
                b = free.pop(0)
                self.table[d, n // BS] = b
                self.refs[b] = 1
                self.tag[b] = self.tag[old[s, n // BS]]

    def compact(self):
        used = [int(b) for b in np.nonzero(self.refs)[0]]
        live = len(used)
        holes = [b for b in range(live) if self.refs[b] == 0]
        high = [b for b in used if b >= live]
        moved = np.where(self.refs > 0, np.arange(len(self.refs)), -1)
        for s, d in zip(high, holes):
            self.table[self.table == s] = d
            self.refs[d], self.refs[s] = self.refs[s], 0
            self.tag[d] = self.tag[s]
            moved[s] = d
        return moved, live


def attention(q, keys, values, pos, window=0, sinks=0, scale=None):
    """One query [H, d] at position pos over keys and values [n, G, d], float64: (o [H, d], lse [H])."""
    H, d = q.shape
    G = keys.shape[1] if len(keys) else 1
    o, lse = np.zeros((H, d)), np.full(H, -np.inf)
    t = np.arange(len(keys))
    seen = (t <= pos) & ((t > pos - window) | (t < sinks) if window else True)
    if pos < 0 or not seen.any():
        return o, lse
    for h in range(H):
        g = h // (H // G)
        s = keys[seen, g] @ q[h] * (scale if scale else d ** -0.5)
        m = s.max()
        p = np.exp(s - m)
        o[h] = p @ values[seen, g] / p.sum()
        lse[h] = m + np.log(p.sum())
    return o, lse
