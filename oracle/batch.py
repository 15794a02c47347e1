"""What the selected batch needs next, in 64 bits on the CPU: pages, the 4-bit cache, cached attention, logits.

Written from the definitions alone: a page pool as Python lists, one value at a
time rounded to its nearest 4-bit neighbour, attention and logits as loops over
requests, tokens and heads.
"""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


class Pages:
    """A stack of free pages and the pages each slot holds."""

    def __init__(self, n_pages: int, page_tokens: int, max_jobs: int, max_pages: int):
        self.P, self.max_pages = page_tokens, max_pages
        self.free = list(range(n_pages - 1, -1, -1))
        self.held = [[] for _ in range(max_jobs)]
        self.short = False

    def grow(self, slots, lens, new):
        """(block rows, slot maps) of the call, as lists."""
        blocks, maps, open_ = [], [], True
        for s, length, m in zip(slots, lens, new):
            need = -(-length // self.P) - len(self.held[s])
            if -(-length // self.P) > self.max_pages:
                need = 0
            if need > 0:
                if open_ and need <= len(self.free):
                    for _ in range(need):
                        self.held[s].append(self.free.pop())
                else:
                    open_, self.short = False, True
            blocks.append(list(self.held[s]))
            maps.append([self.held[s][p // self.P] * self.P + p % self.P if 0 <= p and p // self.P < len(self.held[s]) else -1
                         for p in range(length - m, length)])
        return blocks, maps

    def trim(self, slots, lens):
        give = []
        for s, length in zip(slots, lens):
            keep = min(len(self.held[s]), -(-length // self.P))
            give += self.held[s][keep:]
            del self.held[s][keep:]
        self.free += give[::-1]


def kv_round(x: np.ndarray) -> np.ndarray:
    """What the cache keeps of x (last axis a multiple of 32)."""
    g = np.asarray(x, np.float64).reshape(-1, 32)
    out = np.empty_like(g)
    for i, row in enumerate(g):
        top = np.abs(row).max()
        if not np.isfinite(row).all():
            out[i] = np.nan
            continue
        e = -125
        while top >= 7.0 * 2.0 ** e and e < 125:
            e += 1
        y = np.abs(row) / 2.0 ** e
        for j, v in enumerate(y):
            d = np.abs(E2M1 - v)
            near = np.flatnonzero(d == d.min())
            code = near[0] if len(near) == 1 else near[near % 2 == 0][0]
            out[i, j] = np.sign(row[j]) * E2M1[code] * 2.0 ** e
    return out.reshape(x.shape)


def kv_attention(q, k, v, kv_len: int, scale: float, window: int = 0, seen=None):
    """One request: q [t, heads, d], k and v [>= kv_len, kv heads, d]; seen: bool [kv_len], keys on valid pages."""
    t, H, d = q.shape
    G = H // k.shape[1]
    out = np.zeros((t, H, d))
    for i in range(t):
        p = kv_len - t + i
        lo = max(0, p - window + 1) if window else 0
        keys = [j for j in range(lo, p + 1) if seen is None or seen[j]]
        if not keys:
            continue
        for h in range(H):
            s = k[keys, h // G].astype(np.float64) @ q[i, h].astype(np.float64) * scale
            w = np.exp(s - s.max())
            out[i, h] = (w[:, None] * v[keys, h // G]).sum(0) / w.sum()
    return out


def logits_adjust(x, history, prompt_len: int, repetition=1.0, frequency=0.0, presence=0.0, bias=(), allowed=None):
    """One row: x [vocab], history a list of ids, bias a list of (token, value), allowed bool [vocab] or None."""
    y = np.asarray(x, np.float64).copy()
    V = len(y)
    ids = [t for t in history if 0 <= t < V]
    written = [t for t in history[max(prompt_len, 0):] if 0 <= t < V]
    for v in set(ids):
        y[v] = y[v] / repetition if y[v] > 0 else y[v] * repetition
    for v in set(written):
        y[v] = y[v] - frequency * written.count(v) - presence
    for v, b in bias:
        if 0 <= v < V:
            y[v] += b
    if allowed is not None:
        y[~allowed] = -np.inf
    return y
