"""Plain definitions of the decoding operators in 64 bits, one element after the other (test infrastructure only).

attention(): numpy f64 over a paged cache, with what a tolerance is counted from.  verify(): drafts against probabilities.  Pages: a
cache in Python lists, its pages taken and given back one by one.
"""
from __future__ import annotations

import numpy as np


def attention(q, k, v, table, lens, prefix, seqs, scale):
    """out (B, T, H, D), lse (B, T, H), and per output: weighted |v|, largest |scale| * sum |q k|, visible keys, largest |v|."""
    B, T, H, D = q.shape
    P, ps, Hk, _ = k.shape
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    out, lse = np.zeros((B, T, H, D)), np.full((B, T, H), -np.inf)
    mass, size, count, top = np.zeros((B, T, H, D)), np.zeros((B, T, H)), np.zeros((B, T, H)), np.zeros((B, T, H))
    rows = list(range(B)) if seqs is None else [int(s) for s in seqs]
    for b, row in enumerate(rows):
        n = int(lens[row])
        at = np.arange(n)
        page = np.array([table[rows[0] if j < prefix else row][j // ps] for j in range(n)], dtype=np.int64)
        for t in range(T):
            m = n - (T - 1 - t)
            if m <= 0:
                continue
            for h in range(H):
                kk, vv = k[page[:m], at[:m] % ps, h // (H // Hk)], v[page[:m], at[:m] % ps, h // (H // Hk)]
                with np.errstate(invalid="ignore", over="ignore"):
                    s = scale * (kk @ q[b, t, h])
                    big = s.max()
                    if big == -np.inf:
                        continue
                    w = np.exp(s - big)
                    total = w.sum()
                    out[b, t, h] = (w @ vv) / total
                    lse[b, t, h] = big + np.log(total)
                    mass[b, t, h] = (w @ np.abs(vv)) / total
                    size[b, t, h] = scale * (np.abs(kk) @ np.abs(q[b, t, h])).max()
                    count[b, t, h], top[b, t, h] = m, np.abs(vv).max()
    return out, lse, mass, size, count, top


def verify(target, tokens, draft, u, r, n_drafts=None):
    """accepted (B), tokens (B, L + 1), and how near the drawn token's border the goal came (relative to the total)."""
    B, L = tokens.shape
    V = target.shape[2]
    accepted, out, near = np.zeros((B,), np.int64), np.full((B, L + 1), -1, np.int64), np.full((B,), np.inf)
    for b in range(B):
        n = L if n_drafts is None else min(max(int(n_drafts[b]), 0), L)
        i = 0
        while i < n:
            d = int(tokens[b, i])
            if not 0 <= d < V:
                break
            q = 1.0 if draft is None else float(draft[b, i, d])
            if not float(u[b, i]) * q < float(target[b, i, d]):
                break
            out[b, i] = d
            i += 1
        accepted[b] = i
        p = np.asarray(target[b, i], np.float64)
        w = p.copy()
        if i < n:
            if draft is None:
                if 0 <= tokens[b, i] < V:
                    w[tokens[b, i]] -= 1.0
            else:
                w = p - np.asarray(draft[b, i], np.float64)
        w = np.where(w > 0, w, 0.0)
        if not (w.sum() > 0):
            w = np.where(p > 0, p, 0.0)
        if not (w > 0).any():
            continue
        c = np.cumsum(w)
        goal = float(r[b]) * c[-1]
        out[b, i] = min(int(np.searchsorted(c, goal, side="right")), int(np.nonzero(w > 0)[0][-1]))
        near[b] = np.abs(c[w > 0] - goal).min() / c[-1]
    return accepted, out, near


class Pages:
    """A cache's tables and pools, as lists."""

    def __init__(self, pages, page_size, rows, row_pages, pools):
        self.ps, self.pages, self.row_pages = page_size, pages, row_pages
        self.table = [[-1] * row_pages for _ in range(rows)]
        self.lens, self.refs, self.free = [0] * rows, [0] * pages, list(range(pages - 1, -1, -1))
        self.pools = pools  # numpy (pages, page_size, ...)
        self.status = 0

    def _held(self, n):
        return -(-n // self.ps)

    def _take(self):
        p = self.free.pop()
        self.refs[p] = 1
        return p

    def _give(self, pages):
        ended = []
        for p in pages:
            self.refs[p] -= 1
            if self.refs[p] == 0:
                ended.append(p)
        self.free += sorted(ended, reverse=True)

    def fork(self, parents, children):
        if any(self.lens[c] for c in children):
            self.status |= 2
            return
        if sum(self.lens[p] % self.ps > 0 for p in parents) > len(self.free):
            self.status |= 1
            return
        before = [(self.lens[p], self.table[p][:self._held(self.lens[p])]) for p in parents]   # (a parent may be a child of the same call)
        for (n, row), c in zip(before, children):
            row = list(row)
            part = n % self.ps
            for page in row[:-1] if part else row:
                self.refs[page] += 1
            if part:
                old, row[-1] = row[-1], self._take()
                for pool in self.pools:
                    pool[row[-1], :part] = pool[old, :part]
            self.table[c] = row + [-1] * (self.row_pages - len(row))
            self.lens[c] = n

    def append(self, seqs, values):
        T = values[0].shape[1]
        if any(self.lens[s] + T > self.row_pages * self.ps for s in seqs):
            self.status |= 8
            return
        shared = [self.lens[s] % self.ps > 0 and self.refs[self.table[s][self._held(self.lens[s]) - 1]] > 1 for s in seqs]
        if sum(self._held(self.lens[s] + T) - self._held(self.lens[s]) + c for s, c in zip(seqs, shared)) > len(self.free):
            self.status |= 1
            return
        left = []
        for i, (s, copy) in enumerate(zip(seqs, shared)):
            n, row = self.lens[s], self.table[s]
            if copy:
                at = self._held(n) - 1
                left.append(row[at])
                old, row[at] = row[at], self._take()
                for pool in self.pools:
                    pool[row[at], :n % self.ps] = pool[old, :n % self.ps]
            for k in range(self._held(n), self._held(n + T)):
                row[k] = self._take()
            for x in range(T):
                for pool, v in zip(self.pools, values):
                    pool[row[(n + x) // self.ps], (n + x) % self.ps] = v[i, x]
            self.lens[s] = n + T
        self._give(left)

    def release(self, seqs, drop=None):
        gone = []
        for i, s in enumerate(seqs):
            keep = 0 if drop is None else max(0, self.lens[s] - max(0, int(drop[i])))
            for k in range(self._held(keep), self._held(self.lens[s])):
                gone.append(self.table[s][k])
                self.table[s][k] = -1
            self.lens[s] = keep
        self._give(gone)

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        remap = [p if r > 0 else -1 for p, r in enumerate(self.refs)]
        moves = list(zip([p for p in range(live, self.pages) if self.refs[p] > 0], [p for p in range(live) if self.refs[p] == 0]))
        for a, b in moves:
            remap[a] = b
            self.refs[b], self.refs[a] = self.refs[a], 0
            for pool in self.pools:
                pool[b] = pool[a]
        self.table = [[remap[p] if p >= 0 else -1 for p in row] for row in self.table]
        self.free = list(range(self.pages - 1, live - 1, -1))
        return remap
