"""Plain CPU oracle of the paged key-value cache: page bookkeeping in Python integers, norms, rotation and attention in fp64 from their
definitions.  Shares no code with the GPU path.  Arrays hold fp64 copies of the element type's values."""
from __future__ import annotations

import numpy as np


class PagedOracle:
    """Which page holds what.  `content[page]` is any value that identifies a page's contents; copies carry it along."""

    def __init__(self, pages, max_seqs, max_pages, page_tokens):
        self.pages, self.max_seqs, self.max_pages, self.page = pages, max_seqs, max_pages, page_tokens
        self.tables = [[] for _ in range(max_seqs)]
        self.lengths, self.fresh = [0] * max_seqs, [0] * max_seqs
        self.content = {p: ("initial", p) for p in range(pages)}
        self.error, self.moved = 0, 0

    def refs(self):
        r = [0] * self.pages
        for t in self.tables:
            for p in t:
                r[p] += 1
        return r

    def used(self):
        return len({p for t in self.tables for p in t})

    def table(self):
        return [t + [-1] * (self.max_pages - len(t)) for t in self.tables]

    def _free(self):
        held = {p for t in self.tables for p in t}
        return [p for p in range(self.pages) if p not in held]

    def reserve(self, counts):
        if self.error:
            return
        counts = [max(0, int(c)) for c in counts]
        before, free = self.refs(), self._free()
        jobs = []                                        # (slot, column, page to copy from or None)
        for s, c in enumerate(counts):
            n, held = self.lengths[s], len(self.tables[s])
            need = -(-(n + c) // self.page)
            if need > self.max_pages:
                self.error = 3
                self.moved = 0
                return
            if c and n % self.page and before[self.tables[s][-1]] > 1:
                jobs.append((s, held - 1, self.tables[s][-1]))
            jobs += [(s, j, None) for j in range(held, need)]
        if len(jobs) > len(free):
            self.error, self.moved = 3, 0
            return
        self.moved, taken = 0, {}
        for (s, j, old), p in zip(jobs, free):
            if old is not None:
                taken[p] = self.content[old]
                self.tables[s][j] = p
                self.moved += 1
            else:
                self.tables[s].append(p)
        self.content.update(taken)
        for s, c in enumerate(counts):
            self.lengths[s] += c
            self.fresh[s] = c

    def truncate(self, lengths):
        if self.error == 2:
            return
        self.error = 0
        for s, n in enumerate(lengths):
            n = self.lengths[s] if n < 0 else min(int(n), self.lengths[s])
            self.lengths[s], self.fresh[s] = n, 0
            self.tables[s] = self.tables[s][:-(-n // self.page)]

    def fork(self, src, dst):
        if self.error:
            return
        ok = all(0 <= s < self.max_seqs for s in src) and all(0 <= d < self.max_seqs for d in dst)
        if not ok or len(set(dst)) != len(dst) or any(self.lengths[d] for d in dst):
            self.error, self.moved = 1, 0
            return
        partial = [self.lengths[s] % self.page != 0 for s in src]
        free = self._free()
        if sum(partial) > len(free):
            self.error, self.moved = 3, 0
            return
        tables, lengths = [list(self.tables[s]) for s in src], [self.lengths[s] for s in src]
        self.moved = 0
        for t, n, p, d in zip(tables, lengths, partial, dst):
            if p:
                new = free.pop(0)
                self.content[new] = self.content[t[-1]]
                t[-1] = new
                self.moved += 1
            self.tables[d], self.lengths[d], self.fresh[d] = t, n, 0

    def compact(self):
        if self.error:
            return
        r, used = self.refs(), self.used()
        holes = [p for p in range(used) if not r[p]]
        movers = [p for p in range(self.pages - 1, used - 1, -1) if r[p]]
        assert len(holes) == len(movers)
        to = dict(zip(movers, holes))
        for old, new in to.items():
            self.content[new] = self.content[old]
        self.tables = [[to.get(p, p) for p in t] for t in self.tables]
        self.moved = len(holes)


def frequencies(rotary_dim, base=10000.0, kind="plain", factor=1.0, trained=0.0, slow=1.0, fast=32.0):
    i = np.arange(rotary_dim // 2, dtype=np.float64)
    if kind == "base":
        base = base * factor ** (rotary_dim / (rotary_dim - 2.0))
    f = 1.0 / base ** (2.0 * i / rotary_dim)
    if kind == "linear":
        return f / factor
    if kind == "ramp":
        keep = np.clip((trained * f / (2 * np.pi) - slow) / (fast - slow), 0.0, 1.0)
        return keep * f + (1 - keep) * f / factor
    return f


def norm(x, kind, eps, weight=None, bias=None):
    """x [..., head_dim] fp64"""
    if kind == "none":
        return x
    w = np.ones(x.shape[-1]) if weight is None else np.asarray(weight, np.float64)
    if kind == "rms":
        return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    m = x.mean(-1, keepdims=True)
    y = (x - m) / np.sqrt(((x - m) ** 2).mean(-1, keepdims=True) + eps) * w
    return y if bias is None else y + np.asarray(bias, np.float64)


def rotate(x, position, freq, layout, magnitude=1.0):
    """x [heads, head_dim] of one token"""
    y, r = x.copy(), 2 * len(freq)
    for i, f in enumerate(freq):
        a, b = (i, i + r // 2) if layout == "half" else (2 * i, 2 * i + 1)
        c, s = np.cos(position * f), np.sin(position * f)
        y[:, a], y[:, b] = magnitude * (x[:, a] * c - x[:, b] * s), magnitude * (x[:, a] * s + x[:, b] * c)
    return y


def visible(n, f, start=0, window=0, tree=None):
    """[f, n]: whether new token t of a sequence of n tokens, the last f of them new, sees position j"""
    see = np.zeros((f, n), bool)
    for t in range(f):
        for j in range(n):
            new = j - (n - f)
            ok = new < 0 or (bool(tree[t] >> new & 1) if tree is not None else new <= t)
            see[t, j] = ok and j >= start and (window == 0 or j > n - f + t - window)
    return see


def attend(q, keys, values, see, scale):
    """q [f, heads, d], keys and values [kv_heads, n, d], see [f, n].  Returns out, lse, the weighted sum of |values| and the largest
    sum of |q_d k_d| of a visible position (what error bounds need)."""
    f, heads, d = q.shape
    share = heads // keys.shape[0]
    out, lse = np.zeros((f, heads, d)), np.full((f, heads), -np.inf)
    size, reach = np.zeros((f, heads, d)), np.zeros((f, heads))
    for t in range(f):
        j = np.nonzero(see[t])[0]
        if len(j) == 0:
            continue
        for h in range(heads):
            k, v = keys[h // share, j], values[h // share, j]
            s = scale * (k @ q[t, h])
            w = np.exp(s - s.max())
            out[t, h], lse[t, h] = w @ v / w.sum(), s.max() + np.log(w.sum())
            size[t, h] = w @ np.abs(v) / w.sum()
            reach[t, h] = abs(scale) * (np.abs(k) @ np.abs(q[t, h])).max()
    return out, lse, size, reach
