"""Plain 64-bit forms of the paged 8-bit KV cache's operations (numpy, lists).

Nothing here shares code with the library: pages are Python lists, codes are
decoded from a table of the format's 256 values, and attention goes row by row.
"""

from __future__ import annotations

import math

import numpy as np

INT8, FP8 = 0, 1
TOP = {INT8: 127.0, FP8: 448.0}


def code_values(fmt):
    """The number each of the 256 bytes stands for."""
    out = np.empty(256)
    for b in range(256):
        if fmt == INT8:
            out[b] = b - 256 if b > 127 else b
            continue
        sign, e, m = (-1.0 if b & 128 else 1.0), b >> 3 & 15, b & 7
        if e == 15 and m == 7:
            out[b] = math.nan
        else:
            out[b] = sign * (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return out


def block_index(which, tokens, dim):
    """[tokens, dim] byte offsets inside a block (tiles of 16 tokens)."""
    t, d = np.arange(tokens)[:, None], np.arange(dim)[None]
    tile = t // 16 * (16 * dim)
    if which == 0:
        return tile + d // 16 * 256 + t % 16 * 16 + d % 16
    return tile + d * 16 + t % 16


def read(data, scale, geom, table, n, layer, which, head):
    """[n, dim] values of a sequence's keys (which 0) or values (1)."""
    layers, heads, pt, dim, fmt = geom
    idx, val = block_index(which, pt, dim), code_values(fmt)
    out = np.zeros((n, dim))
    for b in range(-(-n // pt)):
        page = int(table[b])
        block = data[page].reshape(layers, 2, heads, pt * dim)[layer, which, head]
        rows = min(pt, n - b * pt)
        out[b * pt:b * pt + rows] = (val[block[idx]] * float(scale[page, layer, which, head]))[:rows]
    return out


def attend(q, ks, vs, scale, causal, window):
    """One head's queries [m, dim] at the last positions of keys ks [n, dim].

    Returns the outputs, lse, and sum_j p_j |v_j| (what errors are relative to)."""
    m, n = q.shape[0], ks.shape[0]
    out, lse, mag = np.zeros(q.shape), np.full(m, -np.inf), np.zeros(q.shape)
    for i in range(m):
        pos = n - m + i
        hi = max(min(pos + 1, n), 0) if causal else n
        lo = max(pos + 1 - window, 0) if window else 0
        if hi <= lo:
            continue
        x = ks[lo:hi] @ q[i] * scale
        top = x.max()
        p = np.exp(x - top)
        lse[i] = top + math.log(p.sum())
        p /= p.sum()
        out[i], mag[i] = p @ vs[lo:hi], p @ np.abs(vs[lo:hi])
    return out, lse, mag


class Pages:
    """Reference counts, lengths and tables as lists; contents by page number."""

    def __init__(self, num_pages, slots, max_blocks, page_tokens):
        self.n, self.max_blocks, self.pt = num_pages, max_blocks, page_tokens
        self.refs = [0] * num_pages
        self.lens = [0] * slots
        self.tables = [[] for _ in range(slots)]
        self.content = [None] * num_pages

    def blocks(self, tokens):
        return -(-tokens // self.pt)

    def fork(self, src, dst, tokens=None):
        for i, (s, d) in enumerate(zip(src, dst)):
            n = self.lens[s] if tokens is None else min(self.lens[s], tokens[i])
            self.tables[d] = self.tables[s][:self.blocks(n)]
            self.lens[d] = n
            for p in self.tables[d]:
                self.refs[p] += 1

    def reserve(self, seqs, tokens):
        """False if there are too few pages (nothing changes)."""
        plan = []
        for s, t in zip(seqs, tokens):
            n = self.lens[s]
            shared = t > 0 and n % self.pt != 0 and self.refs[self.tables[s][-1]] > 1
            plan.append((s, t, shared, self.blocks(n + t) - self.blocks(n)))
        free = [p for p in range(self.n) if self.refs[p] == 0]
        if sum(sh + nb for _, _, sh, nb in plan) > len(free):
            return False
        free = iter(free)
        for s, t, shared, more in plan:
            if shared:
                old, new = self.tables[s][-1], next(free)
                self.content[new] = self.content[old]
                self.tables[s][-1] = new
                self.refs[old] -= 1
                self.refs[new] = 1
            for _ in range(more):
                new = next(free)
                self.tables[s].append(new)
                self.refs[new] = 1
            self.lens[s] += t
        return True

    def free(self, seqs, keep=None):
        for i, s in enumerate(seqs):
            k = 0 if keep is None else min(keep[i], self.lens[s])
            for p in self.tables[s][self.blocks(k):]:
                self.refs[p] -= 1
            self.tables[s] = self.tables[s][:self.blocks(k)]
            self.lens[s] = k

    def compact(self):
        alive = sum(r > 0 for r in self.refs)
        holes = [p for p in range(alive) if self.refs[p] == 0]
        to = {}
        for p in range(alive, self.n):
            if self.refs[p] > 0:
                h = holes[len(to)]
                to[p] = h
                self.refs[h], self.refs[p] = self.refs[p], 0
                self.content[h] = self.content[p]
        self.tables = [[to.get(p, p) for p in t] for t in self.tables]

    def live_words(self):
        words = [0] * (-(-self.n // 32))
        for p, r in enumerate(self.refs):
            if r > 0:
                words[p // 32] |= 1 << (p % 32)
        return words

    def table_rows(self):
        return [t + [-1] * (self.max_blocks - len(t)) for t in self.tables]
