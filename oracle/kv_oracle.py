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


def visible(m, n, i, causal, window):
    """The keys that query i of m sees of n, as a range."""
    pos = n - m + i
    hi = max(min(pos + 1, n), 0) if causal else n
    lo = max(pos + 1 - window, 0) if window else 0
    return range(lo, max(hi, lo))


def attend(q, ks, vs, scale, causal, window, seen=None):
    """One head's queries [m, dim] at the last positions of keys ks [n, dim]; `seen`
    lists the keys of each query instead.

    Returns the outputs, lse, and sum_j p_j |v_j| (what errors are relative to)."""
    m, n = q.shape[0], ks.shape[0]
    out, lse, mag = np.zeros(q.shape), np.full(m, -np.inf), np.zeros(q.shape)
    for i in range(m):
        keys = list(visible(m, n, i, causal, window) if seen is None else seen[i])
        if not keys:
            continue
        x = ks[keys] @ q[i] * scale
        top = x.max()
        p = np.exp(x - top)
        lse[i] = top + math.log(p.sum())
        p /= p.sum()
        out[i], mag[i] = p @ vs[keys], p @ np.abs(vs[keys])
    return out, lse, mag


def weigh(q, ks, scale, causal, window, lse):
    """What one head's queries [m, dim] add to the weights of keys ks [n, dim]; rows whose
    lse is not finite add nothing."""
    m, n = q.shape[0], ks.shape[0]
    out = np.zeros(n)
    for i in range(m):
        keys = list(visible(m, n, i, causal, window))
        if keys and math.isfinite(lse[i]):
            out[keys] += np.exp(ks[keys] @ q[i] * scale - lse[i])
    return out


def tree(parents):
    """(the sets of tokens that each of a sequence's drafted tokens continues, itself
    among them, their depths)."""
    sets, depth = [], []
    for t, p in enumerate(parents):
        sets.append({t} | (sets[p] if p >= 0 else set()))
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return sets, depth


def tree_words(sets, words):
    """Masks of such sets, 32 bits to a word."""
    return [[sum(1 << (j % 32) for j in s if j // 32 == w) for w in range(words)] for s in sets]


def tree_keys(sets, n):
    """The keys of n that tokens of such sets see."""
    m = len(sets)
    return [[*range(n - m), *(n - m + j for j in sorted(s) if n - m + j >= 0)] for s in sets]


def rotate(x, w, eps, positions, inv_freq, interleaved):
    """Rows x [tokens, heads, dim] normed and turned: (y, the two sides' magnitudes that
    the errors of an element are relative to)."""
    x = np.asarray(x, np.float64)
    tokens, _, dim = x.shape
    half = len(inv_freq)
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(w, np.float64)
    out, mag = x.copy(), np.abs(x)
    for t in range(tokens):
        for i in range(half):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            angle = math.fmod(int(positions[t]) * float(inv_freq[i]), 2 * math.pi)
            c, s = math.cos(angle), math.sin(angle)
            out[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
            out[t, :, b] = x[t, :, b] * c + x[t, :, a] * s
            mag[t, :, a] = mag[t, :, b] = np.abs(x[t, :, a]) + np.abs(x[t, :, b])
    return out, mag


def prune_choice(mass, n, budget, sinks, recent):
    """The tokens of n that stay, ascending."""
    if n <= budget:
        return list(range(n))
    a = min(sinks, budget)
    r = min(recent, budget - a)
    key = [-math.inf if math.isnan(x) else float(x) for x in mass[:n]]
    nan = [math.isnan(x) for x in mass[:n]]
    rest = sorted(range(a, n - r), key=lambda t: (nan[t], -key[t], t))[:budget - a - r]
    return sorted([*range(a), *rest, *range(n - r, n)])


def requantized(codes, was, now, fmt):
    """Bytes of a block of scale `was` on scale `now`: the nearest codes to the 32-bit
    quotients, ties to the even one."""
    val = code_values(fmt)
    x = val[codes].astype(np.float32) * np.float32(was) / np.float32(now)
    order = [b for b in np.argsort(val, kind="stable") if not math.isnan(val[b])]
    order = [b for b in order if b != 128]  # -128 is not a code; minus zero counts as zero
    steps = val[order]
    x64 = np.clip(x.astype(np.float64), steps[0], steps[-1])
    hi = np.clip(np.searchsorted(steps, x64), 1, len(steps) - 1)
    lo = hi - 1
    up, down = steps[hi] - x64, x64 - steps[lo]
    even = np.array([b % 2 == 0 for b in order])
    pick = np.where((up < down) | ((up == down) & even[hi]), hi, lo)
    return np.array(order, np.uint8)[pick]


def keep_tokens(data, scale, geom, table, chosen):
    """Moves the tokens `chosen` (old positions, ascending) of one sequence to its front,
    in place; returns the blocks that changed."""
    layers, heads, pt, dim, fmt = geom
    moved = [t for t, at in enumerate(chosen) if t != at]
    if not moved:
        return range(0)
    blocks = range(moved[0] // pt, -(-len(chosen) // pt))
    old_data, old_scale = data.copy(), scale.copy()

    def block(of, page, layer, w, h):
        return of[page].reshape(layers, 2, heads, pt * dim)[layer, w, h]

    for b in blocks:
        tokens = chosen[b * pt:(b + 1) * pt]
        for layer in range(layers):
            for w in (0, 1):
                idx = block_index(w, pt, dim)
                for h in range(heads):
                    pages = [int(table[at // pt]) for at in tokens]
                    now = max(float(old_scale[p, layer, w, h]) for p in pages)
                    scale[int(table[b]), layer, w, h] = now
                    to = block(data, int(table[b]), layer, w, h)
                    for t, (at, page) in enumerate(zip(tokens, pages)):
                        was = float(old_scale[page, layer, w, h])
                        codes = block(old_data, page, layer, w, h)[idx[at % pt]]
                        if was != now:
                            codes = requantized(codes, was, now, fmt)
                        to[idx[t]] = codes
    return blocks


def same_numbers(a, b, fmt):
    """Whether bytes stand for the same numbers (either zero, any NaN)."""
    val = code_values(fmt)
    return np.array_equal(val[a], val[b], equal_nan=True)


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
