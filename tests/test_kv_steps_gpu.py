"""Steps of a serving loop that use all of it: a tree of drafted tokens is rotated,
appended, attended and cut down to its accepted path, the context is weighed and held to
a budget. Every stage against the 64-bit reference, then the same steps from a graph,
bit for bit. Tolerances are those of the operators' own tests: attention's of
tests/test_kv_gpu.py (the output's rounding and two of the weights').
"""

import numpy as np
import pytest

from oracle import kv_oracle as ko
from tests.test_kv_gpu import i32, ss  # noqa: F401

pytestmark = pytest.mark.gpu

LAYERS, KVH, HEADS, DIM, PT, BUDGET, SINKS, RECENT = 2, 2, 6, 64, 16, 45, 3, 9
TREES = [[-1, 0, 0, 1, 2, 2, 5], [-1, 0, 1, 1]]  # of sequences 2 and 0
PATHS = [[0, 2, 5, 6], [0, 1]]
LENS = [41, 18]


class Loop:
    def __init__(self, ss, fmt):  # noqa: F811
        import torch
        self.ss = ss
        gen = torch.Generator("cuda").manual_seed(11)
        rand = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
        self.c = c = ss.KVCache(32, 3, 12, layers=LAYERS, kv_heads=KVH, head_dim=DIM,
                                page_tokens=PT, format=fmt)
        c.data.zero_()
        self.seqs, self.new = i32([2, 0]), i32([7, 4])
        self.cu, self.parents = i32([0, 7, 11]), i32(sum(TREES, []))
        self.index, self.index_cu = i32(sum(PATHS, [])), i32([0, 4, 6])
        self.freq = 1e4 ** (-torch.arange(DIM // 2, device="cuda").float() / (DIM // 2))
        self.weight = 1 + rand(DIM) / 8
        self.x = rand(LAYERS, 11, HEADS + 2 * KVH, DIM).bfloat16()
        self.next = (2 * rand(LAYERS, 2, HEADS, DIM)).bfloat16()
        self.starts = i32(LENS)  # positions go on whatever leaves
        self.mass = torch.zeros(3, c.max_blocks * PT, device="cuda")
        self.lse = torch.empty(11, HEADS, device="cuda")
        self.last = torch.empty(2, HEADS, device="cuda")
        c.reserve(self.seqs, i32(LENS))
        for layer in range(LAYERS):
            kv = rand(2, sum(LENS), KVH, DIM).bfloat16()
            c.append(layer, kv[0], kv[1], self.seqs, i32([0, LENS[0], sum(LENS)]))
        self.state = (c.book, c.data, c.scale, self.mass, self.starts)

    def draft(self):
        c, out = self.c, []
        c.reserve(self.seqs, self.new)
        mask, positions = c.tree(self.parents, self.seqs, self.cu, self.starts, max_new=7)
        for layer in range(LAYERS):
            x = self.x[layer]
            q, k = self.ss.qk_rotate(x[:, :HEADS], x[:, HEADS:HEADS + KVH], positions, self.freq,
                                     q_weight=self.weight, k_weight=self.weight)
            c.append(layer, k, x[:, HEADS + KVH:], self.seqs, self.cu)
            out.append((q, c.attend(layer, q, self.seqs, self.cu, max_new=7, max_len=64,
                                    tree=mask, lse=self.lse)))
        return positions, out

    def accept(self):
        self.c.keep(self.seqs, self.new, self.index, self.index_cu)
        self.starts += self.index_cu[1:] - self.index_cu[:-1]

    def weigh(self):
        for layer in range(LAYERS):
            q = self.next[layer]
            self.c.attend(layer, q, self.seqs, max_len=64, lse=self.last)
            self.c.weigh(layer, q, self.last, self.mass, self.seqs, max_len=64)

    def bound(self):
        self.c.prune(self.mass, self.seqs, BUDGET, sinks=SINKS, recent=RECENT)

    def host(self):
        c = self.c
        return (c.data.cpu().numpy(), c.scale.cpu().numpy(), c.tables.cpu().numpy(),
                c.lens.tolist(), self.mass.cpu().numpy())


def close(out, want, mag):
    tol = 2.0 ** -8 * np.abs(want) + 2 * (2.0 ** -12 + 2.0 ** -14) * mag + 2.0 ** -24
    assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()


@pytest.mark.parametrize("fmt", [ko.INT8, ko.FP8])
def test_steps(ss, fmt):  # noqa: F811
    import torch
    print("steps", fmt, flush=True)
    loop = Loop(ss, fmt)
    geom, slots, starts = (LAYERS, KVH, PT, DIM, fmt), [2, 0], list(LENS)
    begin = [t.clone() for t in loop.state]
    want = []
    for step in range(7):
        positions, out = loop.draft()
        loop.c.check()
        data, scale, tables, lens, _ = loop.host()
        at = 0
        for i, s in enumerate(slots):
            sets, depth = ko.tree(TREES[i])
            m = len(TREES[i])
            assert positions[at:at + m].tolist() == [starts[i] + d for d in depth]
            keys = ko.tree_keys(sets, lens[s])
            for layer in range(LAYERS):
                q, o = out[layer]
                for h in range(HEADS):
                    k, v = (ko.read(data, scale, geom, tables[s], lens[s], layer, w,
                                    h // (HEADS // KVH)) for w in (0, 1))
                    x, _, mag = ko.attend(q[at:at + m, h].double().cpu().numpy(), k, v,
                                          DIM ** -0.5, True, 0, keys)
                    close(o[at:at + m, h], x, mag)
            at += m
            starts[i] += len(PATHS[i])
        loop.accept()
        got, got_scale, _, now, _ = loop.host()
        for i, s in enumerate(slots):  # (pages that were given back have no numbers any more)
            old = lens[s] - len(TREES[i])
            ko.keep_tokens(data, scale, geom, tables[s], list(range(old)) +
                           [old + j for j in PATHS[i]])
            assert now[s] == old + len(PATHS[i])
            same_tokens(got, got_scale, data, scale, geom, tables[s], now[s])
        loop.weigh()
        data, scale, tables, lens, mass = loop.host()
        loop.bound()
        got, got_scale, _, now, after = loop.host()
        for s in slots:
            chosen = ko.prune_choice(mass[s], lens[s], BUDGET, SINKS, RECENT)
            if lens[s] > BUDGET:
                ko.keep_tokens(data, scale, geom, tables[s], chosen)
            else:
                chosen = list(range(lens[s]))
            assert now[s] == len(chosen) == min(lens[s], BUDGET)
            assert after[s, :now[s]].tolist() == mass[s][chosen].tolist()
            assert (after[s, now[s]:] == 0).all()
            same_tokens(got, got_scale, data, scale, geom, tables[s], now[s])
        loop.c.check()
        want.append([t.clone() for t in loop.state] + [o for _, o in out])
    assert loop.c.lens.tolist() == [32, 0, BUDGET]

    for t, b in zip(loop.state, begin):
        t.copy_(b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = loop.draft()[1]
        loop.accept()
        loop.weigh()
        loop.bound()
    for w in want:
        graph.replay()
        torch.cuda.synchronize()
        for got, x in zip([*loop.state, *(o for _, o in out)], w):
            assert torch.equal(got, x)
    loop.c.check()


def same_tokens(got, got_scale, want, want_scale, geom, table, n):
    for layer in range(LAYERS):
        for w in (0, 1):
            for h in range(KVH):
                a = ko.read(got, got_scale, geom, table, n, layer, w, h)
                b = ko.read(want, want_scale, geom, table, n, layer, w, h)
                assert np.array_equal(a, b)


class Drafts(Loop):
    """Steps whose accepted paths the GPU alone knows: lists of one width, filled up, and the
    accepted rows weighed with the sums of the tree's attention."""

    PATHS = [[[0, 2, 5, 6], [0, 1]], [[], [0, 1, 2]], [[0, 1, 3], []], [[0, 2, 4], [0]],
             [[0], [0, 1, 3]], [[0, 2, 5, 6], [0, 1, 2]]]

    def __init__(self, ss, fmt):  # noqa: F811
        import torch
        super().__init__(ss, fmt)
        self.paths = i32([[p + [-1] * (4 - len(p)) for p in step] for step in self.PATHS])
        self.step, self.width = torch.zeros(1, dtype=torch.int64, device="cuda"), i32([0, 4, 8])
        self.all_lse = torch.empty(LAYERS, 11, HEADS, device="cuda")
        self.place = torch.arange(4, device="cuda")
        self.state = (*self.state, self.step)

    def turn(self):
        import torch
        c = self.c
        c.reserve(self.seqs, self.new)
        mask, positions = c.tree(self.parents, self.seqs, self.cu, self.starts, max_new=7)
        asked = []
        for layer in range(LAYERS):
            x = self.x[layer]
            q, k = self.ss.qk_rotate(x[:, :HEADS], x[:, HEADS:HEADS + KVH], positions, self.freq,
                                     q_weight=self.weight, k_weight=self.weight)
            c.append(layer, k, x[:, HEADS + KVH:], self.seqs, self.cu)
            c.attend(layer, q, self.seqs, self.cu, max_new=7, max_len=64, tree=mask,
                     lse=self.all_lse[layer])
            asked.append(q)
        index = self.paths.index_select(0, self.step)[0]  # (what verification would give)
        self.step += 1
        c.keep(self.seqs, self.new, index.view(-1), self.width)
        there = index >= 0
        count = there.to(torch.int32).sum(1, dtype=torch.int32)
        self.starts += count
        at = self.place - (4 - count)[:, None]  # the rows that stay come last
        rows = self.cu[:-1, None] + index.gather(1, at.clamp(min=0)).clamp(min=0)
        rows, real = rows.view(-1).long(), (at >= 0).view(-1, 1)
        out = []
        for layer in range(LAYERS):
            q = asked[layer].index_select(0, rows)
            lse = self.all_lse[layer].index_select(0, rows).where(real, -float("inf"))
            c.weigh(layer, q, lse, self.mass, self.seqs, self.width, max_new=4, max_len=64)
            out.append((q, lse))
        return out


@pytest.mark.parametrize("fmt", [ko.INT8, ko.FP8])
def test_drafts_within_a_budget(ss, fmt):  # noqa: F811
    import torch
    print("drafts within a budget", fmt, flush=True)
    loop = Drafts(ss, fmt)
    geom, begin, want = (LAYERS, KVH, PT, DIM, fmt), [t.clone() for t in loop.state], []
    for paths in Drafts.PATHS:
        before, old = loop.mass.double().cpu().numpy(), loop.c.lens.tolist()
        out = loop.turn()
        loop.c.check()
        data, scale, tables, lens, mass = loop.host()
        add = np.zeros(mass.shape)
        for i, s in enumerate((2, 0)):
            assert lens[s] == old[s] + len(paths[i])
            for layer in range(LAYERS):
                q, lse = (x[4 * i:4 * i + 4].double().cpu().numpy() for x in out[layer])
                assert np.isfinite(lse).all(1).tolist() == [False] * (4 - len(paths[i])) + [True] * len(
                    paths[i])
                for h in range(HEADS):
                    k = ko.read(data, scale, geom, tables[s], lens[s], layer, 0, h // (HEADS // KVH))
                    add[s, :lens[s]] += ko.weigh(q[:, h], k, DIM ** -0.5, True, 0, lse[:, h])
        assert (np.abs(mass - before - add) <= 2.0 ** -14 * add + 2.0 ** -22 * (before + add)).all()
        loop.bound()
        loop.c.check()
        assert [loop.c.lens.tolist()[s] for s in (2, 0)] == [min(lens[s], BUDGET) for s in (2, 0)]
        want.append([t.clone() for t in loop.state])
    for t, b in zip(loop.state, begin):
        t.copy_(b)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loop.turn()
        loop.bound()
    for w in want:
        graph.replay()
        torch.cuda.synchronize()
        for got, x in zip(loop.state, w):
            assert torch.equal(got, x)
        torch.ones(1000, device="cuda").sum()
    loop.c.check()
