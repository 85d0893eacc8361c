"""Keeping some tokens of sequences against the reference: codes, scales, pages and
lengths are exact (a code is the nearest to a 32-bit quotient, ties to even)."""

import ctypes

import numpy as np
import pytest

from oracle import kv_oracle as ko
from tests.test_kv_gpu import Case, i32, random_codes, ss  # noqa: F401

pytestmark = pytest.mark.gpu


def lists(kept):
    return i32([j for k in kept for j in k]), i32(np.concatenate([[0], np.cumsum(
        [len(k) for k in kept])]))


class Expected:
    """A case's cache after its sequences kept tokens."""

    def __init__(self, case):
        self.case = case
        self.data, self.scale = case.data.copy(), case.scale.copy()
        self.tables, self.lens = case.tables.copy(), list(case.lens)
        self.refs = np.zeros(case.data.shape[0], np.int64)
        for s, n in enumerate(self.lens):
            for p in self.tables[s, :-(-n // case.geom[2])]:
                self.refs[p] += 1

    def keep(self, s, chosen):
        pt = self.case.geom[2]
        ko.keep_tokens(self.data, self.scale, self.case.geom, self.tables[s], chosen)
        for b in range(-(-len(chosen) // pt), -(-self.lens[s] // pt)):
            self.refs[self.tables[s, b]] -= 1
            self.tables[s, b] = -1
        self.lens[s] = len(chosen)

    def check(self):
        c, fmt = self.case.c, self.case.geom[4]
        assert c.lens.tolist() == self.lens and c.refs.tolist() == self.refs.tolist()
        assert np.array_equal(c.tables.cpu().numpy(), self.tables)
        words = [0] * (-(-len(self.refs) // 32))
        for p, r in enumerate(self.refs):
            words[p // 32] |= (r > 0) << (p % 32)
        assert [w & 0xffffffff for w in c.live.tolist()] == words
        assert np.array_equal(c.scale.cpu().numpy(), self.scale)
        data = c.data.cpu().numpy()
        assert ko.same_numbers(data, self.data, fmt)


def path(rng, m, k):
    return sorted(rng.choice(m, min(k, m), replace=False).tolist())


@pytest.mark.parametrize("dim,pt,kv_heads", [(64, 16, 1), (64, 64, 3), (128, 16, 2), (128, 64, 1),
                                             (128, 256, 2), (256, 32, 1), (256, 1024, 1)])
@pytest.mark.parametrize("fmt", [ko.INT8, ko.FP8])
def test_keep(ss, dim, pt, kv_heads, fmt):  # noqa: F811
    """Paths through trees on page borders, all tokens, none, only the end leaving."""
    print("keep", dim, pt, kv_heads, fmt, flush=True)
    rng = np.random.default_rng(dim + pt + fmt)
    lens = [20, 16, 70, 64, 1, 130, 300, 65, 40, 33]
    last = [20, 5, 13, 64, 1, 66, 200, 1, 0, 33]
    kept = [path(rng, 20, 7), [4], [0, 2, 12], path(rng, 64, 30), [], path(rng, 66, 20),
            path(rng, 200, 90), [0], [], list(range(17)) + [20, 30]]
    case = Case(ss, lens, fmt=fmt, dim=dim, pt=pt, kv_heads=kv_heads, layers=2, seed=pt)
    want = Expected(case)
    order = rng.permutation(len(lens)).tolist()
    index, cu = lists([kept[s] for s in order])
    case.c.keep(i32(order), i32([last[s] for s in order]), index, cu)
    case.c.check()
    for s, (n, m) in enumerate(zip(lens, last)):
        want.keep(s, list(range(n - m)) + [n - m + j for j in kept[s]])
    want.check()


@pytest.mark.parametrize("pt", [16, 64])
def test_long_lists(ss, pt):  # noqa: F811
    """Many blocks of one sequence, every density, the first and the last tokens."""
    print("long lists", pt, flush=True)
    rng = np.random.default_rng(pt)
    for share in (0.05, 0.5, 0.97):
        case = Case(ss, [1500, 700], fmt=ko.FP8, dim=64, pt=pt, kv_heads=1, layers=1, layer=0,
                    seed=1)
        want = Expected(case)
        kept = [[t for t in range(n) if rng.random() < share] for n in (1500, 700)]
        index, cu = lists(kept)
        case.c.keep(i32([0, 1]), i32([1500, 700]), index, cu)
        case.c.check()
        for s in (0, 1):
            want.keep(s, kept[s])
        want.check()


def test_equal_scales_keep_their_bytes(ss):  # noqa: F811
    """Codes of blocks of one scale move as they are, whatever byte they are."""
    import torch
    print("equal scales", flush=True)
    for fmt in (ko.INT8, ko.FP8):
        for value in (0.0, 0.7):
            case = Case(ss, [200], fmt=fmt, dim=64, pt=16, kv_heads=2, layers=1, layer=0, seed=2)
            case.data = np.random.default_rng(0).integers(0, 256, case.data.shape).astype(np.uint8)
            case.scale[:] = value
            case.c.data.copy_(torch.from_numpy(case.data))
            case.c.scale.copy_(torch.from_numpy(case.scale))
            want = Expected(case)
            kept = list(range(3, 200, 3))
            index, cu = lists([kept])
            case.c.keep(i32([0]), i32([200]), index, cu)
            case.c.check()
            want.keep(0, kept)
            want.check()
            assert np.array_equal(case.c.data.cpu().numpy(), want.data)


def test_scales_of_every_size(ss):  # noqa: F811
    import torch
    print("scales", flush=True)
    case = Case(ss, [150], fmt=ko.INT8, dim=64, pt=16, kv_heads=1, layers=1, layer=0, seed=3)
    sizes = [2.0 ** -149, 2.0 ** -130, 1e-38, 2.0 ** -70, 1.0, 2.0 ** 60, 2.0 ** 100, 2.0 ** 126, 0]
    for b, size in enumerate(sizes):
        case.scale[case.tables[0, b]] = size
    case.c.scale.copy_(torch.from_numpy(case.scale))
    index, cu = lists([list(range(0, 150, 2))])
    case.c.keep(i32([0]), i32([150]), index, cu)
    case.c.check()
    data, scale, val = case.c.data.cpu().numpy(), case.c.scale.cpu().numpy(), ko.code_values(0)
    for t in range(75):
        at, page = 2 * t, case.tables[0, t // 16]
        src = case.tables[0, at // 16]
        sources = {case.tables[0, u // 16] for u in range(t // 16 * 32, min(t // 16 * 32 + 32, 150))}
        now, was = float(scale[page, 0, 0, 0]), float(case.scale[src, 0, 0, 0])
        assert now == max(float(case.scale[p, 0, 0, 0]) for p in sources)
        idx = ko.block_index(0, 16, 64)
        old = val[case.data[src][:16 * 64][idx[at % 16]]]
        got = val[data[page][:16 * 64][idx[t % 16]]]
        if was == now:
            assert (got == old).all()
        else:  # the nearest code to the quotient
            assert (np.abs(got - old * (was / now)) <= 0.5 + 2.0 ** -16).all()


def test_accepted_tokens_attend_as_before(ss):  # noqa: F811
    """A tree is drafted, its path kept: the context ends as if the path alone had been
    appended."""
    import torch
    print("accept", flush=True)
    gen = torch.Generator("cuda").manual_seed(3)
    parents = [-1, 0, 0, 2, 3, 3, -1, 6]
    kept = [0, 2, 3, 5]
    x = torch.randn(40, 2, 2, 64, generator=gen, device="cuda").clamp(-2, 2).bfloat16()
    x[0, :, :, 0] = 3.0  # (the largest come first: one scale for all)
    x[32:, :, :, 0] = 3.0
    out, books = [], []
    for way in ("tree", "path"):
        c = ss.KVCache(8, 1, 8, layers=1, kv_heads=2, head_dim=64, page_tokens=16)
        c.data.zero_()
        c.reserve(i32([0]), i32([32]))
        c.append(0, x[:32, 0], x[:32, 1], i32([0]), i32([0, 32]))
        rows = x[32:] if way == "tree" else x[32:][kept]
        c.reserve(i32([0]), i32([rows.shape[0]]))
        c.append(0, rows[:, 0], rows[:, 1], i32([0]), i32([0, rows.shape[0]]))
        q = x[32:][kept][:, 0].repeat(1, 2, 1)
        if way == "tree":
            mask, positions = c.tree(i32(parents), i32([0]), i32([0, 8]))
            assert positions[kept].tolist() == [32, 33, 34, 35]
            o = c.attend(0, x[32:, 0].repeat(1, 2, 1), i32([0]), i32([0, 8]), tree=mask)[kept]
            index, cu = lists([kept])
            c.keep(i32([0]), i32([8]), index, cu)
        else:
            o = c.attend(0, q, i32([0]), i32([0, 4]))
        c.check()
        out.append((o, c.attend(0, q, i32([0]), i32([0, 4]))))
        books.append((c.book.clone(), c.scale.clone()))
        c.check()
    assert torch.equal(books[0][0], books[1][0]) and torch.equal(books[0][1], books[1][1])
    assert torch.equal(out[0][1], out[1][1])
    # (in the tree the path's weights are rounded beside other keys': two roundings of
    # the outputs, and of the weights, of magnitudes up to 3)
    assert (out[0][0].double() - out[1][0].double()).abs().max() <= 3 * (2 ** -7 + 2 ** -11)


def test_pages_of_others(ss):  # noqa: F811
    """A shared page is not written: the sequence stays as it was. Pages that only leave
    may be shared."""
    import torch
    print("shared pages", flush=True)

    def fresh():
        c = ss.KVCache(16, 4, 6, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
        c.data.copy_(torch.randint(0, 127, c.data.shape, dtype=torch.uint8, device="cuda"))
        c.scale.uniform_(0.5, 1)
        c.reserve(i32([0, 2]), i32([60, 30]))
        c.fork(i32([0]), i32([1]))
        c.check()
        return c

    c = fresh()
    state = [t.clone() for t in (c.book, c.data, c.scale)]
    index, cu = lists([[1, 3], [0, 5]])
    c.keep(i32([1, 2]), i32([40, 10]), index, cu)
    with pytest.raises(ss.SemschedError) as e:
        c.check()
    assert e.value.code == ss.SEM_EINVAL
    assert c.lens.tolist() == [60, 60, 22, 0]  # the other one is carried out
    assert torch.equal(c.tables[1], state[0][-24:].view(4, 6)[1])
    mine = c.tables[0, :4].long()
    assert torch.equal(c.data[mine], state[1][mine]) and torch.equal(c.scale[mine], state[2][mine])
    c = fresh()  # only the end leaves: nothing is written
    index, cu = lists([[0, 1, 2], []])
    c.keep(i32([1, 0]), i32([40, 60]), index, cu)
    c.check()
    assert c.lens.tolist() == [0, 23, 30, 0] and c.refs.tolist()[:6] == [1, 1, 0, 0, 1, 1]
    c = fresh()  # a branch's own page behind shared ones
    c.reserve(i32([1]), i32([8]))
    index, cu = lists([[1, 4, 7]])
    c.keep(i32([1]), i32([8]), index, cu)
    c.check()
    assert c.lens.tolist() == [60, 63, 30, 0]


def test_device_detected_errors(ss):  # noqa: F811
    import torch
    print("keep errors", flush=True)
    bad = [("a token that is not there", [0], [5], [[0, 5]], None),
           ("a negative token", [0], [5], [[-1, 2]], None),
           ("a list that falls", [0], [5], [[2, 1]], None),
           ("a token twice", [0], [5], [[1, 1]], None),
           ("more than the length", [0], [41], [[1, 2]], None),
           ("a negative count", [0], [-1], [[]], None),
           ("more kept than there are", [0], [1], [[0, 1]], None),
           ("a slot beyond", [4], [5], [[1]], None), ("a negative slot", [-1], [5], [[1]], None),
           ("offsets from 1", [0], [5], [[1, 2]], [1, 2]),
           ("offsets past the list", [0], [5], [[1, 2]], [0, 3]),
           ("offsets that end early", [0], [5], [[1, 2]], [0, 1]),
           ("offsets that fall", [0, 1], [5, 5], [[1, 2], [1]], [0, 4, 3]),
           ("negative offsets", [0], [5], [[1, 2]], [-1, 2])]
    for name, seqs, last, kept, offsets in bad:
        print(" ", name, flush=True)
        c = ss.KVCache(8, 4, 3, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
        c.data.zero_()
        c.reserve(i32([0, 1]), i32([40, 20]))
        c.check()
        book = c.book.clone()
        index, cu = lists(kept)
        c.keep(i32(seqs), i32(last), index, cu if offsets is None else i32(offsets))
        with pytest.raises(ss.SemschedError) as e:
            c.check()
        assert e.value.code == ss.SEM_EINVAL, name
        if offsets is None:
            assert torch.equal(c.book, book), name
        c.check()
    for what in ("page", "length"):
        c = ss.KVCache(8, 4, 3, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
        c.reserve(i32([0]), i32([40]))
        if what == "page":
            c.tables[0, 2] = 1 << 30
        else:
            c.lens[0] = 100
        book = c.book.clone()
        c.keep(i32([0]), i32([40]), *lists([[1, 2]]))
        with pytest.raises(ss.SemschedError):
            c.check()
        assert torch.equal(c.book, book)


def test_a_sequence_twice_and_lists_that_overlap(ss):  # noqa: F811
    """The first one counts, the others are refused."""
    print("keep twice", flush=True)
    for seqs, last, index, cu in (([0, 1, 0], [40, 20, 40], [0, 3, 2, 5, 7], [0, 2, 3, 5]),
                                  ([0, 1, 2], [40, 20, 30], [0, 3, 9, 2], [0, 3, 4, 4]),
                                  ([0, 2, 1], [40, 30, 20], [0, 3, 9, 12], [0, 3, 1, 4])):
        case = Case(ss, [40, 20, 30], fmt=ko.INT8, dim=64, pt=16, kv_heads=2, seed=2)
        case.c.keep(i32(seqs), i32(last), i32(index), i32(cu))
        want, ok, done = Expected(case), True, []
        for i, s in enumerate(seqs):
            lo, hi = cu[i], cu[i + 1]
            if hi < lo or s in done or any(cu[j + 1] > lo for j in range(i)):
                ok = False
                continue
            done.append(s)
            old = case.lens[s] - last[i]
            want.keep(s, list(range(old)) + [old + k for k in index[lo:hi]])
        if ok:
            case.c.check()
        else:
            with pytest.raises(ss.SemschedError) as e:
                case.c.check()
            assert e.value.code == ss.SEM_EINVAL
        want.check()


def test_empty_calls_and_many_sequences(ss):  # noqa: F811
    print("many", flush=True)
    c = ss.KVCache(700, 300, 3, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    none = i32([])
    c.keep(none, none, none, i32([0]))
    rng = np.random.default_rng(4)
    lens = rng.integers(1, 40, 300).tolist()
    c.data.zero_()
    c.reserve(i32(range(300)), i32(lens))
    last = [int(rng.integers(0, n + 1)) for n in lens]
    kept = [path(rng, m, int(rng.integers(0, 5))) for m in last]
    c.keep(i32(range(300)), i32(last), *lists(kept))
    c.check()
    assert c.lens.tolist() == [n - m + len(k) for n, m, k in zip(lens, last, kept)]
    assert int(c.refs.sum()) == sum(-(-n // 16) for n in c.lens.tolist())


def test_graph_streams_and_the_blocking_form(ss):  # noqa: F811
    import torch
    print("keep graph", flush=True)
    case = Case(ss, [100, 70], fmt=ko.FP8, dim=128, pt=16, kv_heads=2, seed=5)
    c = case.c
    kept = [[1, 2, 9], [0, 3, 4, 6]]
    index, cu = lists(kept)
    seqs, last, grow = i32([0, 1]), i32([10, 7]), i32([7, 3])
    start = [t.clone() for t in (c.book, c.data, c.scale)]

    def step():  # the room that was given back is taken again
        c.keep(seqs, last, index, cu)
        c.reserve(seqs, grow)

    want = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            step()
            want.append([t.clone() for t in (c.book, c.data, c.scale)])
        c.check()
        for t, s in zip((c.book, c.data, c.scale), start):
            t.copy_(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for w in want:
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((c.book, c.data, c.scale), w):
            assert torch.equal(a, b)
        torch.ones(1000, device="cuda").sum()
    c.check()
    for t, s in zip((c.book, c.data, c.scale), start):
        t.copy_(s)
    step()
    c.check()
    after = [t.clone() for t in (c.book, c.data, c.scale)]
    for t, s in zip((c.book, c.data, c.scale), start):
        t.copy_(s)
    torch.cuda.synchronize()
    p = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    ss.lib.sem_set_stream(ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert ss.lib.sem_kv_keep(c._ref, p(seqs), p(last), p(index), p(cu), 2, 7) == 0
    c.reserve(seqs, grow)
    c.check()
    for a, b in zip((c.book, c.data, c.scale), after):
        assert torch.equal(a, b)
    last[0] = 1000
    assert ss.lib.sem_kv_keep(c._ref, p(seqs), p(last), p(index), p(cu), 2, 7) == ss.SEM_EINVAL


def padded(kept, width):
    return i32([j for k in kept for j in [*k, *[-1] * (width - len(k))]])


@pytest.mark.parametrize("width", [7, 300])
@pytest.mark.parametrize("fmt", [ko.INT8, ko.FP8])
def test_lists_of_one_width(ss, width, fmt):  # noqa: F811
    """Lists that -1 fills up, wider than what they choose from, too."""
    print("one width", width, flush=True)
    lens, last = [20, 70, 64, 33, 300, 5], [20, 13, 64, 0, 270, 1]
    kept = [[0, 3, 4], [0, 1, 2, 3, 4, 9, 12], [], [], path(np.random.default_rng(1), 270, 6), [0]]
    case = Case(ss, lens, fmt=fmt, dim=64, pt=16, kv_heads=2, seed=width)
    want = Expected(case)
    case.c.keep(i32(range(6)), i32(last), padded(kept, width), i32(range(0, 6 * width + 1, width)))
    case.c.check()
    for s, (n, m) in enumerate(zip(lens, last)):
        want.keep(s, list(range(n - m)) + [n - m + j for j in kept[s]])
    want.check()


def test_what_may_fill_a_list(ss):  # noqa: F811
    import torch
    print("fillers", flush=True)
    for row, ok in (([-1, -1, -1], True), ([2, -1, -1], True), ([0, 1, 4], True),
                    ([-1, 2, -1], False), ([-1, -1, 0], False), ([1, -1, 3], False),
                    ([1, -2, -1], False), ([-2, -1, -1], False), ([1, 1, -1], False),
                    ([3, 2, -1], False), ([5, -1, -1], False), ([0, -1, -2 ** 31], False)):
        case = Case(ss, [40], fmt=ko.FP8, dim=64, pt=16, kv_heads=1, seed=1)
        want, book = Expected(case), case.c.book.clone()
        case.c.keep(i32([0]), i32([5]), i32(row), i32([0, 3]))
        if ok:
            case.c.check()
            want.keep(0, list(range(35)) + [35 + j for j in row if j >= 0])
            want.check()
            continue
        with pytest.raises(ss.SemschedError) as e:
            case.c.check()
        assert e.value.code == ss.SEM_EINVAL, row
        assert torch.equal(case.c.book, book), row


def test_paths_that_the_gpu_alone_knows(ss):  # noqa: F811
    """One graph, other paths in the same buffers for every replay."""
    import torch
    print("paths of a graph", flush=True)
    steps = [[[0, 2, 3], [1]], [[], [0, 1, 2, 3, 5]], [[0, 1, 2, 3, 4], []], [[4], [2, 5]]]
    case = Case(ss, [100, 70], fmt=ko.INT8, dim=64, pt=16, kv_heads=2, seed=4)
    start = [t.clone() for t in (case.c.book, case.c.data, case.c.scale)]
    seqs, last, cu, index = i32([0, 1]), i32([5, 6]), i32([0, 5, 10]), padded([[], []], 5)
    case.c.keep(seqs, last, index, cu)
    case.c.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        case.c.keep(seqs, last, index, cu)
    for kept in steps:
        for t, s in zip((case.c.book, case.c.data, case.c.scale), start):
            t.copy_(s)
        index.copy_(padded(kept, 5))
        want = Expected(case)
        graph.replay()
        torch.cuda.synchronize()
        for s, (n, m) in enumerate(((100, 5), (70, 6))):
            want.keep(s, list(range(n - m)) + [n - m + j for j in kept[s]])
        case.c.check()
        want.check()
        torch.ones(1000, device="cuda").sum()
