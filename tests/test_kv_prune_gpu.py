"""Pruning sequences by attention weights against the reference: the tokens that stay,
their codes, scales and weights, pages and lengths are exact."""

import ctypes

import numpy as np
import pytest

from oracle import kv_oracle as ko
from tests.test_kv_gpu import Case, i32, ss  # noqa: F401
from tests.test_kv_keep_gpu import Expected

pytestmark = pytest.mark.gpu


def masses(rng, kind, shape):
    x = rng.lognormal(0, 2, shape)
    if kind == "ties":
        x = np.floor(x)
    elif kind == "equal":
        x = np.full(shape, 0.25)
    elif kind == "signs":
        x = rng.normal(size=shape)
        x[rng.random(shape) < 0.2] = 0.0
        x[rng.random(shape) < 0.2] = -0.0
    elif kind == "wild":
        x[rng.random(shape) < 0.3] = np.nan
        x[rng.random(shape) < 0.1] = np.inf
        x[rng.random(shape) < 0.1] = -np.inf
    elif kind == "close":  # that differ in their last bits
        x = 1 + rng.integers(0, 40, shape) * 2.0 ** -23
    return x.astype(np.float32)


def run(ss, lens, budget, sinks, recent, *, kind="plain", seqs=None, seed=0, extra=0, **geom):  # noqa: F811
    import torch
    case = Case(ss, lens, seed=seed, **geom)
    width = case.c.max_blocks * case.geom[2] + extra
    mass = masses(case.rng, kind, (len(lens), width))
    held = torch.from_numpy(mass).cuda()
    seqs = list(range(len(lens))) if seqs is None else seqs
    case.c.prune(held, i32(seqs), budget, sinks=sinks, recent=recent)
    case.c.check()
    want, left = Expected(case), mass.copy()
    for s in seqs:
        chosen = ko.prune_choice(mass[s], lens[s], budget, sinks, recent)
        want.keep(s, chosen)
        if lens[s] > budget:
            left[s, :lens[s]] = 0
            left[s, :len(chosen)] = mass[s, chosen]
    assert np.array_equal(held.cpu().numpy(), left, equal_nan=True)
    want.check()
    return case, held


SMALL = dict(fmt=ko.INT8, dim=64, pt=16, kv_heads=1, layers=1, layer=0)


@pytest.mark.parametrize("dim,pt,kv_heads,layers", [(64, 16, 2, 2), (128, 64, 1, 2), (128, 32, 3, 1),
                                                    (256, 128, 1, 1)])
@pytest.mark.parametrize("fmt", [ko.INT8, ko.FP8])
@pytest.mark.parametrize("budget,sinks,recent", [(40, 4, 8), (64, 0, 0), (1, 0, 0), (100, 16, 84),
                                                 (33, 50, 3)])
def test_prune(ss, dim, pt, kv_heads, layers, fmt, budget, sinks, recent):  # noqa: F811
    print("prune", dim, pt, fmt, budget, sinks, recent, flush=True)
    run(ss, [300, 40, 41, 64, 0, 1, 129, 101], budget, sinks, recent, fmt=fmt, dim=dim, pt=pt,
        kv_heads=kv_heads, layers=layers, layer=0, seed=pt)


@pytest.mark.parametrize("kind", ["ties", "equal", "signs", "wild", "close"])
@pytest.mark.parametrize("budget,sinks,recent", [(50, 0, 0), (199, 3, 20), (7, 2, 2), (0, 3, 3)])
def test_weights_of_all_kinds(ss, kind, budget, sinks, recent):  # noqa: F811
    print("kinds", kind, budget, flush=True)
    run(ss, [200, 100, 500], budget, sinks, recent, kind=kind, **SMALL)


@pytest.mark.parametrize("n", [1, 15, 16, 17, 1023, 1024, 1025, 4095, 4096, 4097, 9000])
def test_every_length(ss, n):  # noqa: F811
    """Rounds of tokens that end anywhere; one fewer than all, one alone, a half."""
    print("length", n, flush=True)
    for budget in {n - 1, 1, n // 2, n, n + 1}:
        run(ss, [n, 30], budget, 0, 0, kind="ties", seed=n, **SMALL)


def test_a_long_context(ss):  # noqa: F811
    print("long", flush=True)
    run(ss, [60000, 70], 1000, 4, 100, seed=1, **SMALL)
    run(ss, [30000], 20000, 4, 100, kind="ties", seed=2, extra=3, **SMALL)


def test_only_the_end_leaves_and_only_the_first_stay(ss):  # noqa: F811
    """Weights that fall or rise along the tokens; nothing is to move, or all is."""
    import torch
    print("order", flush=True)
    for sign in (1, -1):
        case = Case(ss, [200, 70], seed=4, **SMALL)
        mass = (sign * torch.arange(13 * 16 + 16, 0, -1, device="cuda").float()).repeat(2, 1)
        before = [t.clone() for t in (case.c.data, case.c.scale)]
        kept = mass.cpu().numpy()
        case.c.prune(mass, i32([0, 1]), 50, sinks=0, recent=0)
        case.c.check()
        want = Expected(case)
        for s, n in enumerate((200, 70)):
            want.keep(s, ko.prune_choice(kept[s], n, 50, 0, 0))
        want.check()
        if sign > 0:
            assert torch.equal(case.c.data, before[0]) and torch.equal(case.c.scale, before[1])


def test_listed_sequences_alone(ss):  # noqa: F811
    print("listed", flush=True)
    case, _ = run(ss, [100, 90, 80, 70], 20, 1, 2, seqs=[3, 1], **SMALL)
    assert case.c.lens.tolist() == [100, 20, 80, 20]


def test_shared_pages(ss):  # noqa: F811
    """A sequence whose changing pages are shared stays as it was, its mass too; shared
    pages that only leave are given back."""
    import torch
    print("shared", flush=True)
    c = ss.KVCache(20, 4, 6, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    c.data.copy_(torch.randint(0, 127, c.data.shape, dtype=torch.uint8, device="cuda"))
    c.scale.uniform_(0.5, 1)
    c.reserve(i32([0, 2]), i32([60, 90]))
    c.fork(i32([0]), i32([1]))
    c.check()
    mass = torch.rand(4, 96, device="cuda")
    state = [t.clone() for t in (c.book, c.data, c.scale, mass)]
    c.prune(mass, i32([0, 2]), 30)
    with pytest.raises(ss.SemschedError) as e:
        c.check()
    assert e.value.code == ss.SEM_EINVAL
    assert c.lens.tolist() == [60, 60, 30, 0] and torch.equal(mass[:2], state[3][:2])
    mine = c.tables[0, :4].long()
    assert torch.equal(c.data[mine], state[1][mine]) and torch.equal(c.scale[mine], state[2][mine])
    mass[1] = torch.arange(96, 0, -1, device="cuda")  # its first tokens stay
    c.prune(mass, i32([1]), 17)
    c.check()
    assert c.lens.tolist() == [60, 17, 30, 0]
    assert c.refs[mine].tolist() == [2, 2, 1, 1]


def test_errors(ss):  # noqa: F811
    import torch
    print("prune errors", flush=True)

    def fresh():
        c = ss.KVCache(8, 4, 3, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
        c.data.zero_()
        c.reserve(i32([0, 1]), i32([40, 20]))
        c.check()
        return c

    for name, seqs, change in (
            ("a slot beyond", [4], None), ("a negative slot", [-1], None),
            ("a page beyond", [0], lambda c: c.tables[0, 2].fill_(1 << 30)),
            ("a negative page", [0], lambda c: c.tables[0, 0].fill_(-1)),
            ("a length beyond", [0], lambda c: c.lens[0].fill_(49)),
            ("a negative length", [0], lambda c: c.lens[0].fill_(-1))):
        print(" ", name, flush=True)
        c, mass = fresh(), torch.arange(192, device="cuda").float().view(4, 48)
        if change:
            change(c)
        book, was = c.book.clone(), mass.clone()
        c.prune(mass, i32(seqs), 10)
        with pytest.raises(ss.SemschedError) as e:
            c.check()
        assert e.value.code == ss.SEM_EINVAL
        assert torch.equal(c.book, book) and torch.equal(mass, was)
    c = fresh()
    for bad in (mass[:3], mass[:, :47], mass.double(), mass.cpu()):
        with pytest.raises(ValueError):
            c.prune(bad, i32([0]), 10)
    for sizes in ((-1, 0, 0), (5, -1, 0), (5, 0, -1)):
        with pytest.raises(ss.SemschedError):
            c.prune(mass, i32([0]), sizes[0], sinks=sizes[1], recent=sizes[2])
    c.prune(mass, i32([]), 10)
    c.prune(mass, i32([0]), 1 << 40, sinks=1 << 50, recent=1 << 60)
    c.check()
    assert c.lens.tolist() == [40, 20, 0, 0]


def test_a_sequence_twice(ss):  # noqa: F811
    """The first one counts, the second is refused."""
    import torch
    print("prune twice", flush=True)
    case = Case(ss, [70, 40], fmt=ko.INT8, dim=64, pt=16, kv_heads=2, seed=4)
    mass = torch.rand(2, case.c.max_blocks * 16, device="cuda")
    was = mass.cpu().numpy()
    case.c.prune(mass, i32([0, 1]), 30, sinks=2)
    case.c.prune(mass, i32([1, 1]), 20, sinks=2)
    with pytest.raises(ss.SemschedError) as e:
        case.c.check()
    assert e.value.code == ss.SEM_EINVAL
    want = Expected(case)
    chosen = [ko.prune_choice(was[s], n, 30, 2, 0) for s, n in enumerate([70, 40])]
    left = was[1, chosen[1]]
    then = ko.prune_choice(left, 30, 20, 2, 0)
    want.keep(0, chosen[0])
    want.keep(1, chosen[1])
    want.keep(1, then)
    want.check()
    assert mass.cpu()[1, :20].tolist() == left[then].tolist()
    assert case.c.lens.tolist()[:2] == [30, 20]


def test_weighed_and_pruned_contexts(ss):  # noqa: F811
    """Decode steps that rotate, append, attend and weigh, a prune, and attention over
    what stayed: it is that of the kept tokens."""
    import torch
    print("together", flush=True)
    gen = torch.Generator("cuda").manual_seed(5)
    c = ss.KVCache(64, 2, 16, layers=2, kv_heads=2, head_dim=64, page_tokens=16)
    seqs, one, lens = i32([0, 1]), i32([1, 1]), [180, 100]
    freq = 10000.0 ** (-torch.arange(32, device="cuda").float() / 32)
    mass = torch.zeros(2, 256, device="cuda")
    c.reserve(seqs, i32(lens))
    pos = i32(list(range(180)) + list(range(100)))
    for layer in (0, 1):
        kv = torch.randn(2, 280, 2, 64, generator=gen, device="cuda").bfloat16()
        k = ss.qk_rotate(kv[0], kv[0], pos, freq)[1]
        c.append(layer, k, kv[1], seqs, i32([0, 180, 280]))
    lse = torch.empty(2, 4, device="cuda")
    for step in range(4):
        c.reserve(seqs, one)
        now = i32([180 + step, 100 + step])
        for layer in (0, 1):
            x = torch.randn(2, 8, 64, generator=gen, device="cuda").bfloat16()
            q, k = ss.qk_rotate(4 * x[:, :4], x[:, 4:6], now, freq)
            c.append(layer, k, x[:, 6:], seqs)
            c.attend(layer, q, seqs, lse=lse)
            c.weigh(layer, q, lse, mass, seqs)
    c.check()
    total = mass.sum(1)
    assert torch.allclose(total, torch.full_like(total, 4 * 2 * 4), rtol=1e-4)
    was = mass.cpu().numpy()
    chosen = [ko.prune_choice(was[s], n + 4, 90, 4, 16) for s, n in enumerate(lens)]
    data, scale, tables = c.data.cpu().numpy(), c.scale.cpu().numpy(), c.tables.cpu().numpy()
    geom = (2, 2, 16, 64, ko.INT8)
    c.prune(mass, seqs, 90, sinks=4, recent=16)
    out = c.attend(1, q, seqs, lse=lse)
    c.check()
    assert c.lens.tolist() == [90, 90]
    assert mass.cpu()[:, :90].tolist() == [was[s, chosen[s]].tolist() for s in (0, 1)]
    assert (mass[:, 90:] == 0).all()
    for s in (0, 1):  # (the tolerance of attention: tests/test_kv_gpu.py)
        ko.keep_tokens(data, scale, geom, tables[s], chosen[s])
        for h in range(4):
            k, v = (ko.read(data, scale, geom, tables[s], 90, 1, w, h // 2) for w in (0, 1))
            want, _, mag = ko.attend(q[s, h].double().cpu().numpy()[None], k, v, 0.125, True, 0)
            tol = 2.0 ** -8 * np.abs(want) + 2 * (2.0 ** -12 + 2.0 ** -14) * mag + 2.0 ** -24
            assert (np.abs(out[s, h].double().cpu().numpy() - want[0]) <= tol).all()


def test_graph_streams_and_the_blocking_form(ss):  # noqa: F811
    import torch
    print("prune graph", flush=True)
    case = Case(ss, [100, 70], fmt=ko.FP8, dim=128, pt=16, kv_heads=2, seed=5)
    c, seqs, grow = case.c, i32([0, 1]), i32([40, 10])
    mass = torch.rand(2, case.c.max_blocks * 16, device="cuda")
    state = (c.book, c.data, c.scale, mass)
    start = [t.clone() for t in state]

    def step():
        c.prune(mass, seqs, 60, sinks=2, recent=10)
        c.reserve(seqs, grow)

    want = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            step()
            want.append([t.clone() for t in state])
        c.check()
        for t, s in zip(state, start):
            t.copy_(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for w in want:
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(state, w):
            assert torch.equal(a, b)
        torch.ones(1000, device="cuda").sum()
    c.check()
    for t, s in zip(state, start):
        t.copy_(s)
    torch.cuda.synchronize()
    p = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    ss.lib.sem_set_stream(ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert ss.lib.sem_kv_prune(c._ref, p(mass), mass.stride(0), p(seqs), 2, 60, 2, 10) == 0
    c.reserve(seqs, grow)
    c.check()
    for a, b in zip(state, want[0]):
        assert torch.equal(a, b)
    c.lens[0] = -4
    assert ss.lib.sem_kv_prune(c._ref, p(mass), mass.stride(0), p(seqs), 2, 60, 2,
                               10) == ss.SEM_EINVAL
