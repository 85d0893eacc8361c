"""Attention weights of cached tokens against the 64-bit reference.

Tolerance: scores are off as attention's are (2^-15 for magnitudes below 2^7), and so
is, relatively, a weight; the sum's logarithm is given in 32 bits (2^-24 of its
magnitude, below 2^6) and the exponential is off by a few 2^-23 of its argument. Hence
2^-14 of what a key's weights add up to, and 2^-22 of the sum that they are added to
(a 32-bit addition each for rows and heads).
"""

import ctypes

import numpy as np
import pytest

from oracle import kv_oracle as ko
from tests.test_kv_gpu import Case, dtype_of, i32, ss  # noqa: F401

pytestmark = pytest.mark.gpu


def offsets(new):
    return i32(np.concatenate([[0], np.cumsum(new)]))


def run(ss, lens, new, *, heads, kv_heads, dim=128, pt=64, fmt=ko.INT8, dtype="bf16",  # noqa: F811
        causal=True, window=0, scale=None, seed=0, pad=8, max_len=0, with_cu=True, dirty=False,
        own_lse=False, extra=0, spoil=()):
    import torch
    case = Case(ss, lens, fmt=fmt, dim=dim, pt=pt, kv_heads=kv_heads, seed=seed, dirty=dirty)
    scale = dim ** -0.5 if scale is None else scale
    t, group = sum(new), heads // kv_heads
    q = case.queries(new, heads, dtype_of(dtype), pad=pad)
    seqs, cu = i32(range(len(lens))), offsets(new) if with_cu else None
    if own_lse:  # attention's
        lse = torch.empty(t, heads, device="cuda")
        case.c.attend(case.layer, q, seqs, cu, causal=causal, window=window, scale=scale, lse=lse)
        sums = lse.double().cpu().numpy()
    else:
        sums = np.zeros((t, heads))
    width = case.c.max_blocks * pt + extra
    before = case.rng.random((len(lens), width)).astype(np.float32)
    add = np.zeros((len(lens), width))
    qh = q.double().cpu().numpy()
    at = 0
    for i, m in enumerate(new):
        for kh in range(kv_heads if m and lens[i] else 0):
            k, v = (ko.read(case.data, case.scale, case.geom, case.tables[i], lens[i], case.layer,
                            w, kh) for w in (0, 1))
            for h in range(kh * group, (kh + 1) * group):
                if not own_lse:
                    x = ko.attend(qh[at:at + m, h], k, v, scale, causal, window)[1]
                    sums[at:at + m, h] = x.astype(np.float32)
                    for row, value in spoil:
                        if at <= row < at + m:
                            sums[row, h] = value
                add[i, :lens[i]] += ko.weigh(qh[at:at + m, h], k, scale, causal, window,
                                             sums[at:at + m, h])
        if not lens[i]:
            sums[at:at + m] = -np.inf
        at += m
    if not own_lse:
        lse = torch.from_numpy(sums.astype(np.float32)).cuda()
    mass = torch.from_numpy(before).cuda()
    case.c.weigh(case.layer, q, lse, mass, seqs, cu, causal=causal, window=window, scale=scale,
                 max_len=max_len)
    case.c.check()
    got = mass.double().cpu().numpy()
    want = before.astype(np.float64) + add
    tol = 2.0 ** -14 * add + 2.0 ** -22 * want
    err = np.abs(got - want)
    assert (err <= tol).all(), (err / tol).max()
    for i, n in enumerate(lens):  # nothing behind the keys
        assert np.array_equal(got[i, n:], before[i, n:].astype(np.float64))
    return case, q, lse, mass


DIMS = [(64, 16), (64, 64), (128, 16), (128, 64), (128, 256), (256, 64), (256, 1024)]


@pytest.mark.parametrize("dim,pt", DIMS)
@pytest.mark.parametrize("fmt", [ko.INT8, ko.FP8])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_single_tokens(ss, dim, pt, fmt, dtype):  # noqa: F811
    print("weigh", dim, pt, fmt, dtype, flush=True)
    lens = [1, 15, 16, 17, 63, 64, 65, 0, 200, 129]
    run(ss, lens, [1] * 10, heads=4, kv_heads=2, dim=dim, pt=pt, fmt=fmt, dtype=dtype,
        with_cu=False, seed=dim + pt)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 1), (17, 1), (40, 1), (6, 3), (5, 5),
                                            (9, 9), (32, 16)])
@pytest.mark.parametrize("max_len", [0, 1, 1 << 20])
def test_head_groups(ss, heads, kv_heads, max_len):  # noqa: F811
    print("groups", heads, kv_heads, max_len, flush=True)
    run(ss, [70, 5, 130], [1, 1, 1], heads=heads, kv_heads=kv_heads, fmt=ko.FP8, max_len=max_len)
    run(ss, [70, 5, 130], [9, 5, 33], heads=heads, kv_heads=kv_heads, dtype="f16", dim=64,
        max_len=max_len)


@pytest.mark.parametrize("dim,pt", [(64, 32), (128, 16), (256, 128)])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 1), (True, 50), (False, 0),
                                           (False, 40)])
@pytest.mark.parametrize("fmt,dtype", [(ko.INT8, "bf16"), (ko.FP8, "f16")])
def test_several_tokens(ss, dim, pt, causal, window, fmt, dtype):  # noqa: F811
    print("several", dim, pt, causal, window, flush=True)
    run(ss, [100, 300, 65, 40, 1, 333], [100, 70, 3, 0, 1, 129], heads=4, kv_heads=2, dim=dim,
        pt=pt, fmt=fmt, dtype=dtype, causal=causal, window=window, own_lse=window == 50)


def test_rows_that_see_nothing(ss):  # noqa: F811
    """Queries before the first key, empty sequences, rows that are no numbers."""
    import torch
    print("empty rows", flush=True)
    run(ss, [3, 0, 70], [20, 4, 90], heads=3, kv_heads=1, fmt=ko.FP8)
    run(ss, [0, 0], [1, 3], heads=2, kv_heads=1)
    inf, nan = float("inf"), float("nan")
    for spoil in ([(1, nan)], [(0, inf), (5, -inf)], [(k, nan) for k in range(9)]):
        case, q, lse, mass = run(ss, [50, 40], [4, 5], heads=2, kv_heads=2, dim=64, spoil=spoil)
    q = q.clone()
    q[3, 1, 5], lse[3, 1] = nan, nan  # (as attention returns it)
    mass.zero_()
    case.c.weigh(1, q, lse * 0, mass, i32([0, 1]), i32([0, 4, 9]))
    lse.fill_(nan)
    mass.zero_()
    case.c.weigh(1, q, lse, mass, i32([0, 1]), i32([0, 4, 9]))
    assert (mass == 0).all()
    case.c.check()


def test_bytes_beyond_the_length_do_not_count(ss):  # noqa: F811
    print("dirty", flush=True)
    for fmt in (ko.INT8, ko.FP8):
        run(ss, [41, 100, 64, 77], [3] * 4, heads=4, kv_heads=2, fmt=fmt, dirty=True, pt=32)


def test_strides_and_scales(ss):  # noqa: F811
    print("strides", flush=True)
    run(ss, [90, 33], [2, 30], heads=4, kv_heads=2, pad=1, extra=5)
    run(ss, [90, 33], [2, 30], heads=4, kv_heads=2, scale=-0.3, dtype="f16", pad=3)
    run(ss, [90, 33], [2, 30], heads=4, kv_heads=2, scale=0.0)


def test_many_sequences_and_long_ones(ss):  # noqa: F811
    """More sequences than a wave counts at a time; more pieces than workgroups."""
    print("many", flush=True)
    rng = np.random.default_rng(3)
    lens = rng.integers(0, 60, 150).tolist()
    new = [int(rng.integers(0, n + 1)) if rng.random() < 0.7 else 0 for n in lens]
    run(ss, lens, new, heads=2, kv_heads=1, dim=64, pt=16, max_len=60)
    run(ss, rng.integers(1, 90, 200).tolist(), [1] * 200, heads=2, kv_heads=2, dim=64, pt=16,
        fmt=ko.FP8, with_cu=False)
    run(ss, [70000, 3, 9001], [1, 2, 1], heads=1, kv_heads=1, dim=64, pt=256, max_len=70000)
    run(ss, [70000, 0, 33000], [1, 0, 17], heads=2, kv_heads=2, dim=64, pt=256, fmt=ko.FP8)


@pytest.mark.parametrize("lens", [[800], [20000], [40000, 5], [100000], [9000] * 9])
def test_teams_of_every_size(ss, lens):  # noqa: F811
    """From a few pieces, whose heads are shared out, to more than there are waves; several
    rounds that hardly fill the last one."""
    print("teams", lens, flush=True)
    run(ss, lens, [1] * len(lens), heads=8, kv_heads=4, dim=64, pt=1024, max_len=max(lens))
    run(ss, lens, [3] * len(lens), heads=5, kv_heads=5, dim=64, pt=512, fmt=ko.FP8, dtype="f16")


def test_the_last_queries_alone(ss):  # noqa: F811
    """Weights of the last rows of a prompt, whose attention was called with all."""
    import torch
    print("last rows", flush=True)
    case = Case(ss, [200, 90], fmt=ko.INT8, dim=64, pt=32, kv_heads=2, seed=1)
    q = case.queries([200, 90], 4, torch.bfloat16)
    lse, seqs = torch.empty(290, 4, device="cuda"), i32([0, 1])
    case.c.attend(1, q, seqs, i32([0, 200, 290]), lse=lse)
    rows = list(range(184, 200)) + list(range(280, 290))
    mass = torch.zeros(2, case.c.max_blocks * 32, device="cuda")
    case.c.weigh(1, q[rows], lse[rows].contiguous(), mass, seqs, i32([0, 16, 26]))
    case.c.check()
    got = mass.double().cpu()
    assert np.allclose(got.sum(1), [16 * 4, 10 * 4], rtol=1e-4)  # a row's weights add up to 1
    want = np.zeros((2, got.shape[1]))
    for i, (n, m, at) in enumerate(((200, 16, 184), (90, 10, 280))):
        for h in range(4):
            k = ko.read(case.data, case.scale, case.geom, case.tables[i], n, 1, 0, h // 2)
            want[i, :n] += ko.weigh(q[at:at + m, h].double().cpu().numpy(), k, 0.125, True, 0,
                                    lse[at:at + m, h].double().cpu().numpy())
    assert (np.abs(got.numpy() - want) <= 2.0 ** -14 * want + 1e-12).all()


def test_results_do_not_depend_on_the_run(ss):  # noqa: F811
    import torch
    print("repeat", flush=True)
    case, q, lse, mass = run(ss, [700, 300, 5], [1, 1, 1], heads=8, kv_heads=8, with_cu=False)
    first = torch.zeros_like(mass)
    case.c.weigh(1, q, lse, first, i32([0, 1, 2]))
    for _ in range(5):
        mass.zero_()
        case.c.weigh(1, q, lse, mass, i32([0, 1, 2]))
        assert torch.equal(mass, first)


def test_errors(ss):  # noqa: F811
    import torch
    print("weigh errors", flush=True)
    q = torch.ones(12, 2, 64, dtype=torch.float16, device="cuda")
    lse = torch.zeros(12, 2, device="cuda")

    def fresh():
        c = ss.KVCache(8, 4, 3, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
        c.data.zero_()
        c.reserve(i32([0, 1]), i32([40, 20]))
        c.check()
        return c

    mass = torch.zeros(4, 48, device="cuda")
    for name, seqs, cu in (("a slot beyond", [0, 9], [0, 5, 12]), ("a negative slot", [-1, 1], [0, 5, 12]),
                           ("offsets past the rows", [0, 1], [0, 5, 20]),
                           ("offsets that fall", [0, 1], [0, 14, 12]),
                           ("offsets from 1", [0, 1], [1, 5, 12]),
                           ("offsets that end early", [0, 1], [0, 5, 10])):
        print(" ", name, flush=True)
        c = fresh()
        c.weigh(0, q, lse, mass, i32(seqs), i32(cu))
        with pytest.raises(ss.SemschedError):
            c.check()
    for name, change in (("page", lambda c: c.tables[0, 1].fill_(1 << 30)),
                         ("negative page", lambda c: c.tables[0, 1].fill_(-7)),
                         ("length", lambda c: c.lens[0].fill_(49)),
                         ("negative length", lambda c: c.lens[0].fill_(-1))):
        print(" ", name, flush=True)
        c = fresh()
        change(c)
        c.weigh(0, q, lse, mass, i32([0, 1]), i32([0, 5, 12]))
        with pytest.raises(ss.SemschedError):
            c.check()
    c = fresh()
    for bad in (mass[:3], mass[:, :47], mass.double(), mass.cpu(), mass.t().contiguous().t()):
        with pytest.raises(ValueError):
            c.weigh(0, q, lse, bad, i32([0, 1]), i32([0, 5, 12]))
    for bad in (lse[:5], lse.half(), lse.t().contiguous().t()):
        with pytest.raises(ValueError):
            c.weigh(0, q, bad, mass, i32([0, 1]), i32([0, 5, 12]))
    none = i32([])
    c.weigh(0, q[:0], lse[:0], mass, none)
    c.weigh(0, q[:0], lse[:0], mass, i32([0]), i32([0, 0]))
    c.check()
    c = ss.KVCache(0, 2, 2, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    c.weigh(0, q[:2], lse[:2], torch.zeros(2, 32, device="cuda"), i32([0, 1]))
    c.check()
    c.lens.fill_(3)
    c.weigh(0, q[:2], lse[:2], torch.zeros(2, 32, device="cuda"), i32([0, 1]))
    with pytest.raises(ss.SemschedError):
        c.check()


def test_graph_streams_and_the_blocking_form(ss):  # noqa: F811
    import torch
    print("weigh graph", flush=True)
    case, q, lse, mass = run(ss, [300, 90], [20, 3], heads=4, kv_heads=2, fmt=ko.FP8, own_lse=True)
    c, seqs, cu = case.c, i32([0, 1]), offsets([20, 3])
    mass.zero_()
    want = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            c.weigh(1, q, lse, mass, seqs, cu)
            want.append(mass.clone())
        mass.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.weigh(1, q, lse, mass, seqs, cu)
    for w in want:
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(mass, w)
        torch.ones(1000, device="cuda").sum()
    c.check()
    mass.zero_()
    torch.cuda.synchronize()
    p = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    ss.lib.sem_set_stream(ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    query = ss.KVQueryC(q.data_ptr(), None, lse.data_ptr(), q.stride(0), 128, 0, 0, 23, 0, 0, 4, 0,
                        1, 0, 128 ** -0.5)
    assert ss.lib.sem_kv_weigh(c._ref, 1, ctypes.byref(query), p(seqs), p(cu), 2, p(mass),
                               mass.stride(0)) == 0
    assert torch.equal(mass, want[0])
    cu[1] = 50
    assert ss.lib.sem_kv_weigh(c._ref, 1, ctypes.byref(query), p(seqs), p(cu), 2, p(mass),
                               mass.stride(0)) == ss.SEM_EINVAL


@pytest.mark.parametrize("n,new", [(2, 1), (5, 40), (64, 2), (65, 1), (300, 1), (1200, 1)])
def test_a_sequence_twice(ss, n, new):  # noqa: F811
    """Nothing is added and the call is reported; the same list without it is none."""
    import torch
    print("weigh twice", n, new, flush=True)
    rng = np.random.default_rng(n)
    lens = (new + rng.integers(0, 150, n)).tolist()
    case = Case(ss, lens, fmt=ko.FP8, dim=64, pt=16, kv_heads=2, seed=n)
    cu = None if new == 1 else offsets([new] * n)
    q, lse = case.queries([new] * n, 4, torch.float16), torch.zeros(n * new, 4, device="cuda")
    order = rng.permutation(n)
    before = torch.rand(n, case.c.max_blocks * 16, device="cuda")
    mass = before.clone()
    for first, other in ((0, 1), (0, n - 1), (n // 2 - 1, n // 2), (n - 2, n - 1)):
        seqs = order.copy()
        seqs[other] = seqs[first]
        case.c.weigh(1, q, lse, mass, i32(seqs), cu)
        with pytest.raises(ss.SemschedError) as e:
            case.c.check()
        assert e.value.code == ss.SEM_EINVAL
        assert torch.equal(mass, before)
    case.c.weigh(1, q, lse, mass, i32(order), cu)
    case.c.check()
    assert (mass > before).any(1).all()


def test_a_sequence_twice_among_very_many(ss):  # noqa: F811
    import torch
    print("weigh twice, many slots", flush=True)
    slots = 300000
    c = ss.KVCache(4, slots, 1, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    c.data.zero_()
    c.reserve(i32([5, 131077, 299999]), i32([3, 4, 5]))
    seqs = [5, 131077, 262149, 299999] + list(range(1000, 1096))
    q, lse = torch.zeros(100, 2, 64, device="cuda").half(), torch.zeros(100, 2, device="cuda")
    mass = torch.zeros(slots, 16, device="cuda")
    c.weigh(0, q, lse, mass, i32(seqs))
    c.check()
    assert mass[[5, 131077, 299999]].sum(1).tolist() == [6, 8, 10] and mass.sum() == 24
    for again in (5, 131077, 262149, 299999):
        c.weigh(0, q, lse, mass, i32(seqs[:-1] + [again]))
        with pytest.raises(ss.SemschedError) as e:
            c.check()
        assert e.value.code == ss.SEM_EINVAL and mass.sum() == 24


def test_rows_of_a_tree_after_their_path_was_kept(ss):  # noqa: F811
    """With the lse of the tree's attention the weights of a row that stays add up to 1:
    it sees what its mask showed it. (One scale for all keys, so that they stay the same.)"""
    import torch
    print("rows of a tree", flush=True)
    gen = torch.Generator("cuda").manual_seed(5)
    parents, kept = [-1, 0, 0, 2, 3, 3, -1, 6], [0, 2, 3, 5]
    for fmt, context in ((ko.INT8, 40), (ko.FP8, 75), (ko.INT8, 0)):
        c = ss.KVCache(8, 2, 8, layers=1, kv_heads=2, head_dim=64, page_tokens=16, format=fmt)
        c.data.zero_()
        x = torch.randn(context + 8, 2, 2, 64, generator=gen, device="cuda").clamp(-2, 2).bfloat16()
        x[:, :, :, 0] = 3.0
        q = (2 * torch.randn(8, 4, 64, generator=gen, device="cuda")).bfloat16()
        lse, seqs, cu = torch.empty(8, 4, device="cuda"), i32([1]), i32([0, 8])
        if context:
            c.reserve(seqs, i32([context]))
            c.append(0, x[:context, 0], x[:context, 1], seqs, i32([0, context]))
        c.reserve(seqs, i32([8]))
        c.append(0, x[context:, 0], x[context:, 1], seqs, cu)
        c.attend(0, q, seqs, cu, tree=c.tree(i32(parents), seqs, cu)[0], lse=lse)
        c.keep(seqs, i32([8]), i32(kept + [-1] * 4), cu)
        # rows that the host does not know of before those that stay
        rows = [0] * 4 + kept
        lse = lse[rows].contiguous()
        lse[:4] = -float("inf")
        mass = torch.zeros(2, 128, device="cuda")
        c.weigh(0, q[rows], lse, mass, seqs, cu)
        c.check()
        got = mass.double().cpu().numpy()
        data, scale = c.data.cpu().numpy(), c.scale.cpu().numpy()
        want = np.zeros(context + 4)
        for h in range(4):
            k = ko.read(data, scale, (1, 2, 16, 64, fmt), c.tables[1].tolist(), context + 4, 0, 0,
                        h // 2)
            add = ko.weigh(q[kept, h].double().cpu().numpy(), k, 0.125, True, 0,
                           lse[4:, h].double().cpu().numpy())
            # (four rows' lse and weights, 2^-14 each)
            assert abs(add.sum() - 4) <= 4 * 2.0 ** -13
            want += add
        assert (np.abs(got[1, :context + 4] - want) <= 2.0 ** -14 * want + 1e-12).all()
        assert (got[1, context + 4:] == 0).all() and (got[0] == 0).all()


@pytest.mark.parametrize("new", [1, 4, 40])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_a_query_that_is_no_number_stays_in_its_row(ss, new, dtype):  # noqa: F811
    """Attention gives such a row a sum that is none; the rows beside it weigh as ever."""
    import torch
    print("no number", new, dtype, flush=True)
    case = Case(ss, [50, 90], fmt=ko.FP8, dim=64, pt=16, kv_heads=2, seed=9)
    q = case.queries([new, new], 4, dtype_of(dtype)).clone()
    seqs, cu, lse = i32([0, 1]), offsets([new, new]), torch.empty(2 * new, 4, device="cuda")
    spoiled = [(0, 1), (new, 2), (2 * new - 1, 0)]
    for row, head in spoiled:
        q[row, head, 5] = float("nan")
    case.c.attend(1, q, seqs, cu, lse=lse)
    finite = torch.ones(2 * new, 4, dtype=torch.bool)
    for row, head in spoiled:
        finite[row, head] = False
    assert torch.equal(lse.isfinite().cpu(), finite)
    mass = torch.zeros(2, case.c.max_blocks * 16, device="cuda")
    case.c.weigh(1, q, lse, mass, seqs, cu)
    case.c.check()
    got, want = mass.double().cpu().numpy(), np.zeros(mass.shape)
    qh, sums = q.double().cpu().numpy(), lse.double().cpu().numpy()
    for i, n in enumerate((50, 90)):
        rows = slice(i * new, (i + 1) * new)
        for h in range(4):
            k = ko.read(case.data, case.scale, case.geom, case.tables[i], n, 1, 0, h // 2)
            want[i, :n] += ko.weigh(qh[rows, h], k, 0.125, True, 0, sums[rows, h])
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= 2.0 ** -14 * want + 1e-12).all()
