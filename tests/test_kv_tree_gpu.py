"""Attention of trees of drafted tokens against the 64-bit reference, by both of
attention's kernels. Masks and positions are exact; the tolerances of outputs and
sums are those of attention (tests/test_kv_gpu.py), which hold for any set of keys.
"""

import ctypes

import numpy as np
import pytest

from oracle import kv_oracle as ko
from tests.test_kv_gpu import DIMS, Case, dtype_of, i32, kernel, ss  # noqa: F401

pytestmark = pytest.mark.gpu


def random_tree(rng, m, near=5, roots=0.15):
    return [-1 if t == 0 or rng.random() < roots else int(rng.integers(max(0, t - near), t))
            for t in range(m)]


def offsets(new):
    return i32(np.concatenate([[0], np.cumsum(new)]))


def signed(words):
    return np.array(words, np.uint32).astype(np.int32).tolist()


def check_rows(case, q, trees, out, lse, scale):
    """Outputs against the reference, as Case.check does for ranges of keys."""
    import torch
    layers, kvh, pt, dim, fmt = case.geom
    group = q.shape[1] // kvh
    qh, o, sums = q.double().cpu().numpy(), out.double().cpu().numpy(), lse.double().cpu().numpy()
    u = torch.finfo(out.dtype).eps / 2
    at = 0
    for i, parents in enumerate(trees):
        m, n = len(parents), case.lens[i]
        keys = ko.tree_keys(ko.tree(parents)[0], n)
        for kh in range(kvh if m else 0):
            k, v = (ko.read(case.data, case.scale, case.geom, case.tables[i], n, case.layer, w, kh)
                    for w in (0, 1))
            for h in range(kh * group, (kh + 1) * group):
                want, wl, mag = ko.attend(qh[at:at + m, h], k, v, scale, True, 0, keys)
                tol = u * np.abs(want) + 2 * (2.0 ** -12 + 2.0 ** -14) * mag + 2.0 ** -24
                worst = np.max(np.abs(o[at:at + m, h] - want) / tol)
                assert worst <= 1, (i, h, worst)
                got, none = sums[at:at + m, h], np.isinf(wl)
                assert (got[none] == wl[none]).all()
                err = np.abs(got[~none] - wl[~none])
                assert (err <= 2.0 ** -15 * (1 + np.abs(wl[~none]))).all(), err.max()
        at += m


def run(ss, lens, trees, *, heads, kv_heads, dim=128, pt=64, fmt=ko.INT8, dtype="bf16", seed=0,  # noqa: F811
        dirty=False, max_new=None, max_len=0, pad=8):
    import torch
    case = Case(ss, lens, fmt=fmt, dim=dim, pt=pt, kv_heads=kv_heads, seed=seed, dirty=dirty)
    new = [len(t) for t in trees]
    q = case.queries(new, heads, dtype_of(dtype), pad=pad)
    seqs, cu = i32(range(len(lens))), offsets(new)
    mask, positions = case.c.tree(i32([p for t in trees for p in t]), seqs, cu, max_new=max(new))
    most = max(new) if max_new is None else max_new  # (attention's bound need not hold)
    lse = torch.empty(sum(new), heads, device="cuda")
    out = case.c.attend(case.layer, q, seqs, cu, tree=mask, max_new=most, max_len=max_len, lse=lse)
    case.c.check()
    sets = [ko.tree(t) for t in trees]
    assert mask.tolist() == [signed(w) for s, _ in sets for w in ko.tree_words(s, mask.shape[1])]
    assert positions.tolist() == [n - len(t) + d for n, t, (_, depth) in zip(lens, trees, sets)
                                  for d in depth]
    check_rows(case, q, trees, out, lse, dim ** -0.5)
    return case, q, out, lse, mask


@pytest.mark.parametrize("dim,pt", DIMS)
@pytest.mark.parametrize("fmt,dtype", [(ko.INT8, "bf16"), (ko.FP8, "f16"), (ko.INT8, "f16")])
def test_small_trees(ss, dim, pt, fmt, dtype, kernel):  # noqa: F811
    # single tokens, a page and a chunk that end inside the tree, no context, none drafted
    rng = np.random.default_rng(dim + pt)
    lens = [1, 16, 70, 7, 64, 130, 300, 65, 40]
    new = [1, 5, 13, 7, 1, 16, 24, 3, 0]
    print("small trees", dim, pt, fmt, dtype, flush=True)
    run(ss, lens, [random_tree(rng, m) for m in new], heads=4, kv_heads=2, dim=dim, pt=pt, fmt=fmt,
        dtype=dtype, seed=pt)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 1), (17, 1), (8, 1), (6, 3)])
def test_head_groups(ss, heads, kv_heads, kernel):  # noqa: F811
    print("groups", heads, kv_heads, flush=True)
    rng = np.random.default_rng(heads)
    trees = [random_tree(rng, m) for m in (9, 64, 33)]
    run(ss, [300, 64, 90], trees, heads=heads, kv_heads=kv_heads, fmt=ko.FP8, pad=1)


@pytest.mark.parametrize("new", [31, 32, 33, 63, 64, 65, 96, 97, 200])
@pytest.mark.parametrize("old", [0, 1, 17, 63, 64, 100])
def test_word_and_tile_borders(ss, new, old, kernel):  # noqa: F811
    """Trees of more than one and two words at every place of tiles and chunks."""
    print("borders", new, old, flush=True)
    rng = np.random.default_rng(new + old)
    run(ss, [old + new, old + new + 5], [random_tree(rng, new, near=40, roots=0.3)] * 2, heads=2,
        kv_heads=1, dim=64, pt=32, fmt=ko.FP8, dtype="f16", dirty=True, seed=new)


def test_a_wide_and_a_deep_tree(ss, kernel):  # noqa: F811
    """Only roots: a token sees the context and itself. Only a chain: as causal rows."""
    import torch
    print("wide and deep", flush=True)
    run(ss, [200, 300], [[-1] * 150, [-1] + list(range(199))], heads=4, kv_heads=2)
    case, q, out, lse, _ = run(ss, [100, 333], [[-1] + list(range(39)), [-1] + list(range(299))],
                               heads=4, kv_heads=2, dim=64)
    sums = torch.empty_like(lse)
    again = case.c.attend(case.layer, q, i32([0, 1]), i32([0, 40, 340]), lse=sums)
    case.c.check()
    if kernel == "few":  # (the other cuts its tiles' keys at other places)
        assert torch.equal(out, again) and torch.equal(lse, sums)


def test_many_words(ss):  # noqa: F811
    """As many tokens as a mask has bits; more than there are bits."""
    print("many words", flush=True)
    rng = np.random.default_rng(3)
    parents = random_tree(rng, 4096, near=4000, roots=0.01)
    c = ss.KVCache(300, 1, 300, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    c.reserve(i32([0]), i32([4100]))
    mask, positions = c.tree(i32(parents), i32([0]), i32([0, 4096]))
    c.check()
    assert mask.shape == (4096, 128)
    sets, depth = ko.tree(parents)
    some = [0, 1, 31, 32, 2000, 4095]
    assert mask[some].tolist() == [signed(w) for w in ko.tree_words([sets[t] for t in some], 128)]
    assert positions.tolist() == [4 + d for d in depth]
    mask, positions = c.tree(i32(parents[:70]), i32([0]), i32([0, 70]), max_new=64)
    with pytest.raises(ss.SemschedError) as e:
        c.check()
    assert e.value.code == ss.SEM_EINVAL
    assert (mask[64:] == 0).all() and mask[:64].tolist() == [
        signed(w) for w in ko.tree_words(sets[:64], 2)]


def test_more_drafted_tokens_than_keys(ss, kernel):  # noqa: F811
    """Keys before the first are not there, and a row may see none."""
    print("few keys", flush=True)
    rng = np.random.default_rng(1)
    run(ss, [3, 0, 40], [random_tree(rng, 20), random_tree(rng, 4), random_tree(rng, 130)],
        heads=3, kv_heads=1, fmt=ko.FP8)


def test_long_contexts(ss, kernel):  # noqa: F811
    """Contexts that are split into parts, by bounds that hold or do not."""
    print("long", flush=True)
    rng = np.random.default_rng(2)
    trees = [random_tree(rng, m) for m in (37, 3, 0, 1, 64)]
    for max_new, max_len in ((None, 0), (1, 1), (3, 100000)):
        run(ss, [2500, 700, 0, 4100, 1300], trees, heads=4, kv_heads=2, pt=128, fmt=ko.FP8,
            dtype="f16", max_len=max_len, max_new=max_new, seed=11)


def test_many_sequences(ss, kernel):  # noqa: F811
    print("many sequences", flush=True)
    rng = np.random.default_rng(12)
    lens = rng.integers(1, 60, 150).tolist()
    trees = [random_tree(rng, int(rng.integers(0, n + 1)) if rng.random() < 0.7 else 0)
             for n in lens]
    run(ss, lens, trees, heads=2, kv_heads=1, dim=64, pt=16, seed=12)


def test_masks_of_other_shapes(ss, kernel):  # noqa: F811
    """Any bits: rows without themselves, without anything, bits of keys that are not
    there."""
    import torch
    print("any mask", flush=True)
    rng = np.random.default_rng(5)
    for old in (0, 50):
        case = Case(ss, [old + 40], fmt=ko.INT8, dim=64, pt=16, kv_heads=1, seed=old)
        q = case.queries([40], 2, torch.bfloat16)
        words = rng.integers(0, 1 << 32, (40, 2), dtype=np.uint64).astype(np.uint32)
        words[7] = 0
        mask = torch.from_numpy(words.view(np.int32)).cuda()
        lse = torch.empty(40, 2, device="cuda")
        out = case.c.attend(1, q, i32([0]), i32([0, 40]), tree=mask, lse=lse)
        case.c.check()
        keys = [[*range(old), *(old + j for j in range(40) if words[t, j // 32] >> (j % 32) & 1)]
                for t in range(40)]
        k, v = (ko.read(case.data, case.scale, case.geom, case.tables[0], old + 40, 1, w, 0)
                for w in (0, 1))
        for h in (0, 1):
            want, wl, mag = ko.attend(q[:, h].double().cpu().numpy(), k, v, 0.125, True, 0, keys)
            tol = 2.0 ** -8 * np.abs(want) + 2 * (2.0 ** -12 + 2.0 ** -14) * mag + 2.0 ** -24
            assert (np.abs(out[:, h].double().cpu().numpy() - want) <= tol).all()
        if old == 0:
            assert (out[7] == 0).all() and (lse[7] == float("-inf")).all()


def test_hidden_branches_take_no_bits(ss, kernel):  # noqa: F811
    """Pages that a row's mask hides may have V scales of any size."""
    import torch
    print("hidden pages", flush=True)
    # 16 tokens to a page: two branches of 32 tokens each, on pages of their own
    parents = [-1] + list(range(31)) + [-1] + list(range(32, 63))
    case = Case(ss, [64], fmt=ko.INT8, dim=64, pt=16, kv_heads=1, seed=9)
    case.scale[case.tables[0, 2:4], :, 1] *= 1e6
    case.c.scale.copy_(torch.from_numpy(case.scale))
    q = case.queries([64], 2, torch.float16)
    seqs, cu = i32([0]), i32([0, 64])
    mask, _ = case.c.tree(i32(parents), seqs, cu)
    lse = torch.empty(64, 2, device="cuda")
    out = case.c.attend(1, q, seqs, cu, tree=mask, lse=lse)
    case.c.check()
    k, v = (ko.read(case.data, case.scale, case.geom, case.tables[0], 64, 1, w, 0) for w in (0, 1))
    keys = ko.tree_keys(ko.tree(parents)[0], 64)
    want, _, mag = ko.attend(q[:, 0].double().cpu().numpy(), k, v, 0.125, True, 0, keys)
    tol = 2.0 ** -11 * np.abs(want) + 2 * (2.0 ** -12 + 2.0 ** -14) * mag + 2.0 ** -24
    rows = slice(0, 32)  # the other branch's values pass half precision
    assert (np.abs(out[rows, 0].double().cpu().numpy() - want[rows]) <= tol[rows]).all()


def test_starts_and_single_tokens(ss):  # noqa: F811
    print("starts", flush=True)
    c = ss.KVCache(16, 3, 4, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    c.reserve(i32([0, 1, 2]), i32([20, 30, 5]))
    mask, positions = c.tree(i32([-1, -1, -1]), i32([2, 0, 1]), starts=i32([7, -3, 1 << 30]))
    assert mask.tolist() == [[1]] * 3 and positions.tolist() == [7, -3, 1 << 30]
    mask, positions = c.tree(i32([-1, 0, -1]), i32([1, 0]), i32([0, 2, 3]), i32([100, 200]))
    assert mask.tolist() == [[1], [3], [1]] and positions.tolist() == [100, 101, 200]
    mask, positions = c.tree(i32([]), i32([]), i32([0]))
    assert mask.shape[0] == 0 and positions.shape[0] == 0
    c.check()


def test_device_detected_errors(ss, kernel):  # noqa: F811
    import torch
    print("tree errors", flush=True)
    c = ss.KVCache(16, 3, 4, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    c.data.zero_()
    c.reserve(i32([0, 1]), i32([40, 30]))
    q = torch.ones(12, 2, 64, dtype=torch.float16, device="cuda")
    good, seqs, cu = [-1] * 12, i32([0, 1]), i32([0, 5, 12])
    bad = [("a parent of its own", [-1, 1] + good[2:], seqs, cu),
           ("a parent behind", [-1, 4] + good[2:], seqs, cu),
           ("a parent of another sequence", [-1] * 5 + [4] + good[6:], seqs, cu),
           ("a parent below -1", [-2] + good[1:], seqs, cu),
           ("a slot beyond", good, i32([0, 3]), cu),
           ("offsets past the rows", good, seqs, i32([0, 5, 13])),
           ("offsets that fall", good, seqs, i32([0, 14, 12])),
           ("offsets from 1", good, seqs, i32([1, 5, 12]))]
    for name, parents, s, o in bad:
        print(" ", name, flush=True)
        mask, positions = c.tree(i32(parents), s, o)
        with pytest.raises(ss.SemschedError) as e:
            c.check()
        assert e.value.code == ss.SEM_EINVAL, name
    mask, _ = c.tree(i32(good), seqs, cu)
    c.check()
    for s, o in ((i32([0, 3]), cu), (seqs, i32([0, 5, 13])), (seqs, i32([0, 14, 12]))):
        c.attend(0, q, s, o, tree=mask)
        with pytest.raises(ss.SemschedError):
            c.check()
    # more drafted tokens than the masks have bits
    wide = torch.ones(40, 2, 64, dtype=torch.float16, device="cuda")
    mask = torch.full((40, 1), -1, dtype=torch.int32, device="cuda")
    c.attend(0, wide, i32([0]), i32([0, 40]), tree=mask)
    with pytest.raises(ss.SemschedError):
        c.check()
    for tree in (mask[:39], mask.float(), mask.view(-1), mask.cpu(), mask.expand(40, 2)):
        with pytest.raises(ValueError):
            c.attend(0, wide, i32([0]), i32([0, 40]), tree=tree)
    with pytest.raises(ss.SemschedError):
        c.attend(0, wide, i32([0]), i32([0, 40]), tree=mask, causal=False)
    with pytest.raises(ss.SemschedError):
        c.attend(0, wide, i32([0]), i32([0, 40]), tree=mask, window=3)
    c.check()


def test_graph_streams_and_the_blocking_forms(ss, kernel):  # noqa: F811
    import torch
    print("tree graph", flush=True)
    rng = np.random.default_rng(8)
    case = Case(ss, [300, 90], fmt=ko.FP8, dim=64, pt=32, kv_heads=2, seed=8)
    c, new = case.c, [24, 9]
    q = case.queries(new, 4, torch.bfloat16)
    seqs, cu = i32([0, 1]), offsets(new)
    parents = [i32([p for m in new for p in random_tree(rng, m)]) for _ in range(4)]
    mask = torch.empty(33, 1, dtype=torch.int32, device="cuda")
    positions = torch.empty(33, dtype=torch.int32, device="cuda")
    held, out, lse = parents[0].clone(), torch.empty_like(q), torch.empty(33, 4, device="cuda")

    def step(out, lse, mask, positions):
        c.tree(held, seqs, cu, mask=mask, positions=positions)
        c.attend(1, q, seqs, cu, tree=mask, out=out, lse=lse)

    want = [torch.empty_like(t) for t in (out, lse, mask, positions)]
    step(*want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(out, lse, mask, positions)
    torch.cuda.synchronize()
    for a, b in zip((out, lse, mask, positions), want):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, lse, mask, positions)
    for p in parents:
        held.copy_(p)
        graph.replay()
        torch.cuda.synchronize()
        step(*want)
        for a, b in zip((out, lse, mask, positions), want):
            assert torch.equal(a, b)
    c.check()
    L, ref, p = ss.lib, c._ref, (lambda t: ctypes.c_void_p(t.data_ptr()))
    torch.cuda.synchronize()
    L.sem_set_stream(ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    out.zero_(), mask.zero_()
    assert L.sem_kv_tree(ref, p(held), None, p(seqs), p(cu), 2, 33, 1, p(mask), p(positions)) == 0
    query = ss.KVQueryC(q.data_ptr(), out.data_ptr(), lse.data_ptr(), q.stride(0), 64, 256, 64, 33,
                        24, 0, 4, 0, 1, 0, 0.125)
    assert L.sem_kv_attend_tree(ref, 1, ctypes.byref(query), p(mask), 1, p(seqs), p(cu), 2) == 0
    for a, b in zip((out, lse, mask, positions), want):
        assert torch.equal(a, b)
    held[0] = 0
    assert L.sem_kv_tree(ref, p(held), None, p(seqs), p(cu), 2, 33, 1, p(mask),
                         p(positions)) == ss.SEM_EINVAL
