"""The paged 8-bit KV cache against its 64-bit reference.

Page numbers, counts and copies are exact. Tolerances:
  * attention: a weight p_j vs_j is rounded to 11 bits (relative 2^-12, to the
    nearest), scores and sums carry 32-bit errors (a score of magnitude below
    2^7 is off by at most 2^-15, and so is its weight, relatively), and the output
    is rounded to its type. Hence |error| <= u |o| + (2^-12 + 2^-14) sum_j p_j |v_j|
    + tiny, with u the type's half unit, 2^-9 (bf16) or 2^-12 (half), both doubled
    for slack.
  * a scale is one 32-bit product, a code the nearest to a 32-bit quotient: it
    is off by at most half a step, plus 2^-20 of the largest code.
"""

import numpy as np
import pytest

from oracle import kv_oracle as ko
from tests._lib import ensure_built, gpu_available

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ss():
    ensure_built()
    if not gpu_available():
        pytest.skip("no GPU")
    import paper_2506_12204_amd as mod
    return mod


@pytest.fixture(params=["few", "tile"])
def kernel(request, monkeypatch):
    """Attention's two kernels, each at sizes that the other is chosen for."""
    monkeypatch.setenv("SEMSCHED_KV_TILES", "1" if request.param == "tile" else "0")
    return request.param


def i32(x):
    import torch
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


def random_codes(rng, shape, fmt):
    if fmt == ko.INT8:
        return rng.integers(-127, 128, shape).astype(np.int8).view(np.uint8)
    b = rng.integers(0, 256, shape).astype(np.uint8)
    return np.where((b & 127) == 127, b - 1, b).astype(np.uint8)


class Case:
    """A cache with sequences of given lengths on scattered pages."""

    def __init__(self, ss, lens, *, fmt, dim, pt, kv_heads, layers=2, layer=1, seed=0, spare=3,
                 dirty=False):
        import torch
        rng = self.rng = np.random.default_rng(seed)
        self.lens, self.layer = lens, layer
        blocks = [-(-n // pt) for n in lens]
        pages, mb = sum(blocks) + spare, max(blocks + [1]) + 1
        self.geom = (layers, kv_heads, pt, dim, fmt)
        self.c = ss.KVCache(pages, len(lens), mb, layers=layers, kv_heads=kv_heads, head_dim=dim,
                            page_tokens=pt, format=fmt)
        self.data = random_codes(rng, (pages, self.c.page_bytes), fmt)
        if dirty:  # bytes that no sequence holds may be anything, NaN codes too
            self.data[:] = 0x7f if fmt == ko.FP8 else 0x80
            good = random_codes(rng, self.data.shape, fmt)
        self.scale = np.exp(rng.normal(size=(pages, layers, 2, kv_heads))).astype(np.float32)
        self.scale *= 1 / 64 if fmt == ko.INT8 else 1 / 200
        perm = rng.permutation(pages)
        self.tables = np.full((len(lens), mb), -1, np.int32)
        at = 0
        for s, nb in enumerate(blocks):
            self.tables[s, :nb] = perm[at:at + nb]
            at += nb
            if dirty:
                for b in range(nb):
                    rows = min(pt, lens[s] - b * pt)
                    p = perm[at - nb + b]
                    view = self.data[p].reshape(layers, 2, kv_heads, pt * dim)
                    new = good[p].reshape(layers, 2, kv_heads, pt * dim)
                    for w in (0, 1):
                        idx = ko.block_index(w, pt, dim)[:rows].reshape(-1)
                        view[:, w][..., idx] = new[:, w][..., idx]
        refs = np.zeros(pages, np.int32)
        refs[perm[:at]] = 1
        self.c.data.copy_(torch.from_numpy(self.data))
        self.c.scale.copy_(torch.from_numpy(self.scale))
        self.c.tables.copy_(torch.from_numpy(self.tables))
        self.c.lens.copy_(i32(lens))
        self.c.refs.copy_(i32(refs))
        words = np.zeros(-(-pages // 32), np.uint32)
        for p in perm[:at]:
            words[p // 32] |= np.uint32(1 << (p % 32))
        self.c.live.copy_(torch.from_numpy(words.view(np.int32)))

    def queries(self, new, heads, dtype, big=False, pad=0):
        import torch
        dim = self.geom[3]
        x = self.rng.normal(size=(sum(new), heads * dim + pad))
        if big:  # magnitudes that half precision does not hold
            x = x * 2.0 ** self.rng.integers(-40, 40, (sum(new), 1))
        t = torch.from_numpy(x).to(dtype).cuda()
        return t[:, :heads * dim].view(sum(new), heads, dim)

    def check(self, q, new, out, lse, scale, causal, window, seqs=None):
        import torch
        layers, kvh, pt, dim, fmt = self.geom
        group = q.shape[1] // kvh
        qh, o = q.double().cpu().numpy(), out.double().cpu().numpy()
        u = 2.0 ** -9 if out.dtype == torch.bfloat16 else 2.0 ** -12
        at = 0
        for i, m in enumerate(new):
            s = i if seqs is None else seqs[i]
            for kh in range(kvh):
                k, v = (ko.read(self.data, self.scale, self.geom, self.tables[s], self.lens[s],
                                self.layer, w, kh) for w in (0, 1))
                for h in range(kh * group, (kh + 1) * group):
                    want, wl, mag = ko.attend(qh[at:at + m, h], k, v, scale, causal, window)
                    got = o[at:at + m, h]
                    tol = 2 * (u * np.abs(want) + (2.0 ** -12 + 2.0 ** -14) * mag) + 2.0 ** -24
                    worst = np.max((np.abs(got - want) / tol)) if m else 0
                    assert worst <= 1, (i, h, worst)
                    if lse is not None:
                        gl = lse[at:at + m, h].double().cpu().numpy()
                        none = np.isinf(wl)
                        assert (gl[none] == wl[none]).all()
                        err = np.abs(gl[~none] - wl[~none])
                        assert (err <= 2.0 ** -15 * (1 + np.abs(wl[~none]))).all(), err.max()
            at += m


def dtype_of(name):
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16}[name]


def run_attend(ss, lens, new, *, heads, kv_heads, dim=128, pt=64, fmt=ko.INT8, dtype="bf16",
               causal=True, window=0, scale=None, seed=0, big=False, pad=8, max_len=0, max_new=0,
               with_cu=True, dirty=False, lse=True, strided_out=False):
    import torch
    case = Case(ss, lens, fmt=fmt, dim=dim, pt=pt, kv_heads=kv_heads, seed=seed, dirty=dirty)
    scale = dim ** -0.5 if scale is None else scale
    q = case.queries(new, heads, dtype_of(dtype), big, pad)
    if big:
        scale *= 2.0 ** -40
    t = sum(new)
    out = None
    if strided_out:
        out = torch.full((t, heads + 1, dim), 7.0, dtype=q.dtype, device="cuda")[:, :heads]
    sums = torch.empty(t, heads, device="cuda") if lse else None
    cu = i32(np.concatenate([[0], np.cumsum(new)])) if with_cu else None
    out = case.c.attend(case.layer, q, i32(range(len(lens))), cu, causal=causal, window=window,
                        scale=scale, max_len=max_len, max_new=max_new, out=out, lse=sums)
    case.c.check()
    case.check(q, new, out, sums, scale, causal, window)
    if strided_out:
        assert (out.as_strided((t, dim), (out.stride(0), 1),
                               out.storage_offset() + heads * dim) == 7.0).all()
    return case, q, out


DIMS = [(64, 16), (64, 64), (128, 16), (128, 32), (128, 64), (128, 256), (256, 64), (256, 1024)]


@pytest.mark.parametrize("dim,pt", DIMS)
@pytest.mark.parametrize("fmt", [ko.INT8, ko.FP8])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_single_tokens(ss, dim, pt, fmt, dtype, kernel):
    # one key, tile and chunk borders, a page that ends inside a chunk, an idle slot
    lens = [1, 15, 16, 17, 63, 64, 65, 0, 200, 129]
    print("decode", dim, pt, fmt, dtype, flush=True)
    run_attend(ss, lens, [1] * len(lens), heads=4, kv_heads=2, dim=dim, pt=pt, fmt=fmt,
               dtype=dtype, with_cu=False, seed=dim + pt + fmt)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 1), (16, 1), (17, 1), (40, 1), (6, 3),
                                            (5, 5)])
def test_head_groups(ss, heads, kv_heads, kernel):
    print("groups", heads, kv_heads, flush=True)
    run_attend(ss, [70, 5, 130], [1, 1, 1], heads=heads, kv_heads=kv_heads, fmt=ko.FP8)
    run_attend(ss, [70, 5, 130], [9, 5, 33], heads=heads, kv_heads=kv_heads, dtype="f16")


@pytest.mark.parametrize("split", [0, 1, 4000])
@pytest.mark.parametrize("fmt", [ko.INT8, ko.FP8])
def test_long_contexts(ss, split, fmt, kernel):
    # few rows: the key axis is split, by a bound that may be wrong either way
    print("long", split, fmt, flush=True)
    run_attend(ss, [3001, 17, 4000, 0], [1] * 4, heads=2, kv_heads=1, fmt=fmt, max_len=split,
               with_cu=False, seed=5)


@pytest.mark.parametrize("dim,pt", [(64, 32), (128, 16), (128, 64), (256, 128)])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 1), (True, 50), (False, 0),
                                           (False, 40)])
@pytest.mark.parametrize("fmt,dtype", [(ko.INT8, "bf16"), (ko.FP8, "f16")])
def test_several_tokens(ss, dim, pt, causal, window, fmt, dtype, kernel):
    # whole prompts, chunks on a context, drafts, a sequence without queries
    lens, new = [100, 300, 65, 40, 1, 333], [100, 70, 3, 0, 1, 129]
    print("several", dim, pt, causal, window, fmt, flush=True)
    run_attend(ss, lens, new, heads=4, kv_heads=2, dim=dim, pt=pt, fmt=fmt, dtype=dtype,
               causal=causal, window=window, seed=window + dim)


@pytest.mark.parametrize("causal", [True, False])
def test_more_queries_than_keys(ss, causal, kernel):
    # rows before the first key see nothing: zeros, and a sum of minus infinity
    print("empty rows", causal, flush=True)
    run_attend(ss, [3, 0, 70], [20, 4, 200], heads=3, kv_heads=1, causal=causal, fmt=ko.FP8)


@pytest.mark.parametrize("fmt", [ko.INT8, ko.FP8])
@pytest.mark.parametrize("new", [1, 40])
def test_bytes_beyond_the_length_do_not_count(ss, fmt, new, kernel):
    print("dirty", fmt, new, flush=True)
    lens = [41, 100, 64, 77]
    run_attend(ss, lens, [new] * 4, heads=4, kv_heads=2, fmt=fmt, dirty=True, pt=32)


def test_magnitudes_and_strides(ss, kernel):
    print("magnitudes", flush=True)
    run_attend(ss, [90, 33], [2, 30], heads=4, kv_heads=2, big=True)
    # rows that are not 16-byte aligned, an output with a stride
    run_attend(ss, [90, 33], [2, 30], heads=4, kv_heads=2, pad=1, strided_out=True)
    run_attend(ss, [90, 33], [1, 1], heads=4, kv_heads=2, pad=3, dtype="f16", strided_out=True)
    run_attend(ss, [90, 33], [1, 1], heads=4, kv_heads=2, scale=0.0)
    run_attend(ss, [90, 33], [1, 9], heads=4, kv_heads=2, scale=-0.3)


def test_scales_of_very_different_pages(ss, kernel):
    """Weights are rounded relative to the largest V scale, zero scales included."""
    import torch
    print("page scales", flush=True)
    for new in (1, 50):
        case = Case(ss, [300, 200], fmt=ko.INT8, dim=64, pt=16, kv_heads=1, seed=3)
        mult = 10.0 ** case.rng.integers(-6, 4, case.scale.shape[0])
        mult[case.tables[0, 0]] = 0.0
        case.scale[:, :, 1] *= mult[:, None, None].astype(np.float32)
        case.c.scale.copy_(torch.from_numpy(case.scale))
        q = case.queries([new, new], 2, torch.bfloat16)
        out = case.c.attend(1, q, i32([0, 1]), i32([0, new, 2 * new]))
        case.c.check()
        case.check(q, [new, new], out, None, 64 ** -0.5, True, 0)
    # all of V zero
    case.scale[:, :, 1] = 0
    case.c.scale.copy_(torch.from_numpy(case.scale))
    assert (case.c.attend(1, q, i32([0, 1]), i32([0, new, 2 * new])) == 0).all()


def test_nan_and_infinity_of_a_query_stay_in_its_row(ss, kernel):
    import torch
    print("nan rows", flush=True)
    case = Case(ss, [130], fmt=ko.FP8, dim=64, pt=32, kv_heads=1)
    q = case.queries([40], 1, torch.float16).clone()
    ref = case.c.attend(1, q, i32([0]), i32([0, 40]))
    q[7, 0, 3], q[20, 0, 0] = float("nan"), float("inf")
    out = case.c.attend(1, q, i32([0]), i32([0, 40]))
    case.c.check()
    rows = [i for i in range(40) if i not in (7, 20)]
    assert torch.equal(out[rows], ref[rows])
    assert out[7].isnan().all()


def test_page_offsets_beyond_32_bits(ss):
    """A pool of more than 4 GiB, read and written beyond that."""
    import torch
    print("large pool", flush=True)
    c = ss.KVCache(1100, 2, 8, layers=8, kv_heads=16, head_dim=256, page_tokens=64,
                   format=ss.KV_INT8)
    assert c.data.numel() > 1 << 32
    c.tables[0, :2] = i32([1098, 1099])
    c.refs[1098:1100] = 1
    c.live[1098 // 32] = (1 << (1098 % 32)) | (1 << (1099 % 32))
    c.lens[0] = 70
    gen = torch.Generator("cuda").manual_seed(1)
    kv = torch.randn(2, 70, 16, 256, generator=gen, device="cuda").bfloat16()
    c.append(7, kv[0], kv[1], i32([0]), i32([0, 70]))
    q = torch.randn(1, 16, 256, generator=gen, device="cuda").bfloat16()
    out = c.attend(7, q, i32([0])).clone()
    c.compact()
    again = c.attend(7, q, i32([0]))
    c.check()
    assert c.tables[0, :2].tolist() == [0, 1] and c.refs[:3].tolist() == [1, 1, 0]
    assert torch.equal(out, again)
    k, v = kv.double().cpu().numpy()
    for h in range(16):
        want, _, mag = ko.attend(q[:, h].double().cpu().numpy(), k[:, h], v[:, h], 1 / 16, True, 0)
        # int8 keys and values: half a step of 1/127 of the largest each
        assert np.abs(again[0, h].double().cpu().numpy() - want).max() < 0.1


@pytest.mark.parametrize("dim,heads,kv_heads", [(64, 6, 2), (128, 5, 1), (256, 4, 4)])
@pytest.mark.parametrize("max_len,max_new", [(0, 0), (1, 1), (100000, 3)])
def test_parts_of_longer_contexts(ss, kernel, dim, heads, kv_heads, max_len, max_new):
    """Ragged chunks over contexts that are split into parts, by bounds that hold
    or do not; a sum of each row."""
    print("parts", kernel, dim, max_len, max_new, flush=True)
    run_attend(ss, [2500, 700, 0, 4100, 1300], [37, 3, 0, 1, 80], heads=heads, kv_heads=kv_heads,
               dim=dim, pt=128, fmt=ko.FP8, dtype="f16", max_len=max_len, max_new=max_new, seed=11)


def test_many_sequences(ss, kernel):
    """More sequences than a wave counts at a time, some without queries."""
    print("many sequences", kernel, flush=True)
    rng = np.random.default_rng(12)
    lens = rng.integers(0, 60, 150).tolist()
    new = [int(rng.integers(0, n + 1)) if rng.random() < 0.7 else 0 for n in lens]
    run_attend(ss, lens, new, heads=2, kv_heads=1, dim=64, pt=16, fmt=ko.INT8, seed=12)
    # one token each, through offsets and without
    lens = rng.integers(1, 90, 200).tolist()
    for with_cu in (True, False):
        run_attend(ss, lens, [1] * 200, heads=2, kv_heads=2, dim=64, pt=16, fmt=ko.FP8,
                   with_cu=with_cu, max_new=1, seed=13)


def test_rounds_of_tiles(ss, kernel):
    """More row tiles than the device has compute units, many times over, and
    as many equal ones as it has."""
    print("rounds", kernel, flush=True)
    rng = np.random.default_rng(14)
    new = [int(x) for x in rng.integers(60, 72, 24)]
    lens = [n + int(x) for n, x in zip(new, rng.integers(0, 40, 24))]
    run_attend(ss, lens, new, heads=256, kv_heads=16, dim=64, pt=32, fmt=ko.INT8, seed=14)
    run_attend(ss, [900] * 8, [16] * 8, heads=256, kv_heads=16, dim=64, pt=128, fmt=ko.FP8,
               seed=15)


def test_all_queries_hidden(ss, kernel):
    """A call in which no row sees a key."""
    import torch
    print("hidden", kernel, flush=True)
    case, q, out = run_attend(ss, [0, 0], [3, 40], heads=4, kv_heads=2)
    assert (out == 0).all() and not torch.signbit(out).any()


def test_rows_of_equal_scores_are_means(ss, kernel):
    """Zero keys (blocks of scale zero): every visible value has the same weight."""
    import torch
    print("means", kernel, flush=True)
    case = Case(ss, [500, 33], fmt=ko.INT8, dim=64, pt=16, kv_heads=1, seed=4)
    case.scale[:, :, 0] = 0
    case.c.scale.copy_(torch.from_numpy(case.scale))
    q = case.queries([60, 33], 2, torch.float16)
    lse = torch.empty(93, 2, device="cuda")
    out = case.c.attend(1, q, i32([0, 1]), i32([0, 60, 93]), lse=lse)
    case.c.check()
    case.check(q, [60, 33], out, lse, 0.125, True, 0)


def test_scores_that_rise_along_the_keys(ss, kernel):
    """The running maximum is raised again and again; late keys dominate."""
    import torch
    print("rising", kernel, flush=True)
    for sign in (1, -1):
        case = Case(ss, [400], fmt=ko.INT8, dim=64, pt=64, kv_heads=1, seed=5)
        data = np.zeros_like(case.data)
        for b in range(7):
            page = case.tables[0, b]
            block = data[page].reshape(2, 2, 1, 64 * 64)
            k = np.zeros((64, 64), np.int8)
            k[:, 0] = np.clip(sign * (np.arange(b * 64, b * 64 + 64) - 200) // 2, -127, 127)
            block[1, 0, 0][ko.block_index(0, 64, 64)] = k.view(np.uint8)
            block[1, 1] = case.data[page].reshape(2, 2, 1, 64 * 64)[1, 1]
        case.data = data
        case.scale[:, :, 0] = 1.0
        case.c.data.copy_(torch.from_numpy(data))
        case.c.scale.copy_(torch.from_numpy(case.scale))
        q = torch.zeros(70, 1, 64, dtype=torch.bfloat16, device="cuda")
        q[:, 0, 0] = 1.0
        lse = torch.empty(70, 1, device="cuda")
        out = case.c.attend(1, q, i32([0]), i32([0, 70]), scale=1.0, lse=lse)
        case.c.check()
        case.check(q, [70], out, lse, 1.0, True, 0)


def test_an_output_may_be_a_slice(ss, kernel):
    """Rows of the output that lie apart, 16-byte aligned and not."""
    import torch
    print("slices", kernel, flush=True)
    case = Case(ss, [90, 33], fmt=ko.FP8, dim=128, pt=32, kv_heads=2, seed=6)
    q = case.queries([40, 33], 4, torch.bfloat16)
    ref = case.c.attend(1, q, i32([0, 1]), i32([0, 40, 73])).clone()
    for pad in (8, 2, 1):
        wide = torch.zeros(73, 4 * 128 + pad, dtype=torch.bfloat16, device="cuda")
        out = wide[:, pad:].view(73, 4, 128)
        case.c.attend(1, q, i32([0, 1]), i32([0, 40, 73]), out=out)
        case.c.check()
        assert torch.equal(out, ref) and (wide[:, :pad] == 0).all()


@pytest.mark.parametrize("dim,pt,kv_heads", [(64, 16, 1), (128, 64, 2), (256, 32, 3),
                                             (128, 256, 1)])
@pytest.mark.parametrize("fmt", [ko.INT8, ko.FP8])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("pad", [8, 1])
def test_append(ss, dim, pt, kv_heads, fmt, dtype, pad):
    """New tokens beside older ones, over page borders, on reused pages."""
    import torch
    print("append", dim, pt, kv_heads, fmt, dtype, pad, flush=True)
    lens = [1, 40, 300, 17, 64, 65, 130, 16]
    new = [1, 1, 300, 16, 1, 64, 33, 0]
    case = Case(ss, lens, fmt=fmt, dim=dim, pt=pt, kv_heads=kv_heads, seed=dim + pt)
    rng, c, t = case.rng, case.c, sum(new)
    x = rng.normal(size=(t, 2 * kv_heads * dim + pad)) * np.exp(rng.normal(size=(t, 1)))
    x[5, :dim] = 0
    x = torch.from_numpy(x).to(dtype_of(dtype)).cuda()
    k = x[:, :kv_heads * dim].view(t, kv_heads, dim)
    v = x[:, kv_heads * dim:2 * kv_heads * dim].view(t, kv_heads, dim)
    c.append(1, k, v, i32(range(len(lens))), i32(np.concatenate([[0], np.cumsum(new)])))
    c.check()
    data, scale = c.data.cpu().numpy(), c.scale.cpu().numpy()
    val, top = ko.code_values(fmt), ko.TOP[fmt]
    steps = np.sort(val[~np.isnan(val)])
    touched = np.zeros(case.data.shape, bool)
    marked = np.zeros(scale.shape, bool)
    L = (2, kv_heads, pt * dim)

    def nearest(codes, quotient):
        """Each code is as near to its quotient as any other one."""
        got = np.abs(val[codes] - quotient)
        j = np.clip(np.searchsorted(steps, quotient), 1, len(steps) - 1)
        best = np.minimum(np.abs(steps[j] - quotient), np.abs(steps[j - 1] - quotient))
        assert (got <= best + top * 2.0 ** -20).all()

    at = 0
    for s, (n, m) in enumerate(zip(lens, new)):
        for b in range((n - m) // pt, -(-n // pt) if m else 0):
            page, lo, hi = case.tables[s, b], max(0, n - m - b * pt), min(pt, n - b * pt)
            r0 = at + b * pt + lo - (n - m)
            for w, src in ((0, k), (1, v)):
                idx = ko.block_index(w, pt, dim)
                for h in range(kv_heads):
                    xs = src[r0:r0 + hi - lo, h].double().cpu().numpy()
                    was = float(case.scale[page, 1, w, h]) if lo else 0.0
                    want = max(was, np.abs(xs).max() / top)
                    now = float(scale[page, 1, w, h])
                    marked[page, 1, w, h] = True
                    assert abs(now - want) <= want * 2.0 ** -22
                    block = data[page].reshape(2, *L)[1, w, h]
                    old = case.data[page].reshape(2, *L)[1, w, h]
                    by = now if now > 0 else 1.0
                    nearest(block[idx[lo:hi]], xs / by)
                    if now > was:
                        nearest(block[idx[:lo]], val[old[idx[:lo]]] * was / by)
                    else:
                        assert (block[idx[:lo]] == old[idx[:lo]]).all()
                    touched[page].reshape(2, *L)[1, w, h][idx[:hi]] = True
        at += m
    assert (data[~touched] == case.data[~touched]).all()
    assert (scale[~marked] == case.scale[~marked]).all()


def test_append_step_by_step_equals_a_prompt_where_scales_do_not_grow(ss):
    """One token at a time with the largest first gives the codes of one call."""
    import torch
    print("append steps", flush=True)
    gen = torch.Generator("cuda").manual_seed(2)
    x = torch.randn(2, 50, 2, 64, generator=gen, device="cuda").clamp(-2, 2).bfloat16()
    x[:, ::16, :, 0] = 3.0
    out = []
    for chunk in (50, 1):
        c = ss.KVCache(8, 1, 8, layers=1, kv_heads=2, head_dim=64, page_tokens=16)
        c.data.zero_()
        for a in range(0, 50, chunk):
            c.reserve(i32([0]), i32([chunk]))
            c.append(0, x[0, a:a + chunk], x[1, a:a + chunk], i32([0]), i32([0, chunk]))
        c.check()
        out.append((c.data.clone(), c.scale.clone(), c.book.clone()))
    for a, b in zip(*out):
        assert torch.equal(a, b)


@pytest.mark.parametrize("fmt", [ko.INT8, ko.FP8])
def test_append_of_values_that_are_not_finite(ss, fmt):
    import torch
    print("append inf", fmt, flush=True)
    c = ss.KVCache(2, 1, 2, layers=1, kv_heads=1, head_dim=64, page_tokens=16, format=fmt)
    c.reserve(i32([0]), i32([3]))
    x = torch.ones(3, 1, 64, dtype=torch.bfloat16, device="cuda")
    x[0, 0, 0], x[0, 0, 1], x[1, 0, 2] = float("inf"), float("-inf"), float("nan")
    c.append(0, x, torch.zeros_like(x), i32([0]), i32([0, 3]))
    with pytest.raises(ss.SemschedRangeError):
        c.check()
    c.check()  # reported once
    val = ko.code_values(fmt)
    got = val[c.data.cpu().numpy()[0][ko.block_index(0, 16, 64)[:3]]]
    top = ko.TOP[fmt]
    assert got[0, 0] == top and got[0, 1] == -top and got[1, 2] == 0 and got[2, 5] == top
    out = c.attend(0, x[2:], i32([0]))
    assert (out == 0).all()  # V of zeros: scale 0
    c.check()


def assert_pages(c, ref, label):
    assert c.refs.tolist() == ref.refs, label
    assert c.lens.tolist() == ref.lens, label
    assert c.tables.tolist() == ref.table_rows(), label
    assert [w & 0xffffffff for w in c.live.tolist()] == ref.live_words(), label
    data = c.data.cpu().numpy()
    scale = c.scale.cpu().numpy().reshape(data.shape[0], -1)
    for p, r in enumerate(ref.refs):
        if r:
            b, s = ref.content[p]
            assert (data[p] == b).all() and (scale[p] == s).all(), (label, p)


@pytest.mark.parametrize("pt,pages,slots,seed", [(16, 40, 9, 0), (64, 33, 12, 1), (16, 300, 40, 2),
                                                 (32, 1000, 70, 3), (16, 5, 3, 4)])
def test_pages_against_the_reference(ss, pt, pages, slots, seed):
    """A random program of all page operations, compared after every step."""
    import torch
    print("pages", pt, pages, slots, seed, flush=True)
    rng = np.random.default_rng(seed)
    mb = max(2, 2 * pages // slots)
    c = ss.KVCache(pages, slots, mb, layers=2, kv_heads=3, head_dim=64, page_tokens=pt,
                   format=ss.KV_FP8)
    data = rng.integers(0, 256, c.data.shape).astype(np.uint8)
    scale = rng.normal(size=tuple(c.scale.shape)).astype(np.float32)
    c.data.copy_(torch.from_numpy(data))
    c.scale.copy_(torch.from_numpy(scale))
    ref = ko.Pages(pages, slots, mb, pt)
    ref.content = [(data[p], scale[p].reshape(-1)) for p in range(pages)]
    refused = 0
    for step in range(60):
        op = rng.choice(["reserve", "reserve", "fork", "free", "compact"])
        some = rng.permutation(slots)[:rng.integers(1, slots + 1)].tolist()
        if op == "reserve":
            grow = [int(min(rng.integers(0, 3 * pt), mb * pt - ref.lens[s])) for s in some]
            ok = ref.reserve(some, grow)
            c.reserve(i32(some), i32(grow))
            if not ok:
                refused += 1
                with pytest.raises(ss.SemschedError) as e:
                    c.check()
                assert e.value.code == ss.SEM_ENOMEM
        elif op == "fork":
            empty = [s for s in some if ref.lens[s] == 0]
            full = [s for s in range(slots) if ref.lens[s] > 0]
            if not full or not empty:
                continue
            src = rng.choice(full, len(empty)).tolist()
            tokens = rng.integers(0, mb * pt, len(empty)).tolist() if rng.random() < 0.5 else None
            ref.fork(src, empty, tokens)
            c.fork(i32(src), i32(empty), None if tokens is None else i32(tokens))
        elif op == "free":
            keep = rng.integers(0, mb * pt, len(some)).tolist() if rng.random() < 0.6 else None
            ref.free(some, keep)
            c.free(i32(some), None if keep is None else i32(keep))
        else:
            ref.compact()
            c.compact()
        c.check()
        assert_pages(c, ref, f"step {step}: {op}")
    assert refused > 0 or pages > 40


def test_many_pages(ss):
    """More live words than the planner has threads, and more sequences."""
    import torch
    print("many pages", flush=True)
    pages, slots, pt = 50_000, 3000, 16
    c = ss.KVCache(pages, slots, 32, layers=1, kv_heads=1, head_dim=64, page_tokens=pt)
    ref = ko.Pages(pages, slots, 32, pt)
    rng = np.random.default_rng(9)
    mark = np.arange(pages, dtype=np.float32)
    c.scale.copy_(torch.from_numpy(mark).view(-1, 1, 1, 1).expand(-1, 1, 2, 1))
    ref.content = [(None, p) for p in range(pages)]
    ids = rng.permutation(slots).tolist()
    grow = rng.integers(1, 32 * pt, slots).tolist()
    assert ref.reserve(ids, grow)
    c.reserve(i32(ids), i32(grow))
    out = rng.permutation(slots)[:2000].tolist()
    keep = rng.integers(0, 100, 2000).tolist()
    ref.free(out, keep)
    c.free(i32(out), i32(keep))
    ref.compact()
    c.compact()
    c.check()
    assert c.refs.tolist() == ref.refs and c.tables.tolist() == ref.table_rows()
    assert [w & 0xffffffff for w in c.live.tolist()] == ref.live_words()
    got = c.scale.cpu().numpy()[:, 0, 0, 0]
    assert all(got[p] == ref.content[p][1] for p in range(pages) if ref.refs[p])


def test_undo_by_the_book(ss):
    import torch
    print("undo", flush=True)
    c = ss.KVCache(16, 4, 4, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    c.reserve(i32([0]), i32([20]))
    saved = c.book.clone()
    c.fork(i32([0, 0]), i32([1, 2]))
    c.reserve(i32([1, 2]), i32([4, 30]))
    c.book.copy_(saved)
    c.reserve(i32([3]), i32([1]))
    c.check()
    assert c.tables[3, 0].item() == 2 and c.lens.tolist() == [20, 0, 0, 1]


def test_device_detected_errors(ss):
    """Each leaves the rest of the cache as it was, and memory alone."""
    import torch
    print("errors", flush=True)

    def fresh():
        c = ss.KVCache(8, 4, 3, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
        c.data.zero_()
        c.reserve(i32([0, 1]), i32([20, 5]))
        c.check()
        return c

    x = torch.ones(1, 1, 64, dtype=torch.bfloat16, device="cuda")
    bad = [
        ("slot beyond", ss.SEM_EINVAL, lambda c: c.reserve(i32([4]), i32([1]))),
        ("negative slot", ss.SEM_EINVAL, lambda c: c.free(i32([-1]))),
        ("negative growth", ss.SEM_ERANGE, lambda c: c.reserve(i32([2]), i32([-1]))),
        ("full table", ss.SEM_EINVAL, lambda c: c.reserve(i32([2, 0]), i32([5, 40]))),
        ("too few pages", ss.SEM_ENOMEM, lambda c: c.reserve(i32([2, 3, 1]), i32([48, 48, 1]))),
        ("fork to a full one", ss.SEM_EINVAL, lambda c: c.fork(i32([0]), i32([1]))),
        ("fork to itself", ss.SEM_EINVAL, lambda c: c.fork(i32([2]), i32([2]))),
        ("fork of a negative count", ss.SEM_ERANGE, lambda c: c.fork(i32([0]), i32([2]), i32([-3]))),
        ("negative keep", ss.SEM_ERANGE, lambda c: c.free(i32([0]), i32([-2]))),
        ("append to a bad slot", ss.SEM_EINVAL, lambda c: c.append(0, x, x, i32([9]))),
        ("append without room", ss.SEM_EINVAL, lambda c: c.append(0, x, x, i32([2]))),
        ("append with bad offsets", ss.SEM_EINVAL, lambda c: c.append(0, x, x, i32([0]), i32([0, 2]))),
        ("attend of a bad slot", ss.SEM_EINVAL, lambda c: c.attend(0, x, i32([7]))),
        ("attend with bad offsets", ss.SEM_EINVAL, lambda c: c.attend(0, x, i32([0]), i32([0, 5]))),
    ]
    for name, code, call in bad:
        print(" ", name, flush=True)
        c = fresh()
        book, scale = c.book.clone(), c.scale.clone()
        call(c)
        with pytest.raises(ss.SemschedError) as e:
            c.check()
        assert e.value.code == code, name
        if name != "fork of a negative count":
            assert torch.equal(c.book, book) and torch.equal(c.scale, scale), name
        c.check()
    # page numbers and lengths that the cache cannot hold
    for what in ("page", "length"):
        print(" ", what, flush=True)
        c = fresh()
        if what == "page":
            c.tables[0, 1] = 1 << 30
        else:
            c.lens[0] = 100
        for call in (lambda: c.attend(0, x, i32([0])), lambda: c.append(0, x, x, i32([0])),
                     lambda: c.reserve(i32([0]), i32([1])), lambda: c.fork(i32([0]), i32([2])),
                     lambda: c.free(i32([0]))):
            call()
            with pytest.raises(ss.SemschedError):
                c.check()


def test_empty_calls(ss):
    import torch
    print("empty", flush=True)
    c = ss.KVCache(4, 2, 2, layers=1, kv_heads=2, head_dim=64, page_tokens=16)
    none = i32([])
    c.reserve(none, none)
    c.fork(none, none)
    c.free(none)
    c.compact()
    q = torch.empty(0, 4, 64, dtype=torch.float16, device="cuda")
    c.append(0, q[:, :2], q[:, :2], none)
    assert c.attend(0, q, none).shape == (0, 4, 64)
    c.check()
    empty = ss.KVCache(0, 0, 0, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    empty.compact()
    empty.check()


def test_on_another_stream_and_in_a_graph(ss):
    """A decode step enqueued on a side stream, then captured and replayed."""
    import torch
    print("graph", flush=True)
    c = ss.KVCache(64, 3, 16, layers=2, kv_heads=2, head_dim=64, page_tokens=16)
    gen = torch.Generator("cuda").manual_seed(4)
    seqs, one = i32([0, 1, 2]), i32([1, 1, 1])
    x = torch.randn(3, 8, 64, generator=gen, device="cuda").bfloat16()
    out = torch.empty(2, 3, 4, 64, dtype=torch.bfloat16, device="cuda")
    c.reserve(seqs, i32([30, 1, 100]))
    for layer in (0, 1):
        kv = torch.randn(2, 131, 2, 64, generator=gen, device="cuda").bfloat16()
        c.append(layer, kv[0], kv[1], seqs, i32([0, 30, 31, 131]))

    def step():
        c.reserve(seqs, one)
        for layer in (0, 1):
            c.append(layer, x[:, 4:6], x[:, 6:], seqs)
            c.attend(layer, x[:, :4], seqs, out=out[layer], max_len=256)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    saved = [t.clone() for t in (c.book, c.data, c.scale)]
    eager = []
    with torch.cuda.stream(side):
        for _ in range(3):
            step()
            eager.append((out.clone(), c.book.clone(), c.data.clone(), c.scale.clone()))
        c.check()
        for t, s in zip((c.book, c.data, c.scale), saved):
            t.copy_(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    torch.cuda.synchronize()
    for want in eager:
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((out, c.book, c.data, c.scale), want):
            assert torch.equal(a, b)
        torch.ones(1000, device="cuda").sum()  # the program's own work between replays
    c.check()


def test_blocking_forms(ss):
    """The blocking C calls give the asynchronous ones' results and statuses."""
    import ctypes

    import torch
    print("blocking", flush=True)
    L = ss.lib
    torch.cuda.synchronize()
    L.sem_set_stream(ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    gen = torch.Generator("cuda").manual_seed(6)
    x = torch.randn(20, 8, 64, generator=gen, device="cuda").half()
    a, b = (ss.KVCache(16, 3, 4, layers=1, kv_heads=2, head_dim=64, page_tokens=16) for _ in "ab")
    a.data.zero_(), b.data.zero_()
    s0, s01, cu = i32([0]), i32([0, 1]), i32([0, 20])
    a.reserve(s0, i32([20]))
    a.append(0, x[:, 4:6], x[:, 6:], s0, cu)
    a.fork(s0, i32([1]), i32([18]))
    a.reserve(s01, i32([3, 3]))
    a.free(s0, i32([17]))
    a.compact()
    want = a.attend(0, x[:, :4], s0, cu)
    a.check()
    p, ref = (lambda t: ctypes.c_void_p(t.data_ptr())), b._ref
    grow, three, keep, eighteen, dst = i32([20]), i32([3, 3]), i32([17]), i32([18]), i32([1])
    out = torch.empty_like(want)
    assert L.sem_kv_reserve(ref, p(s0), p(grow), 1) == 0
    assert L.sem_kv_append(ref, 0, p(x[:, 4:6]), p(x[:, 6:]), 1, 512, 64, 512, 64, p(s0), p(cu), 1,
                           20) == 0
    assert L.sem_kv_fork(ref, p(s0), p(dst), p(eighteen), 1) == 0
    assert L.sem_kv_reserve(ref, p(s01), p(three), 2) == 0
    assert L.sem_kv_free(ref, p(s0), p(keep), 1) == 0
    assert L.sem_kv_compact(ref) == 0
    q = ss.KVQueryC(x.data_ptr(), out.data_ptr(), None, 512, 64, 256, 64, 20, 0, 0, 4, 1, 1, 0,
                    0.125)
    assert L.sem_kv_attend(ref, 0, ctypes.byref(q), p(s0), p(cu), 1) == 0
    assert torch.equal(out, want) and torch.equal(a.book, b.book) and torch.equal(a.scale, b.scale)
    assert L.sem_kv_reserve(ref, p(i32([2])), p(i32([1 << 20])), 1) == ss.SEM_EINVAL
    assert L.sem_kv_free(ref, p(s0), p(i32([-1])), 1) == ss.SEM_ERANGE
    assert L.sem_kv_compact(ref) == 0  # the status does not outlive its call


def test_results_do_not_depend_on_the_run(ss, kernel):
    import torch
    print("repeat", flush=True)
    case = Case(ss, [700, 300, 5], fmt=ko.FP8, dim=128, pt=64, kv_heads=2)
    q = case.queries([1, 1, 1], 8, torch.bfloat16)
    first = case.c.attend(1, q, i32([0, 1, 2])).clone()
    for _ in range(5):
        assert torch.equal(case.c.attend(1, q, i32([0, 1, 2])), first)


def test_eviction_carried_out(ss):
    """sem_evict's victims leave with the prefixes sem_evict_plan saves, and the
    next requests get their pages."""
    import torch
    print("eviction", flush=True)

    class Model:  # reloading pays from 5 tokens of prompt on
        alpha1, alpha2, beta, gamma1, gamma2 = 1 << 32, 0, 5 << 32, 1 << 31, 1 << 31

    c = ss.KVCache(24, 6, 12, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    prompt, decoded = np.array([40, 3, 70, 20, 0, 0]), np.array([8, 30, 0, 25, 0, 0])
    lens = prompt + decoded
    c.reserve(i32(range(6)), i32(lens))
    p = torch.tensor([0, 2, 1, 2, 0, 0], dtype=torch.uint8, device="cuda")
    left = i32([5, 9, 3, 50, 1, 1])
    blocks = torch.from_numpy(-(-lens // 16)).cuda()
    victims, upto = ss.evict(p, left, i32([0, 1, 2, 3]), blocks[:4].contiguous(),
                             int(blocks.sum()), 12, torch.tensor([4], device="cuda"))
    assert victims.tolist() == [3, 1]  # 14 + 4 - 12 = 6 pages over: the two hold 3 each
    keep_prompt, save = ss.evict_plan(i32(prompt), i32(decoded), Model())
    kept = torch.where(keep_prompt.bool(), i32(prompt) + save, torch.zeros_like(save))
    c.free(victims, kept[victims.long()].contiguous())
    c.compact()
    c.check()
    kept = kept.tolist()
    want = [int(lens[0]), kept[1], int(lens[2]), kept[3], 0, 0]
    assert c.lens.tolist() == want
    used = sum(-(-n // 16) for n in want)
    assert c.refs.tolist() == [1] * used + [0] * (24 - used)


def test_errors_of_either_attention_kernel(ss, kernel):
    """Sequences, offsets, page numbers and lengths outside the cache."""
    import torch
    print("attention errors", kernel, flush=True)
    q = torch.ones(40, 2, 64, dtype=torch.float16, device="cuda")

    def fresh():
        c = ss.KVCache(8, 4, 4, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
        c.data.zero_()
        c.reserve(i32([0, 1]), i32([50, 40]))
        c.check()
        return c

    for name, seqs, cu in (("a slot beyond", [0, 9], [0, 10, 40]),
                           ("a negative slot", [-1, 1], [0, 10, 40]),
                           ("offsets past the rows", [0, 1], [0, 10, 90]),
                           ("offsets that fall", [0, 1], [0, 50, 40]),
                           ("offsets from 5", [0, 1], [5, 10, 40]),
                           ("negative offsets", [0, 1], [-5, 10, 40]),
                           ("offsets that end early", [0, 1], [0, 10, 30])):
        print(" ", name, flush=True)
        c = fresh()
        c.attend(0, q, i32(seqs), i32(cu))
        with pytest.raises(ss.SemschedError):
            c.check()
    for name, change in (("page", lambda c: c.tables[0, 1].fill_(1 << 30)),
                         ("negative page", lambda c: c.tables[0, 1].fill_(-7)),
                         ("length", lambda c: c.lens[0].fill_(65)),
                         ("negative length", lambda c: c.lens[0].fill_(-1))):
        print(" ", name, flush=True)
        c = fresh()
        change(c)
        c.attend(0, q, i32([0, 1]), i32([0, 20, 40]))
        with pytest.raises(ss.SemschedError):
            c.check()
    # a cache without pages
    c = ss.KVCache(0, 2, 2, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    out = c.attend(0, q, i32([0, 1]), i32([0, 20, 40]))
    c.check()
    assert (out == 0).all()
    c.lens.fill_(3)
    c.attend(0, q, i32([0, 1]), i32([0, 20, 40]))
    with pytest.raises(ss.SemschedError):
        c.check()


@pytest.mark.parametrize("cu", [[33, 38], [3, 5], [0, 1], [0, 45], [-2, 5], [5, 0]])
def test_append_of_bad_offsets(ss, cu):
    """Reported, with nothing written outside the sequences' own pages."""
    import torch
    print("append offsets", cu, flush=True)
    c = ss.KVCache(8, 3, 4, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    c.data.zero_()
    c.reserve(i32([0, 1, 2]), i32([20, 20, 20]))
    c.check()
    x = torch.ones(40, 1, 64, dtype=torch.bfloat16, device="cuda")
    c.append(0, x, x, i32([1]), i32(cu))
    with pytest.raises(ss.SemschedError):
        c.check()
    own = set(c.tables[1].tolist())
    for page in range(8):
        if page not in own:
            assert (c.data[page] == 0).all() and (c.scale[page] == 0).all(), page


def test_compact_reads_no_bits_past_the_pages(ss):
    import torch
    print("live bits", flush=True)
    c = ss.KVCache(5, 3, 4, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    c.data.copy_(torch.arange(5, dtype=torch.uint8, device="cuda")[:, None].expand_as(c.data))
    c.reserve(i32([0, 1, 2]), i32([16, 32, 16]))
    c.free(i32([1]))
    c.live[0] |= 0x00f00000
    c.compact()
    c.check()
    assert c.tables[0, 0].item() == 0 and c.tables[2, 0].item() == 1
    assert c.refs.tolist() == [1, 1, 0, 0, 0] and c.live[0].item() & 31 == 3
    assert (c.data[1] == 3).all()


@pytest.mark.parametrize("fmt", [ko.INT8, ko.FP8])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("tiny", [2.0 ** -128, 1e-40, 2.0 ** -149])
def test_scales_without_a_finite_reciprocal(ss, kernel, fmt, dim, tiny):
    """V scales that are not normal numbers, on the first pages of a sequence, on
    all of them, on its only key. An output is then off by what it is of normal
    scales, and by the least normal number, which is what outputs may be cut to."""
    import torch
    print("tiny scales", kernel, fmt, dim, tiny, flush=True)
    for new in (1, 40):
        lens = [300, 260, max(new, 1), 90]
        case = Case(ss, lens, fmt=fmt, dim=dim, pt=32, kv_heads=1, seed=21)
        case.scale[case.tables[0, :3], :, 1] = tiny
        case.scale[case.tables[1, :9], :, 1] = tiny
        case.scale[case.tables[2, :2], :, 1] = tiny
        case.scale[case.tables[3, 2], :, 1] = tiny
        case.c.scale.copy_(torch.from_numpy(case.scale))
        q = case.queries([new] * 4, 4, torch.bfloat16)
        lse = torch.empty(4 * new, 4, device="cuda")
        out = case.c.attend(1, q, i32(range(4)), i32(np.arange(5) * new), lse=lse)
        case.c.check()
        case.check(q, [new] * 4, out, lse, dim ** -0.5, True, 0)
        for s in (1, 2):  # what check's absolute term hides: the tiny values themselves
            k, v = (ko.read(case.data, case.scale, case.geom, case.tables[s], lens[s], 1, w, 0)
                    for w in (0, 1))
            for h in range(4):
                rows = slice(s * new, (s + 1) * new)
                want, _, mag = ko.attend(q[rows, h].double().cpu().numpy(), k, v, dim ** -0.5,
                                         True, 0)
                tol = 2 * (2.0 ** -9 * np.abs(want) + (2.0 ** -12 + 2.0 ** -14) * mag) + 2.0 ** -126
                assert (np.abs(out[rows, h].double().cpu().numpy() - want) <= tol).all(), (s, h)


def test_appended_values_below_the_normal_scales(ss, kernel):
    """What append writes for values of 2^-121 at most, read back."""
    import torch
    print("tiny values", kernel, flush=True)
    for fmt in (ss.KV_INT8, ss.KV_FP8):
        c = ss.KVCache(8, 1, 8, layers=1, kv_heads=1, head_dim=64, page_tokens=16, format=fmt)
        gen = torch.Generator("cuda").manual_seed(7)
        k = torch.randn(50, 1, 64, generator=gen, device="cuda").bfloat16()
        v = (torch.rand(50, 1, 64, generator=gen, device="cuda") * 2.0 ** -121).bfloat16()
        c.reserve(i32([0]), i32([50]))
        c.append(0, k, v, i32([0]), i32([0, 50]))
        assert (c.scale[c.tables[0, :4].long(), 0, 1] < 2.0 ** -126).all()
        out = c.attend(0, torch.zeros_like(k), i32([0]), i32([0, 50]))  # means of the values
        c.check()
        want = v.double().cumsum(0) / torch.arange(1, 51, device="cuda")[:, None, None]
        # half a code's step (of 127, or of 8 to the power of two), the output's rounding, the least normal
        step = 2.0 ** -121 * (2.0 ** -8 if fmt == ss.KV_INT8 else 2.0 ** -4)
        assert ((out.double() - want).abs() <= step + 2.0 ** -8 * want + 2.0 ** -126).all()


def test_a_graph_outlives_a_larger_workspace(ss, monkeypatch):
    """Steps of a captured graph before and after an eager call that needs a larger
    workspace: the graph's results stay right, nobody else's memory changes, and
    its errors are still reported."""
    import torch
    print("graph and growth", flush=True)

    def fresh():
        c = ss.KVCache(512, 3, 128, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
        gen = torch.Generator("cuda").manual_seed(8)
        kv = torch.randn(2, 3000, 1, 64, generator=gen, device="cuda").bfloat16()
        c.reserve(seqs, i32([1900, 1000, 100]))
        c.append(0, kv[0], kv[1], seqs, i32([0, 1900, 2900, 3000]))
        return c

    seqs, one = i32([0, 1, 2]), i32([1, 1, 1])
    x = torch.randn(3, 4, 64, device="cuda").bfloat16()
    prompt = torch.randn(600, 2, 64, device="cuda").bfloat16()
    out = torch.empty(3, 2, 64, dtype=torch.bfloat16, device="cuda")

    def step(c):  # (the key axis is split: counters and parts lie in the workspace)
        c.reserve(seqs, one)
        c.append(0, x[:, 2:3], x[:, 3:], seqs)
        c.attend(0, x[:, :2], seqs, out=out)

    want, c = [], fresh()
    for _ in range(6):
        step(c)
        want.append((out.clone(), c.book.clone()))

    def by_tiles(c):  # its partial outputs need more
        with monkeypatch.context() as m:
            m.setenv("SEMSCHED_KV_TILES", "1")
            return c.attend(0, prompt, i32([0]), i32([0, 600])).clone()

    large = by_tiles(c)
    c.check()

    c = fresh()
    step(c)  # takes the workspace that the graph is captured with
    torch.cuda.synchronize()
    assert torch.equal(out, want[0][0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(c)
    others, small = [], c.ws_bytes
    for k in range(1, 6):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[k][0]) and torch.equal(c.book, want[k][1]), k
        if k == 2:
            by_tiles(c)
            assert c.ws_bytes > small
        # the program's own tensors, of the sizes of either workspace
        others += [torch.full((n,), 3, dtype=torch.uint8, device="cuda")
                   for n in (small, small // 2, c.ws_bytes)]
    assert torch.equal(by_tiles(c), large)
    c.check()
    assert all((t == 3).all() for t in others)
    c.lens[2] = 128 * 16  # its table is full: the graph's reserve has no room
    graph.replay()
    with pytest.raises(ss.SemschedError) as e:
        c.check()
    assert e.value.code == ss.SEM_EINVAL
    c.check()  # reported once


def test_no_larger_workspace_while_capturing(ss, monkeypatch):
    """Refused with the capture unharmed; the call goes into a graph once its
    workspace is there."""
    import torch
    print("growth in capture", flush=True)
    monkeypatch.setenv("SEMSCHED_KV_TILES", "1")  # (partial outputs for every compute unit)
    c = ss.KVCache(64, 1, 64, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    q = torch.randn(900, 2, 64, device="cuda").bfloat16()
    c.reserve(i32([0]), i32([900]))
    c.append(0, q[:, :1], q[:, 1:], i32([0]), i32([0, 900]))
    seqs, cu, out, x = i32([0]), i32([0, 900]), torch.empty_like(q), torch.zeros(4, device="cuda")
    torch.cuda.synchronize()
    before, graph = c.workspace, torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x += 1
        with pytest.raises(RuntimeError, match="captured"):
            c.attend(0, q, seqs, cu, out=out)
    assert c.workspace is before
    graph.replay()
    assert (x == 1).all()
    want = c.attend(0, q, seqs, cu).clone()
    c.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.attend(0, q, seqs, cu, out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    c.check()


@pytest.mark.parametrize("cu", [[0, 100, 50, 120], [0, 100, 100, 20, 120], [0, 40, 10, 30, 120],
                                [0, 60, 120, 119, 120], list(range(0, 71)) + [10, 40, 120]])
def test_append_of_offsets_that_fall(ss, cu):
    """Wherever they do, with the ends and every other sequence's rows in order."""
    print("append, falling offsets", len(cu), flush=True)
    import torch
    n = len(cu) - 1
    c = ss.KVCache(16 * n, n, 16, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    c.reserve(i32(range(n)), i32([120] * n))
    c.check()
    x = torch.ones(120, 1, 64, dtype=torch.bfloat16, device="cuda")
    c.append(0, x, x, i32(range(n)), i32(cu))
    with pytest.raises(ss.SemschedError) as e:
        c.check()
    assert e.value.code == ss.SEM_EINVAL
    # the same cache takes offsets that do not
    c.append(0, x, x, i32(range(n)), i32(sorted(cu)))
    c.check()


@pytest.mark.parametrize("at", [1, 40, 63, 64, 65, 70, 149, 299])
@pytest.mark.parametrize("by", [1, 30])
def test_attention_of_offsets_that_fall(ss, kernel, at, by):
    """At any sequence of many, with the ends in order."""
    import torch
    print("attention, falling offsets", kernel, at, by, flush=True)
    n = 300
    c = ss.KVCache(n, n, 1, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    c.data.zero_()
    c.reserve(i32(range(n)), i32([16] * n))
    cu = np.arange(n + 1)
    cu[at] = max(cu[at + 1] + by if at < n - 1 else cu[at - 1] - by, 0)
    assert (np.diff(cu) < 0).any()
    q = torch.ones(n, 2, 64, dtype=torch.float16, device="cuda")
    c.attend(0, q, i32(range(n)), i32(np.arange(n + 1)))
    c.check()
    c.attend(0, q, i32(range(n)), i32(cu))
    with pytest.raises(ss.SemschedError) as e:
        c.check()
    assert e.value.code == ss.SEM_EINVAL


def test_rows_and_sequences_that_do_not_match(ss, kernel):
    """Rows of no sequence; sequences without rows whose offsets say otherwise."""
    import torch
    print("rows and sequences", kernel, flush=True)
    c = ss.KVCache(8, 4, 4, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    c.data.zero_()
    c.reserve(i32([0, 1]), i32([20, 5]))
    x = torch.ones(3, 2, 64, dtype=torch.float16, device="cuda")
    calls = (lambda m, seqs, cu: c.attend(0, x[:m], i32(seqs), i32(cu)),
             lambda m, seqs, cu: c.append(0, x[:m, :1], x[:m, 1:], i32(seqs), i32(cu)))
    for call in calls:
        with pytest.raises(ss.SemschedError) as e:
            call(3, [], [0])
        assert e.value.code == ss.SEM_EINVAL
        for cu in ([0, 0, 3], [0, 5, 0], [-2, 0, 0], [3, 3, 3]):
            call(0, [0, 1], cu)
            with pytest.raises(ss.SemschedError) as e:
                c.check()
            assert e.value.code == ss.SEM_EINVAL, cu
        call(0, [0, 1], [0, 0, 0])
        call(0, [], [0])
        c.check()
    assert (c.data == 0).all() and (c.scale == 0).all()


def test_needs_that_pass_32_bits(ss):
    """33 sequences that ask for 2^32 pages in all: too few are free, and nothing
    changes (a sum of 32 bits would be 0)."""
    import torch
    print("needs beyond 32 bits", flush=True)
    mb, n = (1 << 27) - 1, 33
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("the tables of this size take 18 GB")
    c = ss.KVCache(4, n, mb, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    grow = [mb * 16] * 32 + [32 * 16]
    assert sum(g // 16 for g in grow) == 1 << 32
    c.reserve(i32(range(n)), i32(grow))
    with pytest.raises(ss.SemschedError) as e:
        c.check()
    assert e.value.code == ss.SEM_ENOMEM
    assert (c.lens == 0).all() and (c.refs == 0).all() and (c.live == 0).all()
    assert (c.tables[:, :64] == -1).all()
    c.reserve(i32([3, 1]), i32([33, 16]))
    c.check()
    assert c.tables[3, :4].tolist() == [0, 1, 2, -1] and c.tables[1, :2].tolist() == [3, -1]
    del c
    torch.cuda.empty_cache()


@pytest.mark.parametrize("fmt,dim", [(ko.INT8, 64), (ko.FP8, 128), (ko.INT8, 256)])
@pytest.mark.parametrize("grow", [1e3, 1e-3])
@pytest.mark.parametrize("window", [0, 20])
def test_hidden_pages_take_no_bits(ss, kernel, fmt, dim, grow, window):
    """V scales that rise or fall a thousand times from page to page: what a row
    does not see, by the window or because it is later, does not count."""
    import torch
    if not window and grow < 1:
        return  # (a row sees the first and largest scale then)
    print("hidden pages", kernel, fmt, dim, grow, window, flush=True)
    for new in (1, 60):
        lens = [160, 150, 60]
        case = Case(ss, lens, fmt=fmt, dim=dim, pt=16, kv_heads=1, seed=31)
        for s in range(3):
            for b in range(-(-lens[s] // 16)):
                case.scale[case.tables[s, b], :, 1] *= np.float32(grow ** (b - 5))
        case.c.scale.copy_(torch.from_numpy(case.scale))
        q = case.queries([new] * 3, 2, torch.bfloat16)
        out = case.c.attend(1, q, i32(range(3)), i32(np.arange(4) * new), window=window)
        case.c.check()
        # (check's absolute term would hide the small ones)
        o = out.double().cpu().numpy()
        for s in range(3):
            k, v = (ko.read(case.data, case.scale, case.geom, case.tables[s], lens[s], 1, w, 0)
                    for w in (0, 1))
            for h in range(2):
                rows = slice(s * new, (s + 1) * new)
                want, _, mag = ko.attend(q[rows, h].double().cpu().numpy(), k, v, dim ** -0.5,
                                         True, window)
                tol = 2 * (2.0 ** -9 * np.abs(want) + (2.0 ** -12 + 2.0 ** -14) * mag)
                # a weight is no finer than 2^-31 of the row's largest weight and scale
                for i in range(new):
                    n = lens[s] - new + i + 1
                    low = max(n - window, 0) if window else 0
                    page = case.tables[s, np.arange(low, n) // 16]
                    vs = case.scale[page, 1, 1, 0].astype(np.float64)
                    codes = np.abs(v[low:n]) / vs[:, None]
                    tol[i] += 2.0 ** -31 * vs.max() * codes.sum(0)
                assert (np.abs(o[rows, h] - want) <= tol).all(), (new, s, h)


@pytest.mark.parametrize("new", [1, 40])
def test_blocks_of_scale_zero_count_nothing(ss, kernel, new):
    """V codes under a scale of zero, on the keys of almost all the weight."""
    import torch
    print("scale zero", kernel, new, flush=True)
    case = Case(ss, [128], fmt=ko.INT8, dim=64, pt=16, kv_heads=1, seed=33)
    null = case.tables[0, 3:6]
    data = case.data.reshape(-1, 2, 2, 1, 16 * 64)
    data[:, 1, 0] = 0
    data[null, 1, 0] = 1  # these keys' scores are 14 above the others' 0
    case.scale[:, 1, 0] = 14 / 64
    case.scale[null, 1, 1] = 0
    case.scale[case.tables[0, [0, 1, 2, 6, 7]], 1, 1] = 2.0 ** 16
    case.c.scale.copy_(torch.from_numpy(case.scale))
    q = torch.ones(new, 1, 64, dtype=torch.float16, device="cuda")
    got = []
    for value in (0, 100, 156):  # 156: -100
        data[null, 1, 1] = value
        case.c.data.copy_(torch.from_numpy(case.data))
        got.append(case.c.attend(1, q, i32([0]), i32([0, new]), scale=1.0).clone())
        case.c.check()
    assert (got[0] != 0).any()
    for x in got[1:]:
        assert torch.equal(x, got[0])


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [(1 << 31) - 1, (1 << 31) - 17, 1 << 30])
def test_windows_larger_than_any_length(ss, kernel, causal, window):
    """As none, for rows before the first key, too."""
    print("wide windows", kernel, causal, window, flush=True)
    _, q, out = run_attend(ss, [3, 0, 70, 90], [20, 4, 200, 9], heads=3, kv_heads=1, causal=causal,
                           fmt=ko.FP8, window=window)
    _, _, ref = run_attend(ss, [3, 0, 70, 90], [20, 4, 200, 9], heads=3, kv_heads=1, causal=causal,
                           fmt=ko.FP8)
    import torch
    assert torch.equal(out, ref)


def test_the_bench_reports_the_kernel_that_it_names(ss, capsys):
    """The roofline of a serving iteration is one attention's, not the iteration's."""
    import argparse
    import json

    import bench
    print("bench kv", flush=True)
    assert bench.bench_kv(argparse.Namespace(steps=2, warmup=1, no_cpu_baseline=True)) == 0
    res = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    roof = res["roofline"]
    assert 0 < roof["avg_launch_ms"] * 8 < res["ms_per_step"]  # 8 layers
    assert abs(roof["bytes_per_launch"] / roof["avg_launch_ms"] / 1e6 - roof["achieved"]) < 1


def test_cut_tiles_do_not_depend_on_the_run(ss, monkeypatch):
    """Tiles whose keys go to several workgroups give the same bits in every run."""
    import torch
    print("repeat, tiles", flush=True)
    monkeypatch.setenv("SEMSCHED_KV_TILES", "1")
    for dim, fmt in ((128, ko.FP8), (64, ko.INT8), (256, ko.INT8)):
        case = Case(ss, [3000, 700, 1900], fmt=fmt, dim=dim, pt=64, kv_heads=2)
        q = case.queries([200, 1, 333], 8, torch.float16)
        seqs, cu = i32([0, 1, 2]), i32([0, 200, 201, 534])
        first = case.c.attend(1, q, seqs, cu).clone()
        for _ in range(5):
            assert torch.equal(case.c.attend(1, q, seqs, cu), first)
        case.c.check()
