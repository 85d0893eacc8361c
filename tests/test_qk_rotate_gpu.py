"""The norms and rotation of queries and keys against their 64-bit reference.

Tolerance. Everything is in 32 bits: a row's mean square (16 squares added in a
lane, then the lanes: 20 roundings, halved by the root), the root, the quotient and
two products, 16 * 2^-24 in all; an angle is off by the rounding of a fraction of a
turn, 2 pi * 2^-26, its sine and cosine by 3e-8 more and four roundings, 2^-21 in
all. An element is a sum of two products of these, hence
|error| <= eps / 2 |y| + (|a| + |b|) 2^-19, eps / 2 the rounding to its type (2^-25,
half the least step, where half precision has no more digits).
"""

import ctypes

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


def dtype_of(name):
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16}[name]


class Rows:
    """Queries and keys as slices of wider rows."""

    def __init__(self, tokens, heads, kv_heads, dim, rot, dtype, pad=8, far=None, seed=0):
        import torch
        rng = np.random.default_rng(seed)
        x = rng.normal(size=(tokens, (heads + kv_heads) * dim + pad)) * np.exp(
            rng.normal(size=(tokens, 1)))
        x = torch.from_numpy(x).to(dtype).cuda()
        self.q = x[:, :heads * dim].view(tokens, heads, dim)
        self.k = x[:, heads * dim:(heads + kv_heads) * dim].view(tokens, kv_heads, dim)
        far = far or [0, 1, 100, 131071, -5, 2 ** 31 - 1, -2 ** 31, 123456789]
        pos = np.resize(np.array(far, np.int64), tokens).astype(np.int32)
        freq = (10000.0 ** (-np.arange(rot // 2) / max(rot // 2, 1))).astype(np.float32)
        w = rng.normal(1, 0.3, (2, dim)).astype(np.float32)
        self.pos, self.freq = torch.from_numpy(pos).cuda(), torch.from_numpy(freq).cuda()
        self.wq, self.wk = torch.from_numpy(w).cuda()

    def check(self, ss, q_out, k_out, wq, wk, eps=1e-6, interleaved=False, source=None):
        import torch
        for x, out, w in zip(source or (self.q, self.k), (q_out, k_out), (wq, wk)):
            want, mag = ko.rotate(x.double().cpu().numpy(),
                                  None if w is None else w.double().cpu().numpy(), eps,
                                  self.pos.tolist(), self.freq.double().tolist(), interleaved)
            half = torch.finfo(out.dtype).eps / 2
            tol = half * np.abs(want) + mag * 2.0 ** -19 + (2.0 ** -25 if half < 2 ** -10 else 0)
            err = np.abs(out.double().cpu().numpy() - want)
            assert (err <= tol).all(), (err / np.maximum(tol, 1e-300)).max()


@pytest.mark.parametrize("dim,rot", [(64, 64), (64, 32), (64, 16), (64, 0), (128, 128), (128, 64),
                                     (128, 48), (256, 256), (256, 80)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("norm", ["both", "none", "q", "k"])
def test_rotate(ss, dim, rot, interleaved, dtype, norm):
    print("rotate", dim, rot, interleaved, dtype, norm, flush=True)
    for tokens, heads, kv_heads, pad in ((1, 1, 1, 8), (9, 5, 3, 1), (3, 32, 8, 8), (17, 2, 40, 2)):
        r = Rows(tokens, heads, kv_heads, dim, rot, dtype_of(dtype), pad)
        wq, wk = (r.wq if norm in "both q" else None), (r.wk if norm in "both k" else None)
        q, k = ss.qk_rotate(r.q, r.k, r.pos, r.freq, q_weight=wq, k_weight=wk,
                            interleaved=interleaved)
        r.check(ss, q, k, wq, wk, interleaved=interleaved)


@pytest.mark.parametrize("heads,kv_heads", [(0, 3), (3, 0), (0, 0), (65, 1)])
def test_one_side_alone(ss, heads, kv_heads):
    print("one side", heads, kv_heads, flush=True)
    import torch
    r = Rows(5, heads, kv_heads, 128, 128, torch.float16)
    q, k = ss.qk_rotate(r.q, r.k, r.pos, r.freq, q_weight=r.wq, k_weight=r.wk, eps=0.1)
    assert q.shape == (5, heads, 128) and k.shape == (5, kv_heads, 128)
    r.check(ss, q, k, r.wq, r.wk, eps=0.1)


def test_many_tokens(ss):
    """Steps of a wave that hold rows of both kinds, one step, all of a token's."""
    import torch
    print("many tokens", flush=True)
    for tokens, heads, kv_heads in ((0, 4, 2), (300, 7, 3), (1500, 30, 5)):
        r = Rows(tokens, heads, kv_heads, 64, 64, torch.bfloat16)
        q, k = ss.qk_rotate(r.q, r.k, r.pos, r.freq, q_weight=r.wq, k_weight=r.wk)
        some = slice(max(0, tokens - 40), tokens)
        r.pos = r.pos[some]
        r.check(ss, q[some], k[some], r.wq, r.wk, source=(r.q[some], r.k[some]))
    r = Rows(9000, 30, 5, 64, 64, torch.bfloat16)
    all_q, all_k = ss.qk_rotate(r.q, r.k, r.pos, r.freq, q_weight=r.wq, k_weight=r.wk)
    for at in (0, 4444, 8999):  # a token does not depend on the others
        q, k = ss.qk_rotate(r.q[at:at + 1], r.k[at:at + 1], r.pos[at:at + 1], r.freq,
                            q_weight=r.wq, k_weight=r.wk)
        assert torch.equal(q[0], all_q[at]) and torch.equal(k[0], all_k[at])


@pytest.mark.parametrize("pad", [8, 1])
@pytest.mark.parametrize("rot,interleaved", [(128, False), (32, True), (48, False)])
def test_in_place(ss, pad, rot, interleaved):
    import torch
    print("in place", pad, rot, flush=True)
    r = Rows(50, 6, 2, 128, rot, torch.bfloat16, pad)
    kw = dict(q_weight=r.wq, k_weight=r.wk, interleaved=interleaved)
    want = ss.qk_rotate(r.q, r.k, r.pos, r.freq, **kw)
    wide = r.q.as_strided((50, 8 * 128 + pad), (r.q.stride(0), 1))
    behind = wide[:, 8 * 128:].clone()
    got = ss.qk_rotate(r.q, r.k, r.pos, r.freq, q_out=r.q, k_out=r.k, **kw)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(wide[:, 8 * 128:], behind)


def test_values_that_are_not_finite_stay_in_their_rows(ss):
    import torch
    print("nan", flush=True)
    for dtype in (torch.bfloat16, torch.float16):
        r = Rows(4, 3, 2, 64, 32, dtype)
        want = ss.qk_rotate(r.q, r.k, r.pos, r.freq)[0]
        r.q[1, 1, 40], r.q[2, 0, 50], r.q[3, 2, 3] = float("nan"), float("-inf"), float("inf")
        out = ss.qk_rotate(r.q, r.k, r.pos, r.freq)[0]
        assert out[1, 1, 40].isnan() and out[2, 0, 50] == float("-inf")
        assert not out[3, 2, 3].isfinite() and not out[3, 2, 19].isfinite()
        same = torch.ones_like(out, dtype=torch.bool)
        same[1, 1, 40] = same[2, 0, 50] = same[3, 2, 3] = same[3, 2, 19] = False
        assert torch.equal(out[same], want[same])
        normed = ss.qk_rotate(r.q, r.k, r.pos, r.freq, q_weight=r.wq)[0]
        bad = ~normed.isfinite().all(-1)
        assert bad.tolist() == [[False] * 3, [False, True, False], [True, False, False],
                                [False, False, True]]
    # rows of zeros, rows whose squares pass half precision
    z = torch.zeros(2, 1, 64, dtype=torch.float16, device="cuda")
    z[1] = 60000.0
    pos, freq, w = torch.zeros(2, dtype=torch.int32, device="cuda"), r.freq, r.wq
    out = ss.qk_rotate(z, z, pos, freq, q_weight=w)[0]
    assert (out[0] == 0).all() and torch.equal(out[1, 0], w.half())


def test_streams_graphs_and_the_blocking_form(ss):
    import torch
    print("graph", flush=True)
    r = Rows(70, 8, 2, 128, 128, torch.bfloat16)
    qo, ko_ = torch.empty(70, 8, 128, dtype=r.q.dtype, device="cuda"), torch.empty(
        70, 2, 128, dtype=r.q.dtype, device="cuda")
    kw = dict(q_weight=r.wq, k_weight=r.wk)
    want = ss.qk_rotate(r.q, r.k, r.pos, r.freq, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = ss.qk_rotate(r.q, r.k, r.pos, r.freq, **kw)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ss.qk_rotate(r.q, r.k, r.pos, r.freq, q_out=qo, k_out=ko_, **kw)
    for step in range(3):
        graph.replay()
        torch.cuda.synchronize()
        now = ss.qk_rotate(r.q, r.k, r.pos, r.freq, **kw)
        assert torch.equal(qo, now[0]) and torch.equal(ko_, now[1])
        r.pos += 1
        r.q *= 1.5
    torch.cuda.synchronize()
    ss.lib.sem_set_stream(ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    now = ss.qk_rotate(r.q, r.k, r.pos, r.freq, **kw)
    p = lambda t: t.data_ptr()  # noqa: E731
    c = ss.QKRotaryC(p(r.q), p(r.k), p(qo), p(ko_), r.q.stride(0), 128, r.k.stride(0), 128, 1024,
                     128, 256, 128, p(r.pos), p(r.freq), p(r.wq), p(r.wk), 70, 8, 2, 128, 128, 0, 0,
                     1e-6)
    assert ss.lib.sem_qk_rotate(ctypes.byref(c)) == 0
    assert torch.equal(qo, now[0]) and torch.equal(ko_, now[1])


def crossings(freqs, low, high, seed):
    """Positions in [low, high) with the frequency whose cosine or sine is below 2^-16 there:
    (position, frequency, the quarter turns to it, the angle beyond them), from 70 digits."""
    from decimal import Decimal, getcontext
    getcontext().prec = 70
    two_pi = Decimal("6.2831853071795864769252867665590057683943387987502116419498891846156328")
    rng = np.random.default_rng(seed)
    found = []
    for f in freqs:
        pos = rng.integers(low, high, 1 << 20)
        # (extended precision finds them: 64 bits of up to 2^29 turns)
        quarters = 4 * (pos.astype(np.longdouble) * np.longdouble(f)) / np.longdouble(str(two_pi))
        near = np.abs(quarters - np.rint(quarters)) * 1.6 < 2.0 ** -16
        for p in pos[near][:12].tolist():
            turns = 4 * Decimal(p) * Decimal(float(f)) / two_pi
            whole = turns.to_integral_value()
            found.append((p, f, int(whole) % 4, float((turns - whole) * two_pi / 4)))
    return found


@pytest.mark.parametrize("low,high", [(1 << 10, 1 << 20), (1 << 30, (1 << 31) - 1),
                                      (-(1 << 31), -(1 << 30))])
def test_far_positions_are_as_exact_as_near_ones(ss, low, high):
    """Angles beside whole quarters of a turn, whose small sines or cosines bfloat16 shows to
    2^-25: an angle is off by the rounding of its fraction of a turn to 32 bits, 2 pi 2^-26,
    whatever the position, its small sine by 2^-21 of itself more (the subtraction of the
    quarter is exact, then come the factor 2 pi and the series' last product), and by the
    output's rounding: bfloat16 has eight bits, so a step is 2^-7 of the power of two below
    a value and half of one up to 2^-8 of the value."""
    import torch
    print("far", low, flush=True)
    freqs = (1.0 - np.arange(32) / 37).astype(np.float32)
    found = crossings(freqs, low, high, 7)
    assert len(found) > 100
    x = torch.zeros(len(found), 1, 64, dtype=torch.bfloat16, device="cuda")
    x[:, :, :32] = 1.0  # (cos t, sin t) of every pair
    pos = torch.tensor([p for p, *_ in found], dtype=torch.int32, device="cuda")
    out = ss.qk_rotate(x, x, pos, torch.from_numpy(freqs).cuda())[0].double().cpu().numpy()
    worst = 0.0
    for row, (p, f, quarter, beyond) in enumerate(found):
        i = int(np.flatnonzero(freqs == f)[0])
        # cos(q pi / 2 + b), sin(q pi / 2 + b): one of them is b, but for its sign
        got = out[row, 0, i] if quarter % 2 else out[row, 0, 32 + i]
        want = beyond if quarter in (0, 3) else -beyond
        tol = 2 * np.pi * 2.0 ** -26 + (2.0 ** -8 + 2.0 ** -21) * abs(want)
        worst = max(worst, abs(got - want) / tol)
    assert worst <= 1, worst
