"""Attention weights of cached tokens: the reference's closed forms and the library's
host checks (no GPU is touched by any call here)."""

import ctypes

import numpy as np

from oracle import kv_oracle as ko
from tests.test_kv_oracle import cache, ss  # noqa: F401


def test_reference_closed_forms():
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(3, 4)), rng.normal(size=(9, 4)), rng.normal(size=(9, 1))
    for causal, window in ((True, 0), (True, 2), (False, 0)):
        out, lse, _ = ko.attend(q, k, v, 0.5, causal, window)
        w = ko.weigh(q, k, 0.5, causal, window, lse)
        assert np.isclose(w.sum(), 3) and (w >= 0).all()  # a row's weights add up to 1
        assert np.isclose(w @ v[:, 0], out[:, 0].sum())
    assert (ko.weigh(q, k, 0.5, True, 1, lse)[:6] == 0).all()
    lse[1] = -np.inf
    assert np.isclose(ko.weigh(q, k, 0.5, False, 0, lse).sum(), 2)
    # equal scores: equal weights
    assert np.allclose(ko.weigh(q[:1], 0 * k, 1.0, False, 0, [np.log(9)]), 1 / 9)


GOOD = dict(q=1 << 40, out=None, lse=1 << 40, q_token_stride=1024, q_head_stride=128,
            out_token_stride=-5, out_head_stride=0, tokens=2, max_new=0, max_len=0, heads=8,
            dtype=0, causal=1, window=0, scale=0.1)


def weigh(ss, c, n=2, layer=0, mass=1 << 40, stride=1024, **over):  # noqa: F811
    p = ctypes.c_void_p
    q = ctypes.byref(ss.KVQueryC(*[{**GOOD, **over}[f[0]] for f in ss.KVQueryC._fields_]))
    a = (c, layer, q, p(1 << 40), p(1 << 40), n, p(mass), stride)
    return {ss.lib.sem_kv_weigh(*a), ss.lib.sem_kv_weigh_async(*a, p(1 << 40), 1 << 30, None)}


def test_bad_arguments_are_refused(ss):  # noqa: F811
    E, c = {ss.SEM_EINVAL}, cache(ss)
    for over in (dict(n=-1), dict(n=9), dict(n=0), dict(layer=2), dict(layer=-1), dict(mass=0),
                 dict(mass=(1 << 40) + 2), dict(stride=1023), dict(stride=-1), dict(q=None),
                 dict(lse=None), dict(q=(1 << 40) + 1), dict(q_token_stride=-1), dict(tokens=-1),
                 dict(max_len=-1), dict(heads=6), dict(dtype=2), dict(window=-1),
                 dict(scale=float("nan"))):
        assert weigh(ss, c, **over) == E, over
    for bad in (dict(slots=-1), dict(tables=None), dict(page_tokens=8)):
        assert weigh(ss, cache(ss, **bad)) == E
    assert weigh(ss, cache(ss, head_dim=96)) == {ss.SEM_ENOTIMPL}
    x = ctypes.c_void_p(1 << 40)
    assert ss.lib.sem_kv_weigh(c, 0, None, x, x, 2, x, 1024) == ss.SEM_EINVAL
    q = ctypes.byref(ss.KVQueryC(*GOOD.values()))
    for ws, size in ((None, 1 << 30), (x, 4351), (ctypes.c_void_p((1 << 40) + 8), 1 << 30)):
        assert ss.lib.sem_kv_weigh_async(c, 0, q, x, x, 2, x, 1024, ws, size, None) == ss.SEM_EINVAL
    # as many rows as attention takes
    assert weigh(ss, c, tokens=1 << 29) == {ss.SEM_ENOTIMPL}
