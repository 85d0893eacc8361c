"""Trees of drafted tokens: the reference's closed forms and the library's host
checks (no GPU is touched by any call here)."""

import ctypes

import numpy as np
import pytest

from oracle import kv_oracle as ko
from tests.test_kv_oracle import cache, ss  # noqa: F401


def test_reference_closed_forms():
    chain, depth = ko.tree([-1, 0, 1, 2])
    assert chain == [{0}, {0, 1}, {0, 1, 2}, {0, 1, 2, 3}] and depth == [0, 1, 2, 3]
    sets, depth = ko.tree([-1, -1, 0, 2, 1])
    assert sets[3] == {0, 2, 3} and sets[4] == {1, 4} and depth == [0, 0, 1, 2, 1]
    assert ko.tree_words(sets, 2) == [[1, 0], [2, 0], [5, 0], [13, 0], [18, 0]]
    assert ko.tree_words([{0, 31, 32, 65}], 3) == [[0x80000001, 1, 2]]
    assert ko.tree_keys([{0}, {1}], 4) == [[0, 1, 2], [0, 1, 3]]
    assert ko.tree_keys([{0}, {0, 1}, {2}], 2) == [[], [0], [1]]  # the first has no key
    # a chain sees what the causal mask shows
    rng = np.random.default_rng(0)
    q, k, v = rng.normal(size=(3, 4)), rng.normal(size=(9, 4)), rng.normal(size=(9, 4))
    a = ko.attend(q, k, v, 0.5, True, 0)
    b = ko.attend(q, k, v, 0.5, True, 0, ko.tree_keys(ko.tree([-1, 0, 1])[0], 9))
    assert all(np.allclose(x, y) for x, y in zip(a, b))


GOOD = dict(q=1 << 40, out=1 << 40, lse=None, q_token_stride=1024, q_head_stride=128,
            out_token_stride=1024, out_head_stride=128, tokens=2, max_new=0, max_len=0, heads=8,
            dtype=0, causal=1, window=0, scale=0.1)


def attend(ss, c, words=1, mask=1 << 40, n=2, layer=0, ws=1 << 40, ws_bytes=1 << 30, **over):  # noqa: F811
    """The statuses of both forms of a call that fails."""
    x = ctypes.c_void_p(1 << 40)
    q = ctypes.byref(ss.KVQueryC(*[{**GOOD, **over}[f[0]] for f in ss.KVQueryC._fields_]))
    a = (c, layer, q, ctypes.c_void_p(mask), words, x, x, n)
    return {ss.lib.sem_kv_attend_tree(*a),
            ss.lib.sem_kv_attend_tree_async(*a, ctypes.c_void_p(ws), ws_bytes, None)}


def tree(ss, c, parents=1 << 40, words=1, mask=1 << 40, positions=1 << 40, n=2, tokens=2,  # noqa: F811
         cu=1 << 40):
    p = ctypes.c_void_p
    a = (c, p(parents), None, p(1 << 40), p(cu), n, tokens, words, p(mask), p(positions))
    return {ss.lib.sem_kv_tree(*a), ss.lib.sem_kv_tree_async(*a, p(1 << 40), 1 << 30, None)}


def test_bad_arguments_are_refused(ss):  # noqa: F811
    E, c = {ss.SEM_EINVAL}, cache(ss)
    for over in (dict(words=0), dict(words=129), dict(words=-1), dict(mask=0), dict(causal=0),
                 dict(window=5), dict(q=None), dict(heads=6), dict(n=9), dict(n=0), dict(layer=2),
                 dict(dtype=3), dict(tokens=-1)):
        assert attend(ss, c, **over) == E, over
    for over in (dict(words=0), dict(words=129), dict(mask=0), dict(positions=0), dict(parents=0),
                 dict(n=-1), dict(n=9), dict(n=0), dict(tokens=-1), dict(tokens=1 << 31),
                 dict(tokens=3, cu=0)):
        assert tree(ss, c, **over) == E, over
    for bad in (dict(slots=-1), dict(tables=None), dict(page_tokens=8)):
        assert attend(ss, cache(ss, **bad)) == E and tree(ss, cache(ss, **bad)) == E
    assert attend(ss, cache(ss, head_dim=96)) == {ss.SEM_ENOTIMPL}
    x = ctypes.c_void_p(1 << 40)
    q = ctypes.byref(ss.KVQueryC(*GOOD.values()))
    for ws, size in ((None, 1 << 30), (x, 255), (ctypes.c_void_p((1 << 40) + 8), 1 << 30)):
        assert ss.lib.sem_kv_attend_tree_async(c, 0, q, x, 1, x, x, 2, ws, size,
                                               None) == ss.SEM_EINVAL
        assert ss.lib.sem_kv_tree_async(c, x, None, x, x, 2, 2, 1, x, x, ws, size,
                                        None) == ss.SEM_EINVAL
    # more threads than a launch may have
    big = 1 << 24
    wide = cache(ss, slots=big, max_blocks=1, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    assert ss.lib.sem_kv_tree_async(wide, x, None, x, None, big, big, 1, x, x, x, 1 << 30,
                                    None) == ss.SEM_ENOTIMPL
