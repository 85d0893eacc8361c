"""Pruning by attention weights: the reference's closed forms and the library's host
checks (no GPU is touched by any call here)."""

import ctypes

from oracle import kv_oracle as ko
from tests.test_kv_oracle import cache, ss  # noqa: F401


def test_reference_closed_forms():
    nan, inf = float("nan"), float("inf")
    pick = ko.prune_choice
    assert pick([1, 5, 2, 4, 3], 5, 3, 0, 0) == [1, 3, 4]
    assert pick([1, 5, 2, 4, 3], 5, 3, 1, 1) == [0, 1, 4]
    assert pick([1, 5, 2, 4, 3], 5, 5, 1, 1) == [0, 1, 2, 3, 4] == pick([0] * 9, 5, 7, 0, 0)
    assert pick([7, 7, 7, 7], 4, 2, 0, 0) == [0, 1] and pick([0.0, -0.0, 0.0], 3, 1, 0, 0) == [0]
    assert pick([nan, -inf, nan, 0], 4, 2, 0, 0) == [1, 3] and pick([nan] * 4, 4, 3, 0, 0) == [0, 1, 2]
    assert pick([1, 2, 3, 4], 4, 2, 5, 5) == [0, 1] and pick([9, 9, 3, 4], 4, 2, 0, 5) == [2, 3]
    assert pick([1, 2], 2, 0, 1, 1) == []


def prune(ss, c, mass=1 << 40, stride=1024, seqs=1 << 40, n=2, budget=5, sinks=1, recent=1):  # noqa: F811
    p = ctypes.c_void_p
    a = (c, p(mass), stride, p(seqs), n, budget, sinks, recent)
    return {ss.lib.sem_kv_prune(*a), ss.lib.sem_kv_prune_async(*a, p(1 << 40), 1 << 40, None)}


def test_bad_arguments_are_refused(ss):  # noqa: F811
    E, c = {ss.SEM_EINVAL}, cache(ss)
    for over in (dict(n=-1), dict(n=9), dict(seqs=0), dict(mass=0), dict(mass=(1 << 40) + 2),
                 dict(stride=1023), dict(stride=-1), dict(budget=-1), dict(sinks=-1),
                 dict(recent=-1)):
        assert prune(ss, c, **over) == E, over
    for bad in (dict(slots=-1), dict(tables=None), dict(page_tokens=8), dict(live=None)):
        assert prune(ss, cache(ss, **bad)) == E
    assert prune(ss, cache(ss, head_dim=96)) == {ss.SEM_ENOTIMPL}
    W = ss.lib.sem_kv_prune_workspace_bytes
    need = W(c, 2, 100)
    assert need >= 4352 + 2 * 32 + 8 * 200 + 4 * 4 * 16
    assert W(c, -1, 3) == 0 and W(c, 9, 3) == 0 and W(c, 2, -1) == 0
    assert W(c, 2, 1 << 62) == W(c, 2, 1024)  # no more than a sequence holds
    x = ctypes.c_void_p(1 << 40)
    for ws, size in ((None, 1 << 30), (x, need - 1), (ctypes.c_void_p((1 << 40) + 8), 1 << 30)):
        assert ss.lib.sem_kv_prune_async(c, x, 1024, x, 2, 100, 0, 0, ws, size,
                                         None) == ss.SEM_EINVAL
    wide = cache(ss, slots=1 << 23, max_blocks=1, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    assert ss.lib.sem_kv_prune_async(wide, x, 16, x, 1 << 23, 3, 0, 0, x, 1 << 62,
                                     None) == ss.SEM_ENOTIMPL  # more threads than a launch may have
