"""Keeping tokens: the reference's closed forms and the library's host checks (no GPU
is touched by any call here)."""

import ctypes

import numpy as np
import pytest

from oracle import kv_oracle as ko
from tests.test_kv_oracle import cache, ss  # noqa: F401


@pytest.mark.parametrize("fmt", [ko.INT8, ko.FP8])
def test_requantized(fmt):
    codes = np.array([b for b in range(256) if b not in (128, 127, 255)], np.uint8)
    val = ko.code_values(fmt)
    assert (val[ko.requantized(codes, 0.3, 0.3, fmt)] == val[codes]).all()
    got, x = val[ko.requantized(codes, 1.0, 3.0, fmt)], val[codes] / 3
    near = np.sort(val[~np.isnan(val)])
    best = np.abs(near[None] - x[:, None]).min(1)
    assert (np.abs(got - x) <= best + 1e-5).all()
    # ties go to the even code
    one, three = (1, 3) if fmt == ko.INT8 else (0x01, 0x03)
    assert ko.requantized(np.array([one, three], np.uint8), 1.0, 2.0, fmt).tolist() == [0, 2]
    torch = pytest.importorskip("torch")
    if fmt == ko.FP8:
        t = torch.from_numpy(val[codes] * 0.7).float().to(torch.float8_e4m3fn).double().numpy()
        assert (val[ko.requantized(codes, 0.7, 1.0, fmt)] == t).all()


def test_keep_tokens():
    geom = (1, 1, 16, 16, ko.INT8)
    data = np.zeros((3, 2 * 256), np.uint8)
    for p in range(3):
        for w in (0, 1):
            data[p].reshape(2, 256)[w][ko.block_index(w, 16, 16)] = np.arange(16)[:, None] + 16 * p
    scale = np.array([1.0, 2.0, 4.0], np.float32).reshape(3, 1, 1, 1).repeat(2, 2)
    table = [1, 2, 0]  # scales 2, 4, 1; codes 16.., 32.., 0..
    was = data.copy()
    assert list(ko.keep_tokens(data, scale, geom, table, [0, 1, 2])) == []
    assert (data == was).all()
    assert list(ko.keep_tokens(data, scale, geom, table, [0, 2, 33])) == [0]
    k = data[1].reshape(2, 256)[0][ko.block_index(0, 16, 16)]
    assert k[0, 0] == 16 and k[1, 0] == 18 and k[2, 0] == 0 and k[3, 0] == 19  # 1 * 1 / 2 to even
    assert scale[1, 0].tolist() == [[2.0], [2.0]] and (data[[0, 2]] == was[[0, 2]]).all()


def keep(ss, c, n=2, total=3, seqs=1 << 40, last=1 << 40, index=1 << 40, cu=1 << 40):  # noqa: F811
    p = ctypes.c_void_p
    a = (c, p(seqs), p(last), p(index), p(cu), n, total)
    return {ss.lib.sem_kv_keep(*a), ss.lib.sem_kv_keep_async(*a, p(1 << 40), 1 << 40, None)}


def test_bad_arguments_are_refused(ss):  # noqa: F811
    E, c = {ss.SEM_EINVAL}, cache(ss)
    for over in (dict(n=-1), dict(n=9), dict(total=-1), dict(total=1 << 31), dict(n=0), dict(seqs=0),
                 dict(last=0), dict(index=0), dict(cu=0)):
        assert keep(ss, c, **over) == E, over
    for bad in (dict(slots=-1), dict(tables=None), dict(page_tokens=8), dict(refs=None)):
        assert keep(ss, cache(ss, **bad)) == E
    assert keep(ss, cache(ss, head_dim=96)) == {ss.SEM_ENOTIMPL}
    need = ss.lib.sem_kv_keep_workspace_bytes(c, 2, 3)
    assert need >= 4352 + 2 * 32 + 8 * (3 + 2 * 64) + 4 * 4 * 16
    assert ss.lib.sem_kv_keep_workspace_bytes(c, -1, 3) == 0
    assert ss.lib.sem_kv_keep_workspace_bytes(c, 9, 3) == 0
    assert ss.lib.sem_kv_keep_workspace_bytes(c, 2, -1) == 0
    x = ctypes.c_void_p(1 << 40)
    for ws, size in ((None, 1 << 30), (x, need - 1), (ctypes.c_void_p((1 << 40) + 8), 1 << 30)):
        assert ss.lib.sem_kv_keep_async(c, x, x, x, x, 2, 3, ws, size, None) == ss.SEM_EINVAL
    wide = cache(ss, slots=1 << 20, max_blocks=1, layers=256, kv_heads=64, head_dim=64,
                 page_tokens=16)  # more threads than a launch may have
    assert ss.lib.sem_kv_keep_async(wide, x, x, x, x, 1 << 20, 3, x, 1 << 62,
                                    None) == ss.SEM_ENOTIMPL
