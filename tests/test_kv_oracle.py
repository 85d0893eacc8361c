"""The KV cache's 64-bit reference against closed forms, and the library's host
checks of KV cache arguments (no GPU is touched by any call here)."""

import ctypes
import gc
import math
import weakref

import numpy as np
import pytest

from oracle import kv_oracle as ko
from tests._lib import ensure_built


@pytest.fixture(scope="module")
def ss():
    ensure_built()
    import paper_2506_12204_amd as mod
    return mod


def test_code_values():
    v = ko.code_values(ko.FP8)
    assert np.isnan(v[[0x7f, 0xff]]).all() and np.nanmax(v) == 448.0 and v[1] == 2.0 ** -9
    assert v[0x38] == 1.0 and v[0xb8] == -1.0
    torch = pytest.importorskip("torch")
    t = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double()
    assert np.array_equal(np.nan_to_num(v, nan=9.0), np.nan_to_num(t.numpy(), nan=9.0))
    assert ko.code_values(ko.INT8)[[0, 127, 129, 255]].tolist() == [0, 127, -127, -1]


@pytest.mark.parametrize("tokens,dim", [(16, 64), (32, 128), (64, 256)])
def test_block_index_is_a_permutation(tokens, dim):
    for which in (0, 1):
        idx = ko.block_index(which, tokens, dim)
        assert sorted(idx.reshape(-1).tolist()) == list(range(tokens * dim))
    assert ko.block_index(0, tokens, dim)[1, 0] == 16  # the next token of a K tile
    assert ko.block_index(1, tokens, dim)[1, 0] == 1   # the next token of a V tile


def test_attend_closed_forms():
    rng = np.random.default_rng(0)
    v = rng.normal(size=(7, 4))
    k = np.zeros((7, 4))
    out, lse, _ = ko.attend(np.ones((2, 4)), k, v, 1.0, True, 0)  # equal scores: means
    assert np.allclose(out, [v[:6].mean(0), v.mean(0)]) and np.allclose(lse, np.log([6, 7]))
    out, lse, _ = ko.attend(np.ones((2, 4)), k, v, 1.0, True, 1)  # a window of its own key
    assert np.allclose(out, v[5:7]) and np.allclose(lse, 0)
    out, lse, _ = ko.attend(np.ones((3, 4)), k[:2], v[:2], 1.0, True, 0)  # before the first key
    assert (out[0] == 0).all() and lse[0] == -math.inf and np.allclose(out[1], v[0])
    out, _, _ = ko.attend(np.ones((1, 4)), k, v, 1.0, False, 0)
    assert np.allclose(out, v.mean(0))


def test_pages_reference():
    p = ko.Pages(8, 4, 4, 16)
    assert p.reserve([0], [20]) and p.tables[0] == [0, 1]
    p.content[:2] = ["a", "b"]
    p.fork([0, 0], [1, 2])
    assert p.refs[:2] == [3, 3]
    assert p.reserve([1, 2, 0], [1, 20, 0])
    assert p.tables[1] == [0, 2] and p.tables[2] == [0, 3, 4] and p.content[2:4] == ["b", "b"]
    assert p.refs == [3, 1, 1, 1, 1, 0, 0, 0] and p.live_words() == [31]
    assert not p.reserve([3], [64])
    p.free([0, 2], [0, 16])
    assert p.tables[2] == [0] and p.refs == [2, 0, 1, 0, 0, 0, 0, 0]
    p.compact()
    assert p.tables[1] == [0, 1] and p.content[1] == "b" and p.live_words() == [3]


def cache(ss, **over):
    fake = 1 << 40  # never dereferenced: the call fails first
    c = dict(data=fake, scale=fake, live=fake, refs=fake, lens=fake, tables=fake, num_pages=64,
             slots=8, max_blocks=16, layers=2, kv_heads=4, head_dim=128, page_tokens=64, format=0)
    c.update(over)
    return ctypes.byref(ss.KVCacheC(*[c[f[0]] for f in ss.KVCacheC._fields_]))


BAD = [dict(num_pages=-1), dict(num_pages=1 << 31), dict(slots=-1), dict(max_blocks=-1),
       dict(layers=0), dict(layers=4097), dict(kv_heads=0), dict(kv_heads=1025),
       dict(page_tokens=8), dict(page_tokens=48), dict(page_tokens=2048), dict(format=2),
       dict(max_blocks=1 << 26), dict(data=None), dict(scale=None), dict(live=None),
       dict(refs=None), dict(lens=None), dict(tables=None), dict(data=(1 << 40) + 8)]


def calls(ss, c, n=2, x=None, ws=None, ws_bytes=1 << 30, tokens=2, layer=0, dtype=0):
    """Every entry point on one cache: {name: status}."""
    x = ctypes.c_void_p(1 << 40) if x is None else x
    ws = ctypes.c_void_p(1 << 40) if ws is None else ws
    q = ss.KVQueryC((1 << 40), (1 << 40), None, 1024, 128, 1024, 128, tokens, 0, 0, 8, dtype, 1,
                    0, 0.1)
    q = ctypes.byref(q)
    a = (ws, ws_bytes, None)
    ap = (c, layer, x, x, dtype, 512, 128, 512, 128, x, None, n, tokens)
    L = ss.lib
    return {"fork": L.sem_kv_fork(c, x, x, None, n),
            "fork_async": L.sem_kv_fork_async(c, x, x, None, n, *a),
            "reserve": L.sem_kv_reserve(c, x, x, n),
            "reserve_async": L.sem_kv_reserve_async(c, x, x, n, *a),
            "free": L.sem_kv_free(c, x, None, n),
            "free_async": L.sem_kv_free_async(c, x, None, n, *a),
            "append": L.sem_kv_append(*ap), "append_async": L.sem_kv_append_async(*ap, *a),
            "attend": L.sem_kv_attend(c, layer, q, x, None, n),
            "attend_async": L.sem_kv_attend_async(c, layer, q, x, None, n, *a)}


@pytest.mark.parametrize("over", BAD, ids=[str(b) for b in BAD])
def test_bad_caches_are_refused(ss, over):
    c = cache(ss, **over)
    assert set(calls(ss, c).values()) == {ss.SEM_EINVAL}
    assert ss.lib.sem_kv_compact(c) == ss.SEM_EINVAL
    if not set(over) & {"data", "scale", "live", "refs", "lens", "tables"}:
        assert ss.lib.sem_kv_page_bytes(c) == 0 and ss.lib.sem_kv_workspace_bytes(c) == 0


def test_bad_arguments_are_refused(ss):
    L, E = ss.lib, ss.SEM_EINVAL
    c, nul, fake = cache(ss), ctypes.c_void_p(0), ctypes.c_void_p(1 << 40)
    assert L.sem_kv_page_bytes(c) == 2 * 2 * 4 * 64 * 128
    assert L.sem_kv_page_bytes(None) == 0 and L.sem_kv_compact(None) == E
    assert set(calls(ss, cache(ss, head_dim=96)).values()) == {ss.SEM_ENOTIMPL}
    assert set(calls(ss, c, n=-1, tokens=-1).values()) == {E}
    assert set(calls(ss, c, n=9, tokens=9).values()) == {E}  # more sequences than slots
    assert set(calls(ss, c, x=nul).values()) == {E}
    for name, code in calls(ss, c, ws_bytes=255).items():
        if name.endswith("_async"):
            assert code == E, name
    for name, code in calls(ss, c, ws=ctypes.c_void_p((1 << 40) + 8)).items():
        if name.endswith("_async"):
            assert code == E, name
    for over in (dict(layer=2), dict(layer=-1), dict(dtype=2), dict(tokens=3)):
        got = calls(ss, c, **over)
        assert {got[k] for k in ("append", "append_async", "attend", "attend_async")} == {E}, over
    need = L.sem_kv_workspace_bytes(c)
    assert need >= 256 + 12 * 8 + 4 * 64
    assert L.sem_kv_reserve_async(c, fake, fake, 2, fake, need - 1, None) == E
    assert L.sem_kv_compact_async(c, fake, need - 1, None) == E
    W = L.sem_kv_attend_workspace_bytes
    assert W(c, 8, 2, 2, 0, 0) >= 256 and W(c, 7, 2, 2, 0, 0) == 0 and W(c, 8, -1, 2, 0, 0) == 0
    assert W(c, 8, 2, -1, 0, 0) == 0 and W(c, 8, 2, 2, -1, 0) == 0
    good = dict(q=1 << 40, out=1 << 40, lse=None, q_token_stride=1024, q_head_stride=128,
                out_token_stride=1024, out_head_stride=128, tokens=2, max_new=0, max_len=0,
                heads=8, dtype=0, causal=1, window=0, scale=0.1)
    for over in (dict(q=None), dict(out=None), dict(q=(1 << 40) + 1), dict(out=(1 << 40) + 1),
                 dict(q_token_stride=-1), dict(out_head_stride=-1), dict(max_new=-1),
                 dict(max_len=-1), dict(heads=0), dict(heads=6), dict(window=-1),
                 dict(scale=float("nan")), dict(scale=float("inf")), dict(tokens=1 << 31)):
        q = ss.KVQueryC(*[{**good, **over}[f[0]] for f in ss.KVQueryC._fields_])
        assert L.sem_kv_attend(c, 0, ctypes.byref(q), fake, fake, 2) == E, over
    assert L.sem_kv_attend(c, 0, None, fake, None, 2) == E


def test_binding_refuses_cpu_tensors_and_sizes(ss):
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError):
        ss.KVCache(4, 2, 2, layers=1, kv_heads=1, head_dim=96, device="cpu")
    with pytest.raises(TypeError):  # there is no CPU path
        ss.KVCache(4, 2, 2, layers=1, kv_heads=1, head_dim=64, device="cpu")
    with pytest.raises(TypeError):
        ss.KVCache(4, 2, 2, layers=1, kv_heads=1, head_dim=64, device="cpu",
                   book=torch.zeros(4, dtype=torch.int64))


def test_a_replaced_workspace_stays_allocated(ss, monkeypatch):
    """Graphs hold the address of the workspace that they were captured with; a
    larger one is not taken while capturing."""
    torch = pytest.importorskip("torch")
    capturing = False
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing)
    c = ss.KVCache.__new__(ss.KVCache)  # (no device here: the workspace alone)
    c.device, c.ws_bytes, c._replaced = torch.device("cpu"), 8192, []
    c.workspace = torch.full((8192,), 5, dtype=torch.uint8)
    c._ws = c.workspace.data_ptr()
    first = weakref.ref(c.workspace)
    capturing = True
    with pytest.raises(RuntimeError):
        c._room(8193)
    assert c.workspace is first() and c.ws_bytes == 8192
    c._room(8192)  # large enough: nothing is taken
    assert c.workspace is first()
    capturing = False
    need = 8192
    for _ in range(5):
        need += 1000
        c._room(need)
        assert c.ws_bytes == c.workspace.numel() >= need and c._ws == c.workspace.data_ptr()
        assert (c.workspace == 0).all()
    gc.collect()
    assert first() is not None and (first() == 5).all()
    assert sum(w.numel() for w in c._replaced) <= c.ws_bytes


def test_grids_that_cannot_be_launched_are_refused(ss, monkeypatch):
    """Calls whose threads pass 32 bits, with every pointer in order; nothing is
    launched."""
    L, big = ss.lib, 1 << 24
    x = ctypes.c_void_p(1 << 40)
    a = (x, 1 << 50, None)
    c = cache(ss, slots=big, max_blocks=1, layers=1, kv_heads=1, head_dim=64, page_tokens=16)
    assert L.sem_kv_fork_async(c, x, x, None, big, *a) == ss.SEM_ENOTIMPL
    assert L.sem_kv_free_async(c, x, None, big, *a) == ss.SEM_ENOTIMPL
    rows = (0, 64, 64, 64, 64, x)
    assert L.sem_kv_append_async(c, 0, x, x, *rows, None, big, big, *a) == ss.SEM_ENOTIMPL
    assert L.sem_kv_append_async(c, 0, x, x, *rows, x, big // 2, 1 << 20, *a) == ss.SEM_ENOTIMPL
    assert L.sem_kv_append_async(c, 0, x, x, *rows, x, 1, 1 << 28, *a) == ss.SEM_ENOTIMPL

    def attend(cache, heads, n, tokens, cu, max_new=0):
        q = ss.KVQueryC(1 << 40, 1 << 40, None, heads * 64, 64, heads * 64, 64, tokens, max_new, 0,
                        heads, 0, 1, 0, 0.1)
        return L.sem_kv_attend_async(cache, 0, ctypes.byref(q), x, cu, n, *a)

    assert attend(c, 1, big, big, None) == ss.SEM_ENOTIMPL
    assert attend(c, 1, big - 1, big, x) == ss.SEM_ENOTIMPL  # with those that check offsets
    wide = cache(ss, slots=1 << 18, max_blocks=1, layers=1, kv_heads=64, head_dim=64, page_tokens=16)
    assert attend(wide, 64, 1 << 18, 1 << 18, None) == ss.SEM_ENOTIMPL
    monkeypatch.setenv("SEMSCHED_KV_TILES", "1")  # tiles of 512 threads
    assert attend(c, 64, 1 << 23, 1 << 23, None) == ss.SEM_ENOTIMPL


def test_rows_of_no_sequence_are_refused(ss):
    fake = ctypes.c_void_p(1 << 40)
    c = cache(ss)
    q = ss.KVQueryC(1 << 40, 1 << 40, None, 1024, 128, 1024, 128, 5, 0, 0, 8, 0, 1, 0, 0.1)
    assert ss.lib.sem_kv_attend(c, 0, ctypes.byref(q), fake, fake, 0) == ss.SEM_EINVAL
    assert ss.lib.sem_kv_append(c, 0, fake, fake, 0, 512, 128, 512, 128, fake, fake, 0,
                                5) == ss.SEM_EINVAL
