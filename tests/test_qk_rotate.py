"""The norms and rotation of queries and keys: the 64-bit reference against closed
forms, and the library's host checks (no GPU is touched by any call here)."""

import ctypes
import math

import numpy as np
import pytest

from oracle import kv_oracle as ko
from tests._lib import ensure_built


@pytest.fixture(scope="module")
def ss():
    ensure_built()
    import paper_2506_12204_amd as mod
    return mod


def test_reference_closed_forms():
    x = np.arange(1.0, 9.0).reshape(1, 1, 8)
    still, _ = ko.rotate(x, None, 0, [0], [1.0, 0.5], False)
    assert (still == x).all()
    # a quarter turn: (a, b) -> (-b, a)
    turned, mag = ko.rotate(x, None, 0, [1], [math.pi / 2], True)
    assert np.allclose(turned[0, 0, :4], [-2, 1, 3, 4]) and mag[0, 0, :3].tolist() == [3, 3, 3]
    turned, _ = ko.rotate(x, None, 0, [2], [math.pi / 4, 0.0], False)
    assert np.allclose(turned[0, 0], [-3, 2, 1, 4, 5, 6, 7, 8])
    back, _ = ko.rotate(turned, None, 0, [-2], [math.pi / 4, 0.0], False)
    assert np.allclose(back, x)
    normed, _ = ko.rotate(x, np.full(8, 2.0), 0.0, [7], [], False)
    assert math.isclose((normed ** 2).mean(), 4.0)
    assert (ko.rotate(0 * x, np.ones(8), 1e-6, [7], [], False)[0] == 0).all()


GOOD = dict(q=1 << 40, k=1 << 40, q_out=1 << 40, k_out=1 << 40, q_token_stride=1024,
            q_head_stride=128, k_token_stride=512, k_head_stride=128, q_out_token_stride=1024,
            q_out_head_stride=128, k_out_token_stride=512, k_out_head_stride=128,
            positions=1 << 40, inv_freq=1 << 40, q_weight=None, k_weight=None, tokens=3, heads=8,
            kv_heads=4, head_dim=128, rot_dim=128, dtype=0, interleaved=0, eps=1e-6)


def status(ss, **over):
    r = ss.QKRotaryC(*[{**GOOD, **over}[f[0]] for f in ss.QKRotaryC._fields_])
    codes = {ss.lib.sem_qk_rotate(ctypes.byref(r)), ss.lib.sem_qk_rotate_async(ctypes.byref(r), None)}
    assert len(codes) == 1, over
    return codes.pop()


@pytest.mark.parametrize("over", [
    dict(q=None), dict(k=None), dict(q_out=None), dict(k_out=None), dict(positions=None),
    dict(inv_freq=None), dict(q=(1 << 40) + 1), dict(k_out=(1 << 40) + 1),
    dict(positions=(1 << 40) + 2), dict(inv_freq=(1 << 40) + 2), dict(q_weight=(1 << 40) + 2),
    dict(k_weight=(1 << 40) + 1), dict(q_token_stride=-1), dict(k_out_head_stride=-1),
    dict(tokens=-1), dict(tokens=1 << 31), dict(heads=-1), dict(kv_heads=-1), dict(rot_dim=-16),
    dict(rot_dim=8), dict(rot_dim=144), dict(dtype=2), dict(dtype=-1), dict(eps=-1e-6),
    dict(eps=float("nan")), dict(eps=float("inf"))], ids=str)
def test_bad_arguments_are_refused(ss, over):
    assert status(ss, **over) == ss.SEM_EINVAL


def test_sizes_that_are_not_there(ss):
    assert ss.lib.sem_qk_rotate(None) == ss.SEM_EINVAL
    assert status(ss, head_dim=96, rot_dim=96) == ss.SEM_ENOTIMPL
    assert status(ss, heads=1 << 17) == ss.SEM_ENOTIMPL
    # more threads than a launch may have, with every pointer in order: nothing is launched
    r = ss.QKRotaryC(*[{**GOOD, "head_dim": 256, "heads": 4096, "kv_heads": 0,
                        "tokens": (1 << 31) - 1}[f[0]] for f in ss.QKRotaryC._fields_])
    assert ss.lib.sem_qk_rotate_async(ctypes.byref(r), None) == ss.SEM_ENOTIMPL


def test_binding_refuses_what_it_cannot_take(ss):
    torch = pytest.importorskip("torch")
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(TypeError):  # there is no CPU path
        ss.qk_rotate(q, q, torch.zeros(2, dtype=torch.int32), torch.zeros(32))
    with pytest.raises(TypeError):
        ss.qk_rotate(q.float(), q.float(), torch.zeros(2, dtype=torch.int32), torch.zeros(32))
