"""Arrays of different tensors of an AdamW plan that share memory, one of them
written, are refused before anything touches a device."""
from __future__ import annotations

import ctypes as C
import os

import pytest

from paper_2410_23244_amd import bart, ops

MB = 1 << 20


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(bart.LIB_PATH):
        pytest.skip("libbart.so not built")
    return ops.lib()


def _tensor(at, **kw):
    """Arrays of 1000 f32 elements, 1 MB apart from address `at` on."""
    v = dict(param=at, grad=at + MB, master=None, m=at + 2 * MB, v=at + 3 * MB, m_scale=None,
             v_scale=None, n=1000, param_dtype=ops.BART_F32, grad_dtype=ops.BART_F32,
             weight_decay=0.0, lr_scale=1.0)
    return ops.AdamwTensor(*[(v | kw)[f] for f, _ in ops.AdamwTensor._fields_])


def _init(L, tensors, bits):
    table = (ops.AdamwTensor * len(tensors))(*tensors)
    h = C.c_void_p()
    # a workspace that is not aligned is refused after the tensors and before the device
    rc = L.bart_adamw_init(table, len(tensors), bits, MB + 8, 1 << 30, None, C.byref(h))
    assert h.value is None
    return rc


A, B, D = 64 * MB, 128 * MB, 256 * MB
PAIRS = [dict(param=A), dict(param=A + 3996), dict(param=A - 3996), dict(m=A), dict(v=A + 2 * MB),
         dict(param=A + MB), dict(grad=A), dict(grad=A + 3 * MB + 3996), dict(m=A + 3 * MB - 3996)]


@pytest.mark.parametrize("shared", PAIRS)
@pytest.mark.parametrize("order", [1, -1])
def test_shared_memory_is_refused(L, shared, order):
    t = [_tensor(A), _tensor(D), _tensor(B, **shared)][::order]
    assert _init(L, t, 32) == bart.BART_EINVAL
    assert "overlap" in L.bart_last_error().decode()


def test_the_same_tensor_twice(L):
    assert _init(L, [_tensor(A), _tensor(A)], 32) == bart.BART_EINVAL
    assert "overlap" in L.bart_last_error().decode()


def test_masters_codes_and_scales(L):
    def t(at, **kw):
        v = dict(param_dtype=ops.BART_BF16, grad_dtype=ops.BART_BF16, master=at + 4 * MB,
                 m_scale=at + 5 * MB, v_scale=at + 6 * MB)
        return _tensor(at, **(v | kw))

    assert _init(L, [t(A), t(B)], 8) == bart.BART_ENOSPACE
    for shared in (dict(master=A + 4 * MB + 3996), dict(m_scale=A + 5 * MB + 12),
                   dict(v_scale=A + 6 * MB), dict(m=A + 2 * MB + 999), dict(param=A + 1998)):
        assert _init(L, [t(A), t(B, **shared)], 8) == bart.BART_EINVAL
    for apart in (dict(master=A + 4 * MB + 4000), dict(m_scale=A + 5 * MB + 16),
                  dict(m=A + 2 * MB + 1000), dict(param=A + 2000)):
        assert _init(L, [t(A), t(B, **apart)], 8) == bart.BART_ENOSPACE


def test_neighbours_and_shared_gradients_are_taken(L):
    assert _init(L, [_tensor(A), _tensor(B)], 32) == bart.BART_ENOSPACE
    assert _init(L, [_tensor(A), _tensor(B, param=A + 4000, m=A - 4000)], 32) == bart.BART_ENOSPACE
    assert _init(L, [_tensor(A), _tensor(B, grad=A + MB)], 32) == bart.BART_ENOSPACE
    assert _init(L, [_tensor(A), _tensor(A, n=0)], 32) == bart.BART_ENOSPACE
