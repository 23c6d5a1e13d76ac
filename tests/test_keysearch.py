"""The search for a threshold among distinct 64-bit keys (csrc/keysearch.hpp),
compiled for the host: however the keys lie, a threshold that at least k and at
most `most` keys reach is found within 64 counts."""
from __future__ import annotations

import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CXX = shutil.which("g++") or shutil.which("c++")

SOURCE = r"""
#include <algorithm>
#include "keysearch.hpp"
// Sorted keys; the number of counts until one fits, its threshold in *at.
extern "C" int search(const uint64_t *key, uint32_t n, uint64_t lo, uint32_t k, uint32_t most,
                      uint64_t *at) {
  bart::KeySearch s{lo, ~(uint64_t)0};
  for (int i = 1; i <= 1000; ++i) {
    *at = s.probe();
    const uint32_t count = (uint32_t)(key + n - std::lower_bound(key, key + n, *at));
    if (count >= k && count <= most) return i;
    s.take(*at, count, k);
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def search(tmp_path_factory):
    if CXX is None:
        pytest.skip("no host C++ compiler")
    d = tmp_path_factory.mktemp("keysearch")
    src, so = d / "search.cpp", d / "search.so"
    src.write_text(SOURCE)
    subprocess.run([CXX, "-std=c++17", "-O2", "-shared", "-fPIC", "-I",
                    os.path.join(ROOT, "paper_2410_23244_amd", "csrc"), str(src), "-o", str(so)],
                   check=True, capture_output=True)
    f = C.CDLL(str(so)).search
    f.argtypes = [C.c_void_p, C.c_uint32, C.c_uint64, C.c_uint32, C.c_uint32,
                  C.POINTER(C.c_uint64)]
    f.restype = C.c_int
    return f


def _keys(x):
    """Keys of f32 scores in class order, as the kernels make them."""
    b = (x.astype(np.float32) + np.float32(0)).view(np.uint32).astype(np.uint64)
    u = np.where(b >> 31, ~b & 0xFFFFFFFF, b | 0x80000000)
    j = np.arange(len(x), dtype=np.uint64)
    return np.sort(u << np.uint64(32) | (~j & np.uint64(0xFFFFFFFF)))


def _cases():
    rng = np.random.default_rng([2410, 23244, 62])
    n = 1 << 18
    yield "ascending", _keys(np.arange(n) + 1.0)
    yield "equal", _keys(np.full(n, 3.0))
    yield "equal, -inf among them", _keys(np.where(np.arange(n) % 3 == 0, -np.inf, 0.0))
    yield "normal", _keys(rng.normal(size=n))
    yield "negative", _keys(-np.exp(rng.normal(0, 20, n)))
    yield "halves", _keys(np.float32(2.0) ** -(np.arange(n) % 250 - 120.0))
    yield "one above the rest", _keys(np.where(np.arange(n) == n - 1, 3e38, -3e38))
    yield "infinite", _keys(np.where(np.arange(n) % 2 == 0, np.inf, -1.0))
    yield "dense words", np.arange(n, dtype=np.uint64) + np.uint64(1 << 40)
    yield "powers of two", np.sort(np.uint64(1) << np.arange(64, dtype=np.uint64))
    yield "random words", np.unique(rng.integers(0, 2 ** 64 - 1, n, dtype=np.uint64))


@pytest.mark.parametrize("name,keys", list(_cases()), ids=lambda v: v if isinstance(v, str) else "")
@pytest.mark.parametrize("k", [1, 3, 20, 64])
@pytest.mark.parametrize("most", [64, 256, 1024])
def test_at_most_64_counts(search, name, keys, k, most):
    keys = np.ascontiguousarray(keys)
    for lo in {0, int(keys[0]), int(keys[-k])}:
        at = C.c_uint64()
        counts = search(keys.ctypes.data, len(keys), lo, k, most, C.byref(at))
        assert 1 <= counts <= 64
        reach = int((keys >= np.uint64(at.value)).sum())
        assert k <= reach <= most
