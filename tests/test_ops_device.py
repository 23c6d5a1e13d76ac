"""A step of an AdamW plan leaves the caller's device as it was.  Without a GPU:
a child process loads stand-ins for the few runtime calls that the entry points
make before it loads the library."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

import pytest

from paper_2410_23244_amd import bart

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CC = shutil.which("gcc") or shutil.which("cc")

RUNTIME = r"""
#include <stddef.h>
#include <string.h>
typedef struct { unsigned x, y, z; } dim3;
static int device, launches[8], error;
int now(void) { return device; }
int launched(int d) { return launches[d]; }
void fail_from_now(void) { error = 1; }
int hipGetDevice(int *d) { *d = device; return 0; }
int hipSetDevice(int d) { device = d; return 0; }
int hipMemcpyAsync(void *to, const void *from, size_t n, int kind, void *stream) { return 0; }
int hipStreamSynchronize(void *stream) { return 0; }
int hipGetLastError(void) { return error; }
int __hipPushCallConfiguration(dim3 grid, dim3 block, size_t shared, void *stream) { return 0; }
int __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *shared, void **stream) {
  memset(grid, 0, sizeof *grid);
  memset(block, 0, sizeof *block);
  *shared = 0;
  *stream = 0;
  return 0;
}
int hipLaunchKernel(const void *f, dim3 grid, dim3 block, void **args, size_t shared, void *stream) {
  ++launches[device];
  return 0;
}
"""

CHILD = r"""
import ctypes as C, sys
rt = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
sys.path.insert(0, sys.argv[2])
from paper_2410_23244_amd import ops
L = ops.lib()
P = 1 << 20
t = ops.AdamwTensor(P, 2 * P, None, 3 * P, 4 * P, None, None, 100, ops.BART_F32, ops.BART_F32, 0.0,
                    1.0)
h, y = C.c_void_p(), ops.AdamwHyper(1e-3, 0.9, 0.999, 1e-8, 1.0, 1)
rt.hipSetDevice(1)
assert L.bart_adamw_init(t, 1, 32, P, 1 << 20, None, C.byref(h)) == 0 and rt.now() == 1
for d in (1, 0, 3):
    rt.hipSetDevice(d)
    assert L.bart_adamw_step(h, y, None) == 0
    print("device", rt.now(), "launches", rt.launched(1), rt.launched(0) + rt.launched(3))
rt.fail_from_now()
assert L.bart_adamw_step(h, y, None) == -3
print("device", rt.now())
L.bart_adamw_destroy(h)
"""


@pytest.mark.skipif(CC is None, reason="no host C compiler")
def test_a_step_leaves_the_current_device_as_it_was(tmp_path):
    if not os.path.exists(bart.LIB_PATH):
        pytest.skip("libbart.so not built")
    (tmp_path / "runtime.c").write_text(RUNTIME)
    so = str(tmp_path / "runtime.so")
    subprocess.run([CC, "-shared", "-fPIC", str(tmp_path / "runtime.c"), "-o", so], check=True,
                   capture_output=True)
    out = subprocess.run([sys.executable, "-c", CHILD, so, ROOT], capture_output=True, text=True,
                         timeout=300)
    assert out.returncode == 0, out.stderr
    assert out.stdout.splitlines() == ["device 1 launches 1 0", "device 0 launches 2 0",
                                       "device 3 launches 3 0", "device 3"]
