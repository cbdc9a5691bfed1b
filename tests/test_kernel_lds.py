"""The LDS that launches of hg_muon_step ask for, against what their kernels were
allowed before (no GPU is needed: a library of stand-ins for the runtime's calls,
loaded first, writes down what it is asked for and launches nothing)."""
import os
import shutil
import subprocess
import sys

import pytest

pytest.importorskip("torch")

from paper_2608_02168_amd import api

# hipFuncAttributeMaxDynamicSharedMemorySize is 8
STAND_INS = r"""
#include <stdio.h>
typedef struct { unsigned x, y, z; } dim;
int hipGetDevice(int* d) { *d = 0; return 0; }
int hipGetLastError(void) { return 0; }
int hipDeviceGetAttribute(int* n, int what, int device) { *n = 256; return 0; }
int hipFuncSetAttribute(const void* f, int what, int value) { printf("allow %p %d %d\n", f, what, value); return 0; }
static dim grid_, block_;
static size_t lds_;
static void* stream_;
int __hipPushCallConfiguration(dim grid, dim block, size_t lds, void* stream) {
  grid_ = grid, block_ = block, lds_ = lds, stream_ = stream;
  return 0;
}
int __hipPopCallConfiguration(dim* grid, dim* block, size_t* lds, void** stream) {
  *grid = grid_, *block = block_, *lds = lds_, *stream = stream_;
  return 0;
}
int hipLaunchKernel(const void* f, dim grid, dim block, void** args, size_t lds, void* stream) {
  printf("launch %p %u %zu\n", f, block.x, lds);
  return 0;
}
"""
CALLS = r"""
import ctypes as C, struct, sys
C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
L = C.CDLL(sys.argv[2])
L.hg_muon_workspace_size.restype = C.c_size_t
L.hg_muon_step.argtypes = [C.c_char_p] + [C.c_void_p] * 4 + [C.c_size_t, C.c_void_p]
for m, n, dtype in eval(sys.argv[3]):
    d = struct.pack("@iiiiiifffffi", 1, m, n, dtype, 5, 1, 0.1, 0.9, 0.0, 1.0, 1e-7, 0)
    size = L.hg_muon_workspace_size(d)
    assert L.hg_muon_step(d, 1 << 32, 2 << 32, 3 << 32, 4 << 32, size, None) == 0
"""
SMALL_STATIC = 8192  # of the one-block kernel (1024 threads): the norm's sums


def asked(tmp_path, calls):
    src, lib = tmp_path / "calls.c", tmp_path / "calls.so"
    src.write_text(STAND_INS)
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(lib), str(src)], check=True)
    out = subprocess.run([sys.executable, "-c", CALLS, str(lib), api.LIB_PATH, repr(calls)], check=True, capture_output=True,
                         text=True, timeout=120).stdout
    return [line.split() for line in out.splitlines()]


@pytest.mark.parametrize("calls", [
    [(63, 200, 0), (64, 544, 0)],                     # a larger matrix after a smaller one, on the same kernel
    [(64, 190, 0)], [(64, 190, 1)], [(30, 440, 0)], [(32, 470, 1)],   # 60 or 64 KB beside the static 8
    [(128, 128, 1), (128, 170, 1), (16, 16, 0), (300, 500, 0), (4096, 8192, 1)]])
def test_launches_are_allowed_their_lds(tmp_path, calls):
    if not shutil.which("gcc") or not os.path.exists(api.LIB_PATH):
        pytest.skip("gcc or libhg.so is missing")
    allowed, launches = {}, 0
    for what, f, a, b in asked(tmp_path, calls):
        if what == "allow":
            assert int(a) == 8
            allowed[f] = int(b)
            continue
        launches += 1
        threads, lds = int(a), int(b)
        static = SMALL_STATIC if threads == 1024 else 0
        assert lds + static <= 160 * 1024
        if lds + static > 64 * 1024:
            assert allowed.get(f, 0) >= lds, (threads, lds, allowed.get(f))
    assert launches >= len(calls)
