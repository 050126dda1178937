"""The launches of attention's gradients stay within what a HIP launch takes, on the host (no GPU): 2^32 threads, and nothing goes out
after a kernel that was refused."""
import os
import subprocess
import sys

import pytest

from test_block_abi import ROCM, STUBS, build_and_run, bwd, refused

pytest.importorskip("paper_2606_19271_amd")
from paper_2606_19271_amd import _lib  # noqa: E402
from paper_2606_19271_amd import block as B  # noqa: E402
from paper_2606_19271_amd.build import BLOCK_LIB  # noqa: E402

GRID = STUBS + r"""
namespace tsblock {
hipError_t configure_kernels() { return hipErrorUnknown; }
hipError_t launch_rope(const RopeArgs&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_rope_bwd(const RopeBwdArgs&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_attn_bwd(const BwdArgs&, hipStream_t) { return hipErrorUnknown; }
}
static uint64_t state = 5;
static int64_t rnd(int64_t n) { state = state * 6364136223846793005ull + 1442695040888963407ull; return (int64_t)(state >> 33) % n; }
static int32_t upto(int32_t bits) { return (int32_t)(rnd((int64_t)1 << 31) >> rnd(bits)); }
int main() {
  int accepted = 0, large = 0, most = 0;
  for (int i = 0; i < 500000; ++i) {
    const int32_t d = rnd(2) ? 64 : 128, H = 1 + (upto(31) >> 14), nseq = 1 + (upto(31) >> 11), n = 1 + (int32_t)rnd(16);
    const int32_t mq = upto(31) >> 3, mk = upto(31) >> 3, Tq = upto(31), Tk = upto(31);
    if (ts_attn_bwd_workspace(nseq, mq, mk, Tq, Tk, H, d, n) == 0) continue;
    ++accepted;
    const BwdParts p = bwd_parts(nseq, mq, mk, Tq, Tk, H, d, n, INT64_MAX, 1);
    const int64_t items = H * (bwd_tiles(nseq, mq, Tq, p.tile) * p.n_q + bwd_tiles(nseq, mk, Tk, p.tile) * p.n_k);
    CHECK(items * (2 * p.tile) < (int64_t)1 << 32);                                  // attn_bwd_kernel
    CHECK((1 + ((int64_t)Tq + 63) / 64 * H) * 256 < (int64_t)1 << 32);               // bwd_prepare_kernel
    CHECK((((int64_t)Tq * H + 15) / 16 + ((int64_t)Tk * H + 15) / 16) * 256 < (int64_t)1 << 32);  // bwd_join_kernel
    large += items > 1 << 20;
    most = items > most ? (int)items : most;
  }
  CHECK(accepted > 20000 && large > 100 && most > 1 << 22);
  printf("accepted %d, large %d, most %d, failures %d\n", accepted, large, most, bad);
  return bad != 0;
}
"""


def test_launches_stay_within_their_grid(tmp_path):
    build_and_run(tmp_path, GRID, "-fno-omit-frame-pointer", "-fsanitize=address,undefined", "-fno-sanitize-recover=all")


def test_forced_ranges_of_too_many_segments_are_refused():
    lib = B.load_block()
    sizes = dict(nseq=1 << 18, max_q=1, max_k=1, Tq=1 << 18, Tk=1 << 18, H=1, d=128)
    refused(bwd(lib, **sizes, n=16, bytes=1 << 36), "TS_ERR_SHAPE")
    assert lib.ts_attn_bwd_workspace(*sizes.values(), 16) == 0
    for n in (1, 15):
        assert lib.ts_attn_bwd_workspace(*sizes.values(), n) > 0


HIP = r"""
#include <hip/hip_runtime_api.h>
#include <string.h>
static int launches = 0, refuse = -1;
static unsigned long long most = 0;
static hipError_t error = hipSuccess;
extern "C" {  // in place of HIP: a device whose kernels are counted, the one numbered `refuse` being refused
void refuse_launch(int n) { refuse = n; launches = 0; }
int launched() { return launches; }
unsigned long long most_threads() { return most; }
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipGetLastError() { const hipError_t e = error; error = hipSuccess; return e; }
hipError_t hipGetDeviceProperties(hipDeviceProp_t* p, int) {
  memset(p, 0, sizeof(*p));
  strcpy(p->gcnArchName, "gfx950:sramecc+");
  p->multiProcessorCount = 256;
  return hipSuccess;
}
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { *v = 256; return hipSuccess; }
hipError_t hipFuncSetAttribute(const void*, hipFuncAttribute, int) { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus* st) { *st = hipStreamCaptureStatusNone; return hipSuccess; }
static dim3 grid_of, block_of;
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t) { grid_of = grid, block_of = block; return hipSuccess; }
hipError_t __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* lds, hipStream_t* s) {
  *grid = grid_of, *block = block_of, *lds = 0, *s = nullptr;
  return hipSuccess;
}
hipError_t hipLaunchKernel(const void*, dim3 grid, dim3 block, void**, size_t, hipStream_t) {
  const unsigned long long threads = (unsigned long long)grid.x * grid.y * grid.z * block.x * block.y * block.z;
  most = threads > most ? threads : most;
  if (launches++ == refuse) return error = hipErrorInvalidConfiguration;
  return hipSuccess;
}
}
"""

CALLS = r"""
import ctypes, sys
hip = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
hip.most_threads.restype = ctypes.c_ulonglong
lib = ctypes.CDLL(sys.argv[2])
P, I, L = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
at = [P((i + 1) << 40) for i in range(20)]
class Rows(ctypes.Structure):
    _fields_ = [("p", P), ("stride", L), ("heads", I)]
def attn(nseq, most, total, H, d, n):
    return lib.ts_attn_bwd(*at[:11], I(nseq), I(most), I(most), I(total), I(total), I(H), I(d), ctypes.c_float(0.1), I(n), at[11], L(1 << 39), None)
def rope():
    r = [ctypes.byref(Rows((i + 1) << 40, 512, 4)) for i in range(6)]
    return lib.ts_qk_rope_bwd(*r, *at[6:10], None, I(100), I(128), ctypes.c_float(1e-6), at[10], L(1 << 30), None)
TS_OK, TS_ERR_HIP = 0, int(sys.argv[3])
for call, kernels in ((lambda: attn(2, 900, 1000, 4, 64, 3), 3), (lambda: attn(2, 900, 1000, 4, 128, 3), 3), (lambda: attn(9, 9000, 50000, 12, 128, 2), 3),
                      (lambda: attn(2, 900, 1000, 4, 128, 1), 2), (rope, 2)):
    hip.refuse_launch(-1)
    rc = call()
    assert rc == TS_OK and hip.launched() == kernels, (rc, hip.launched())
    for i in range(kernels):
        hip.refuse_launch(i)
        assert call() == TS_ERR_HIP and hip.launched() == i + 1, (i, hip.launched())
hip.refuse_launch(-1)
assert attn(1 << 18, 1, 1 << 18, 1, 128, 15) == TS_OK and 1 << 31 < hip.most_threads() < 1 << 32, hip.most_threads()
print("failures 0")
"""


def test_nothing_goes_out_after_a_kernel_that_was_refused(tmp_path):
    src, so = tmp_path / "hip.cpp", str(tmp_path / "libhip.so")
    src.write_text(HIP)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I" + os.path.join(ROCM, "include"), str(src), "-o", so],
                   check=True)
    # a process of its own, in which the stand-in comes before the library's HIP
    r = subprocess.run([sys.executable, "-c", CALLS, so, BLOCK_LIB, str(_lib.TS_ERR_HIP)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "failures 0" in r.stdout, r.stdout + r.stderr
