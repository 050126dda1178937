"""Set-up of a device by the session cache's host code (csrc/ts_cache.cpp, csrc/cache_plan.cpp), compiled with g++ together with
a driver that stands in for HIP: a device's first call under stream capture is refused, whatever was asked before, and
the workspace query, which has no stream, sets nothing up."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_19271_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")

DRIVER = r"""
#include <hip/hip_runtime_api.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>
#include "cache_launch.h"
#include "ts_cache.h"
static int configured = 0, launches = 0;
static const hipStream_t capturing = (hipStream_t)16, eager = (hipStream_t)32;
namespace tscache {  // in place of the kernels
hipError_t configure_kernels() { ++configured; return hipSuccess; }
hipError_t launch_attn(const AttnArgs&, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_weigh(const WeighArgs&, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_append(const AppendArgs&, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_evict(const EvictArgs&, hipStream_t) { ++launches; return hipSuccess; }
}
extern "C" {  // in place of HIP: one device, one stream being captured (which the null stream's state cannot be asked during)
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipGetDeviceProperties(hipDeviceProp_t* p, int) {
  memset(p, 0, sizeof(*p));
  strcpy(p->gcnArchName, "gfx950:sramecc+");
  p->multiProcessorCount = 256;
  return hipSuccess;
}
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { *v = 256; return hipSuccess; }
hipError_t hipMemcpyAsync(void*, const void*, size_t, hipMemcpyKind, hipStream_t) { return hipErrorUnknown; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipErrorUnknown; }
hipError_t hipStreamIsCapturing(hipStream_t s, hipStreamCaptureStatus* st) {
  *st = s == capturing ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
  return s ? hipSuccess : hipErrorStreamCaptureImplicit;
}
}
static char* at(int i) { return (char*)((uintptr_t)(i + 1) << 40); }
static int call(int which, hipStream_t s) {
  const ts_cache c{at(0), at(1), (uint8_t*)at(2), (uint8_t*)at(3), (float*)at(4), 100, 2, 128};
  auto n = [](int i) { return (int32_t*)at(i); };
  switch (which) {
    case 0: return ts_cache_append(&c, at(5), at(6), n(7), n(8), n(9), n(10), 2, 20, 300, 600, s);
    case 1: return ts_cache_attn(&c, at(5), at(6), nullptr, n(7), n(8), n(9), 2, 20, 300, 1000, 600, 2, 0.1f, 0, nullptr, 0, s);
    case 2: return ts_cache_weigh(&c, at(5), (float*)at(6), n(7), n(8), n(9), (float*)at(10), 2, 20, 300, 1000, 600, 2, 0.1f, s);
    default: return ts_cache_evict(&c, n(5), n(6), n(7), n(8), n(9), 2, 20, 20, 1000, 300, 10, 10, s);
  }
}
int main() {
  int bad = 0;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); ++bad; } } while (0)
  const int64_t need = ts_cache_attn_workspace(1, 300, 20000, 300, 2, 2, 128, 0);
  CHECK(need > 0 && ts_cache_attn_workspace(2, 10, 200, 20, 2, 4, 64, 3) > 0);
  CHECK(configured == 0);
  for (int i = 0; i < 4; ++i) CHECK(call(i, capturing) == TS_ERR_CAPTURE);
  CHECK(configured == 0 && launches == 0);
  for (int i = 0; i < 4; ++i) CHECK(call(i, eager) == TS_OK);
  CHECK(configured == 1 && launches == 4);
  for (int i = 0; i < 4; ++i) CHECK(call(i, capturing) == TS_OK);
  CHECK(configured == 1 && launches == 8);
  CHECK(ts_cache_attn_workspace(1, 300, 20000, 300, 2, 2, 128, 0) == need);
  printf("failures %d\n", bad);
  return bad != 0;
}
"""


def test_a_device_s_first_call_under_capture_is_refused(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    src, exe = tmp_path / "driver.cpp", str(tmp_path / "driver")
    src.write_text(DRIVER)
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-Wall", "-Wextra", "-Werror", "-Wno-missing-field-initializers", "-D__HIP_PLATFORM_AMD__",
           "-I" + os.path.join(ROCM, "include"), "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, str(src),
           os.path.join(CSRC, "ts_cache.cpp"), os.path.join(CSRC, "cache_plan.cpp"), "-o", exe, "-pthread"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and "failures 0" in r.stdout, r.stdout + r.stderr
