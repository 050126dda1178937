"""The host side of the session cache (csrc/ts_cache.cpp, csrc/cache_plan.cpp) under AddressSanitizer and UBSan, compiled
with g++ together with a driver: every entry point over random and extreme sizes, scales and pointers (device set-up
fails, so nothing is launched), and the division of attention calls over random sessions."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_19271_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")

DRIVER = r"""
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include "cache_launch.h"
#include "ts_cache.h"
using namespace tscache;
namespace tscache {  // in place of the kernels
hipError_t configure_kernels() { return hipErrorUnknown; }
hipError_t launch_attn(const AttnArgs&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_weigh(const WeighArgs&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_append(const AppendArgs&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_evict(const EvictArgs&, hipStream_t) { return hipErrorUnknown; }
}
static int bad = 0;
#define CHECK(x) do { if (!(x)) { if (bad < 20) printf("line %d: %s\n", __LINE__, #x); ++bad; } } while (0)
static uint64_t state = 99;
static int64_t rnd(int64_t n) { state = state * 6364136223846793005ull + 1442695040888963407ull; return (int64_t)(state >> 33) % n; }
static int32_t size() {
  const int32_t edge[] = {INT_MIN, -1, 0, 1, 2, 16, 17, 33, 63, 64, 65, 255, 256, 257, 32760, 65536, 1 << 23, 1 << 27, 1 << 30, INT_MAX};
  return rnd(2) ? (int32_t)rnd(5000) : edge[rnd(20)];
}
static void* ptr(int i) {  // far apart, now and then null, odd or somebody else's
  if (rnd(40) == 0) return nullptr;
  if (rnd(60) == 0) i = (int)rnd(14);
  return (void*)(((uintptr_t)(i + 1) << 44) + (rnd(60) ? 0 : 4));
}
int main() {
  const float scales[] = {0.0f, 0.1f, -2.0f, NAN, INFINITY, -INFINITY};
  for (int i = 0; i < 400000; ++i) {
    const int32_t d[] = {-1, 0, 63, 64, 128, 128, 64, 256};
    const ts_cache c{ptr(0), ptr(1), (uint8_t*)ptr(2), (uint8_t*)ptr(3), (float*)ptr(4), size(), rnd(3) ? 1 + (int32_t)rnd(50) : size(), d[rnd(8)]};
    const int32_t Hq = rnd(3) ? (int32_t)((int64_t)(c.H & 1023) * (1 + rnd(8))) : size(), n = rnd(2) ? 0 : (int32_t)rnd(70) - 2;
    const int64_t work = rnd(3) ? rnd((int64_t)1 << 31) << rnd(20) : -rnd(2);
    const float sc = scales[rnd(4) ? 1 : rnd(6)];
    auto* t = [](void* p) { return (int32_t*)p; }(ptr(5));
    auto *lens = (int32_t*)ptr(6), *cu = (int32_t*)ptr(7);
    const int32_t nseq = size(), width = size(), rows = size(), len = size(), total = size(), keep = size(), first = size(), last = size();
    const ts_cache* cp = rnd(100) ? &c : nullptr;
    const int got[] = {
        ts_cache_append(cp, ptr(8), ptr(9), cu, t, lens, (int32_t*)ptr(10), nseq, width, rows, total, nullptr),
        ts_cache_attn(cp, ptr(8), ptr(9), (float*)ptr(10), cu, t, lens, nseq, width, rows, len, total, Hq, sc, n, ptr(11), work, nullptr),
        ts_cache_weigh(cp, ptr(8), (float*)ptr(9), cu, t, lens, (float*)ptr(10), nseq, width, rows, len, total, Hq, sc, nullptr),
        ts_cache_evict(cp, t, lens, (int32_t*)ptr(8), (int32_t*)ptr(9), (int32_t*)ptr(10), nseq, width, size(), len, keep, first, last, nullptr)};
    for (int s : got) CHECK(s >= TS_OK && s <= TS_ERR_SCRATCH);
    CHECK(ts_cache_attn_workspace(nseq, rows, len, total, c.H, Hq, c.d, n) >= 0);
  }
  // divided calls: the workspace is what the launch uses, more of it never divides less, and shares fit their slots
  for (int i = 0; i < 200000; ++i) {
    const int32_t H = 1 + (int32_t)rnd(64), G = 1 + (int32_t)rnd(8), d = rnd(2) ? 64 : 128, cus = rnd(4) ? 256 : 1 + (int32_t)rnd(400);
    const int32_t rows = 1 + (int32_t)rnd(rnd(2) ? 40 : 5000), nseq = 1 + (int32_t)rnd(rnd(2) ? 3 : 200), forced = rnd(2) ? 0 : 1 + (int32_t)rnd(64);
    const Sessions ss{nullptr, nullptr, nullptr, nseq, 1 << 16, rows, (int32_t)rnd(100000), 1 + (int32_t)rnd((int64_t)rows * nseq)};
    const int tile = row_tile((int64_t)rows * G, rnd(9) ? 0.1f : 0.0f);
    const Parts most = attn_parts(ss, H, G, d, tile, forced, INT64_MAX, cus);
    CHECK(most.bytes == 0 || most.n_split > 1 || most.shares > 1);
    CHECK(most.o_offset % 256 == 0 && most.n_split >= 1 && most.n_split <= TS_CACHE_MAX_SPLITS);
    CHECK(most.shares == 0 || (tile == kTileRows && forced == 0 && most.n_split == 1 && most.shares <= cus &&
                               most.bytes == most.o_offset + 2ll * most.shares * kTileRows * d * 4));
    if (forced > 0) { CHECK(most.n_split == forced); continue; }
    const Parts same = attn_parts(ss, H, G, d, tile, 0, most.bytes, cus);
    CHECK(same.n_split == most.n_split && same.shares == most.shares && same.bytes == most.bytes);
    const Parts less = attn_parts(ss, H, G, d, tile, 0, rnd(most.bytes + 1), cus);
    CHECK(less.bytes <= most.bytes && less.n_split >= 1);
    CHECK(attn_parts(ss, H, G, d, tile, 0, 0, cus).bytes == 0);
  }
  printf("failures %d\n", bad);
  return bad != 0;
}
"""


def test_the_cache_s_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    src, exe = tmp_path / "driver.cpp", str(tmp_path / "driver")
    src.write_text(DRIVER)
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", "-Wall", "-Wextra", "-Werror", "-Wno-missing-field-initializers", "-D__HIP_PLATFORM_AMD__",
           "-I" + os.path.join(ROCM, "include"), "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, str(src),
           os.path.join(CSRC, "ts_cache.cpp"), os.path.join(CSRC, "cache_plan.cpp"), "-o", exe,
           "-L" + os.path.join(ROCM, "lib"), "-lamdhip64", "-Wl,-rpath," + os.path.join(ROCM, "lib")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "failures 0" in r.stdout
