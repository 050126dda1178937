"""The transformer block's C ABI and binding without a GPU: exports, the header, and every refusal, which the host makes before any
HIP call (fake pointers are never dereferenced); the host code under sanitizers and against a stand-in for HIP."""
import ctypes
import math
import os
import re
import shutil
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "ts_block.h")
CSRC = os.path.join(ROOT, "paper_2606_19271_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")

ts = pytest.importorskip("paper_2606_19271_amd")
from paper_2606_19271_amd import _lib  # noqa: E402
from paper_2606_19271_amd import block as B  # noqa: E402
from paper_2606_19271_amd.build import BLOCK_LIB  # noqa: E402

P = ctypes.c_void_p
TOP = (1 << 31) - 1
AT = {n: (i + 1) << 36 for i, n in enumerate(("q", "k", "v", "o", "do", "lse", "dq", "dk", "dv", "cu_q", "cu_k", "work", "q_out", "k_out",
                                             "wq", "wk", "gwq", "gwk", "pos", "freq"))}
# without a GPU a call that passes every check ends at the device
PASSES = (_lib.TS_ERR_UNSUPPORTED, _lib.TS_ERR_HIP)
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="would launch on fake pointers")


class Rows(ctypes.Structure):
    _fields_ = [("p", P), ("stride", ctypes.c_int64), ("heads", ctypes.c_int32)]


class RopeStruct(ctypes.Structure):
    _fields_ = [("pos", P), ("freq", P), ("axes", ctypes.c_int32 * 3), ("interleaved", ctypes.c_int32)]


@pytest.fixture(scope="module")
def lib():
    return B.load_block()


def refused(rc, name):
    assert rc == getattr(_lib, name), (rc, name)


def ref(x):
    return None if x is None else ctypes.addressof(x)


def a_rope(pos=AT["pos"], freq=AT["freq"], axes=(12, 10, 10), interleaved=1):
    return RopeStruct(pos, freq, (ctypes.c_int32 * 3)(*axes), interleaved)


def rope(lib, q=AT["q"], k=AT["k"], q_out=AT["q_out"], k_out=AT["k_out"], Hq=4, Hk=2, qs=None, ks=None, qos=None, kos=None, wq=AT["wq"],
         wk=AT["wk"], r="default", T=10, d=64, eps=1e-6, has_k=True, has_k_out=True, Hqo=None, Hko=None):
    r = a_rope() if r == "default" else r
    rows = [Rows(q, Hq * d if qs is None else qs, Hq), Rows(k, Hk * d if ks is None else ks, Hk),
            Rows(q_out, Hq * d if qos is None else qos, Hq if Hqo is None else Hqo), Rows(k_out, Hk * d if kos is None else kos, Hk if Hko is None else Hko)]
    return lib.ts_qk_rope(ref(rows[0]), ref(rows[1]) if has_k else None, ref(rows[2]), ref(rows[3]) if has_k_out else None, P(wq), P(wk),
                          ref(r), T, d, eps, None)


def rope_bwd(lib, go=AT["q_out"], ho=AT["k_out"], q=AT["q"], k=AT["k"], dq=AT["dq"], dk=AT["dk"], Hq=4, Hk=2, wq=AT["wq"], wk=AT["wk"], gwq=AT["gwq"],
             gwk=AT["gwk"], r="default", T=10, d=64, eps=1e-6, work=AT["work"], bytes=1 << 22, has_q=True, has_k=True):
    r = a_rope() if r == "default" else r
    rows = [Rows(p, h * d, h) for p, h in ((go, Hq), (ho, Hk), (q, Hq), (k, Hk), (dq, Hq), (dk, Hk))]
    return lib.ts_qk_rope_bwd(ref(rows[0]), ref(rows[1]), ref(rows[2]) if has_q else None, ref(rows[3]) if has_k else None, ref(rows[4]),
                              ref(rows[5]), P(wq), P(wk), P(gwq), P(gwk), ref(r), T, d, eps, P(work), bytes, None)


def bwd(lib, do=AT["do"], q=AT["q"], k=AT["k"], v=AT["v"], o=AT["o"], lse=AT["lse"], dq=AT["dq"], dk=AT["dk"], dv=AT["dv"], cu_q=AT["cu_q"],
        cu_k=AT["cu_k"], nseq=2, max_q=100, max_k=300, Tq=150, Tk=400, H=4, d=64, scale=0.1, n=0, work=AT["work"], bytes=1 << 30):
    return lib.ts_attn_bwd(*[P(x) for x in (do, q, k, v, o, lse, dq, dk, dv, cu_q, cu_k)], nseq, max_q, max_k, Tq, Tk, H, d, scale, n,
                           P(work), bytes, None)


def test_exports_and_version(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(ts_\w+)\s*\(", text)))
    assert names == ["ts_attn_bwd", "ts_attn_bwd_workspace", "ts_block_abi_version", "ts_qk_rope", "ts_qk_rope_bwd",
                     "ts_qk_rope_bwd_workspace"]
    out = subprocess.run(["nm", "-D", "--defined-only", BLOCK_LIB], capture_output=True, text=True, check=True).stdout
    assert sorted(re.findall(r"^[0-9a-fA-F]+ [A-Za-z] (\S+)$", out, flags=re.M)) == names
    assert lib.ts_block_abi_version() == int(re.search(r"#define\s+TS_BLOCK_ABI_VERSION\s+(\d+)", open(HEADER).read()).group(1))


def test_header_compiles_as_c_and_cxx(tmp_path):
    src = tmp_path / "use.c"
    src.write_text('#include "ts_block.h"\nint main(void){ts_rows r; ts_rope p; r.heads = 1; p.interleaved = r.heads; return p.interleaved;}\n')
    inc = "-I" + os.path.dirname(HEADER)
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-fsyntax-only", inc, str(src)], check=True)
    subprocess.run(["g++", "-std=c++11", "-Wall", "-Werror", "-fsyntax-only", "-x", "c++", inc, str(src)], check=True)


def test_the_binding_s_words_are_the_header_s_structs(tmp_path):
    src = tmp_path / "use.c"
    src.write_text("""#include <stddef.h>
#include "ts_block.h"
_Static_assert(sizeof(ts_rows) == 24 && offsetof(ts_rows, stride) == 8 && offsetof(ts_rows, heads) == 16, "rows");
_Static_assert(sizeof(ts_rope) == 32 && offsetof(ts_rope, freq) == 8 && offsetof(ts_rope, axes) == 16 && offsetof(ts_rope, interleaved) == 28, "rope");
int main(void) { return 0; }
""")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-fsyntax-only", "-I" + os.path.dirname(HEADER), str(src)], check=True)


@no_gpu
def test_good_arguments_reach_the_device(lib):
    for call in (rope, rope_bwd, bwd):
        assert call(lib) in PASSES
    assert rope(lib, has_k=False, has_k_out=False) in PASSES
    assert rope(lib, wq=0, wk=0, r=None) in PASSES
    # in place, and beside each other in fused rows
    assert rope(lib, q_out=AT["q"], k_out=AT["k"]) in PASSES
    row = (4 + 2 + 2) * 64
    fused = dict(qs=row, ks=row, k=AT["q"] + 4 * 64 * 2)
    assert rope(lib, **fused) in PASSES
    assert rope(lib, **fused, qos=row, kos=row, q_out=AT["q"], k_out=AT["q"] + 4 * 64 * 2) in PASSES
    assert rope_bwd(lib, dq=AT["q_out"], dk=AT["k_out"]) in PASSES
    assert rope_bwd(lib, dq=AT["q"], dk=AT["k"]) in PASSES
    assert rope_bwd(lib, wq=0, gwq=0, has_q=False) in PASSES
    assert rope_bwd(lib, wq=0, gwq=0, wk=0, gwk=0, has_q=False, has_k=False, work=0, bytes=0) in PASSES
    for scale in (0.0, -0.1, 2.0 ** -100, -2.0 ** 100):
        assert bwd(lib, scale=scale) in PASSES
    assert bwd(lib, Tq=0, do=0, q=0, o=0, lse=0, dq=0) in PASSES  # keys without queries have gradients of 0
    assert bwd(lib, Tk=0, k=0, v=0, dk=0, dv=0) in PASSES
    assert bwd(lib, k=AT["q"], v=AT["q"], o=AT["do"]) in PASSES  # inputs may be one another
    assert lib.ts_attn_bwd_workspace(2, 100, 300, 150, 400, 4, 64, 0) == 0  # the library's choice needs the device


@pytest.mark.parametrize("call", [rope, rope_bwd])
def test_rope_sizes_and_values(lib, call):
    for d in (0, 32, 96, 256, -64):
        refused(call(lib, d=d, r=None), "TS_ERR_HEAD_DIM")
    for bad in ({"T": -1}, {"T": TOP}, {"T": TOP // 6}, {"Hq": 0}, {"Hk": -1}, {"Hq": 1 << 24}):
        refused(call(lib, **bad), "TS_ERR_SHAPE")
    for eps in (0.0, -1e-6, 1e-39, math.nan, math.inf):
        refused(call(lib, eps=eps), "TS_ERR_SCALE")
    for axes in ((12, 10, 9), (12, 10, 11), (-1, 23, 10), (TOP, TOP, 34), (0, 0, 0)):
        refused(call(lib, r=a_rope(axes=axes)), "TS_ERR_SHAPE")
    refused(call(lib, r=a_rope(pos=0)), "TS_ERR_NULL")
    refused(call(lib, r=a_rope(freq=0)), "TS_ERR_NULL")
    refused(call(lib, r=a_rope(pos=AT["pos"] + 2)), "TS_ERR_ALIGN")
    refused(call(lib, r=a_rope(freq=AT["freq"] + 4)), "TS_ERR_ALIGN")
    refused(call(lib, wq=AT["wq"] + 2), "TS_ERR_ALIGN")
    refused(call(lib, q=0), "TS_ERR_NULL")
    refused(call(lib, k=AT["k"] + 8), "TS_ERR_ALIGN")


def test_rope_checks(lib):
    for bad in ({"has_k": False}, {"has_k_out": False}, {"q_out": 0}, {"k_out": 0}, {"k": 0}):
        refused(rope(lib, **bad), "TS_ERR_NULL")
    assert lib.ts_qk_rope(None, None, None, None, None, None, None, 1, 64, 1e-6, None) == _lib.TS_ERR_NULL
    for bad in ({"qs": 255}, {"ks": 120}, {"qos": 1 << 30}, {"Hqo": 3}, {"Hko": 4}):
        refused(rope(lib, **bad), "TS_ERR_SHAPE")
    for bad in ({"qs": 260}, {"kos": 132}, {"q_out": AT["q_out"] + 8}):
        refused(rope(lib, **bad), "TS_ERR_ALIGN")
    for bad in ({"q_out": AT["q"] + 64}, {"q_out": AT["k"]}, {"k_out": AT["q"]}, {"k_out": AT["q_out"] + 1024}, {"q_out": AT["wq"]},
                {"k_out": AT["pos"]}, {"q_out": AT["freq"]}, {"q_out": AT["q"], "qos": 320}, {"q_out": AT["q"], "qs": 320}):
        refused(rope(lib, **bad), "TS_ERR_ALIAS")
    row = 8 * 64  # fused rows whose parts meet
    refused(rope(lib, qs=row, ks=row, k=AT["q"] + 4 * 64 * 2, q_out=AT["q"] + 64 * 2, qos=row), "TS_ERR_ALIAS")
    refused(rope(lib, qos=row, kos=row, k_out=AT["q_out"] + 3 * 64 * 2), "TS_ERR_ALIAS")
    refused(rope(lib, qos=row, kos=row, k_out=AT["q_out"] + 7 * 64 * 2), "TS_ERR_ALIAS")  # runs into the next row
    refused(rope(lib, qos=row, kos=row, k_out=AT["q_out"] - 64 * 2), "TS_ERR_ALIAS")
    # nothing to do
    assert rope(lib, T=0, q=0, k=0, q_out=0, k_out=0, r=a_rope(pos=0)) == _lib.TS_OK


def test_rope_bwd_checks(lib):
    for bad in ({"gwq": 0}, {"gwk": 0}, {"wq": 0}, {"wk": 0}, {"has_q": False}, {"has_k": False}, {"dq": 0}, {"go": 0}):
        refused(rope_bwd(lib, **bad), "TS_ERR_NULL")
    need = lib.ts_qk_rope_bwd_workspace(10, 4, 2, 64)
    assert need > 0 and need % (2 * 64 * 4) == 0
    for bad in ({"work": 0}, {"bytes": need - 1}, {"bytes": 0}):
        refused(rope_bwd(lib, **bad), "TS_ERR_SCRATCH")
    refused(rope_bwd(lib, bytes=-1), "TS_ERR_SHAPE")
    refused(rope_bwd(lib, work=AT["work"] + 64), "TS_ERR_ALIGN")
    for bad in ({"dq": AT["k"]}, {"dk": AT["q_out"]}, {"dq": AT["q"] + 16}, {"gwq": AT["wq"]}, {"gwq": AT["gwk"]}, {"work": AT["q"]}, {"work": AT["dq"]},
                {"dk": AT["dq"]}):
        refused(rope_bwd(lib, **bad), "TS_ERR_ALIAS")
    for bad in ((-1, 4, 2, 64), (10, 0, 2, 64), (10, 4, -1, 64), (10, 4, 2, 96), (TOP, 4, 2, 64)):
        assert lib.ts_qk_rope_bwd_workspace(*bad) == 0
    assert lib.ts_qk_rope_bwd_workspace(1 << 20, 40, 40, 128) == lib.ts_qk_rope_bwd_workspace(1 << 24, 40, 40, 128)  # bounded
    assert rope_bwd(lib, T=0, wq=0, gwq=0, wk=0, gwk=0, go=0, ho=0, q=0, k=0, dq=0, dk=0, r=None) == _lib.TS_OK


def test_attn_bwd_checks(lib):
    for t in ("do", "q", "k", "v", "o", "lse", "dq", "dk", "dv", "cu_q", "cu_k"):
        refused(bwd(lib, **{t: 0}), "TS_ERR_NULL")
    for t in ("do", "q", "k", "v", "o", "dq", "dk", "dv"):
        refused(bwd(lib, **{t: AT[t] + 8}), "TS_ERR_ALIGN")
    for t in ("lse", "cu_q", "cu_k"):
        refused(bwd(lib, **{t: AT[t] + 2}), "TS_ERR_ALIGN")
    refused(bwd(lib, work=AT["work"] + 128), "TS_ERR_ALIGN")
    for d in (0, 32, 96, 256, -64):
        refused(bwd(lib, d=d), "TS_ERR_HEAD_DIM")
    for bad in ({"nseq": -1}, {"max_q": -1}, {"max_k": -1}, {"Tq": -1}, {"Tk": -1}, {"H": 0}, {"H": -1}, {"H": TOP}, {"n": -1}, {"n": 17}, {"bytes": -1},
                {"max_q": TOP}, {"max_k": (1 << 31) // (4 * 64 * 2)}, {"H": 1 << 20, "max_k": 3000}, {"nseq": TOP}, {"nseq": 1 << 20, "max_k": 200000},
                {"Tq": 1 << 25, "max_q": 100}, {"nseq": 1 << 18}):
        refused(bwd(lib, **bad), "TS_ERR_SHAPE")
    for s in (math.nan, math.inf, -math.inf, 2.0 ** -101, -2.0 ** -120, 2.0 ** 101):
        refused(bwd(lib, scale=s), "TS_ERR_SCALE")
    for bad in ({"dq": AT["q"]}, {"dk": AT["k"]}, {"dv": AT["dk"]}, {"dq": AT["dv"] + 16}, {"dq": AT["do"]}, {"dk": AT["lse"]}, {"dv": AT["cu_k"]},
                {"work": AT["q"]}, {"work": AT["dq"]}, {"work": AT["cu_q"]}):
        refused(bwd(lib, **bad), "TS_ERR_ALIAS")
    # the plan, two statistics, and with three ranges the parts
    tiles = min(2, 150 // 128 + 2) + min(2 * 3, 400 // 128 + 2)
    plan = lambda n: (32 + 32 * n * tiles + 255) // 256 * 256  # noqa: E731
    least = plan(1) + (2 * 150 * 4 * 4 + 255) // 256 * 256
    assert lib.ts_attn_bwd_workspace(2, 100, 300, 150, 400, 4, 64, 1) == least
    three = plan(3) + (2 * 150 * 4 * 4 + 255) // 256 * 256 + 3 * 150 * 4 * 64 * 4 + 2 * 3 * 400 * 4 * 64 * 4
    assert lib.ts_attn_bwd_workspace(2, 100, 300, 150, 400, 4, 64, 3) == three
    for n, need in ((0, least), (1, least), (3, three)):
        refused(bwd(lib, n=n, bytes=need - 1), "TS_ERR_SCRATCH")
        refused(bwd(lib, n=n, work=0), "TS_ERR_SCRATCH")
    for bad in ((0, 100, 300, 150, 400, 4, 64, 3), (2, 100, 300, 150, 400, 4, 65, 3), (2, 100, 300, 150, 400, 4, 64, 17), (2, TOP, 300, 150, 400, 4, 64, 3),
                (2, 100, 300, -1, 400, 4, 64, 3)):
        assert lib.ts_attn_bwd_workspace(*bad) == 0
    # nothing to do
    assert bwd(lib, nseq=0) == _lib.TS_OK and bwd(lib, Tq=0, Tk=0, work=0) == _lib.TS_OK


def test_binding_refuses_what_does_not_fit():
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    ints = torch.zeros(2, dtype=torch.int32)
    for f in (lambda: ts.ts_qk_rope(x, x), lambda: ts.ts_qk_rope_bwd(x, x, x, x),
              lambda: ts.ts_attn_bwd(x, x, x, x, x, torch.zeros(4, 2), ints, ints, 4, 4)):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: ts.ts_qk_rope(None, x), lambda: ts.ts_qk_rope_bwd(None, x, x, x), lambda: ts.ts_attn_bwd(x, None, x, x, x, x, ints, ints, 4, 4)):
        with pytest.raises(TypeError):
            f()
    r = ts.rope((2, 1, 0), theta=100.0, interleaved=False, device="cpu")
    assert r.freq.tolist() == [1.0, 100.0 ** -0.5, 1.0] and r.freq.dtype == torch.float64 and r.axes == (2, 1, 0) and r.interleaved is False


STUBS = r"""
#include <hip/hip_runtime_api.h>
#include <limits.h>
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>
#include "block_launch.h"
#include "ts_block.h"
using namespace tsblock;
static int configured = 0, launches = 0, bad = 0;
#define CHECK(x) do { if (!(x)) { if (bad < 20) printf("line %d: %s\n", __LINE__, #x); ++bad; } } while (0)
"""

CAPTURE = STUBS + r"""
static const hipStream_t recording = (hipStream_t)16, eager = (hipStream_t)32;
namespace tsblock {  // in place of the kernels
hipError_t configure_kernels() { ++configured; return hipSuccess; }
hipError_t launch_rope(const RopeArgs&, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_rope_bwd(const RopeBwdArgs&, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_attn_bwd(const BwdArgs&, hipStream_t) { ++launches; return hipSuccess; }
}
extern "C" {  // in place of HIP: one device, one stream being captured
hipError_t hipGetDevice(int* d) { *d = 0; return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipGetDeviceProperties(hipDeviceProp_t* p, int) {
  memset(p, 0, sizeof(*p));
  strcpy(p->gcnArchName, "gfx950:sramecc+");
  p->multiProcessorCount = 256;
  return hipSuccess;
}
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) { *v = 256; return hipSuccess; }
hipError_t hipMemcpyAsync(void* to, const void* from, size_t n, hipMemcpyKind, hipStream_t) { memcpy(to, from, n); return hipSuccess; }
hipError_t hipStreamSynchronize(hipStream_t) { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t s, hipStreamCaptureStatus* st) {
  *st = s == recording ? hipStreamCaptureStatusActive : hipStreamCaptureStatusNone;
  return s ? hipSuccess : hipErrorStreamCaptureImplicit;
}
}
static char* at(int i) { return (char*)((uintptr_t)(i + 1) << 40); }
static int32_t cu_q[3] = {0, 100, 150}, cu_k[3] = {0, 0, 400};
static int call(int which, hipStream_t s) {
  const ts_rows q{at(0), 512, 4}, k{at(1), 512, 4}, o{at(2), 512, 4}, p{at(3), 512, 4}, r{at(4), 512, 4}, t{at(5), 512, 4};
  float *w = (float*)at(6), *gw = (float*)at(7), *gw2 = (float*)at(8);
  switch (which) {
    case 0: return ts_qk_rope(&q, &k, &o, &p, w, w, nullptr, 100, 128, 1e-6f, s);
    case 1: return ts_qk_rope_bwd(&q, &k, &o, &p, &r, &t, w, w, gw, gw2, nullptr, 100, 128, 1e-6f, at(9), 1 << 22, s);
    default: return ts_attn_bwd(at(0), at(1), at(2), at(3), at(4), w, at(10), at(11), at(12), cu_q, cu_k, 2, 100, 400, 150, 400, 4, 64, 0.1f, 0,
                                at(13), 1 << 28, s);
  }
}
int main() {
  const int64_t need = ts_attn_bwd_workspace(1, 1000, 1000, 1000, 1000, 2, 64, 0);
  CHECK(need > 0 && configured == 0);
  for (int i = 0; i < 3; ++i) CHECK(call(i, recording) == TS_ERR_CAPTURE);
  CHECK(configured == 0 && launches == 0);
  for (int i = 0; i < 3; ++i) CHECK(call(i, eager) == TS_OK);
  CHECK(configured == 1 && launches == 3);
  for (int i = 0; i < 3; ++i) CHECK(call(i, recording) == TS_OK);
  CHECK(configured == 1 && launches == 6);
  CHECK(ts_attn_bwd_workspace(1, 1000, 1000, 1000, 1000, 2, 64, 0) == need);
  // validation mode: what breaks the offsets' rules is refused, but not on a capturing stream
  setenv("TS_ATTN_VALIDATE", "1", 1);
  CHECK(call(2, eager) == TS_OK);
  const int32_t wrong[][6] = {{1, 100, 150, 0, 0, 400}, {0, 101, 150, 0, 0, 400}, {0, 100, 149, 0, 0, 400}, {0, -1, 150, 0, 0, 400},
                              {0, 100, 150, 0, 10, 400 - 1}, {0, 100, 150, 0, 500, 400}, {0, 100, 99, 0, 0, 400}, {0, INT_MIN, INT_MAX, 0, 0, 400}};
  for (const auto& x : wrong) {
    memcpy(cu_q, x, 12);
    memcpy(cu_k, x + 3, 12);
    const int before = launches;
    CHECK(call(2, eager) == TS_ERR_SEGMENTS && launches == before);
    CHECK(call(2, recording) == TS_OK && launches == before + 1);
  }
  printf("failures %d\n", bad);
  return bad != 0;
}
"""

SANITIZED = STUBS + r"""
namespace tsblock {
hipError_t configure_kernels() { return hipErrorUnknown; }
hipError_t launch_rope(const RopeArgs&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_rope_bwd(const RopeBwdArgs&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_attn_bwd(const BwdArgs&, hipStream_t) { return hipErrorUnknown; }
}
static uint64_t state = 99;
static int64_t rnd(int64_t n) { state = state * 6364136223846793005ull + 1442695040888963407ull; return (int64_t)(state >> 33) % n; }
static int32_t size() {
  const int32_t edge[] = {INT_MIN, -1, 0, 1, 2, 16, 17, 63, 64, 65, 127, 128, 129, 255, 256, 32760, 65536, 1 << 19, 1 << 23, 1 << 27, 1 << 30, INT_MAX};
  return rnd(2) ? (int32_t)rnd(5000) : edge[rnd(22)];
}
static void* ptr(int i) {  // far apart, now and then null, odd or somebody else's
  if (rnd(40) == 0) return nullptr;
  if (rnd(60) == 0) i = (int)rnd(14);
  return (void*)(((uintptr_t)(i + 1) << 44) + (rnd(60) ? 0 : 4));
}
static ts_rows rows(int i, int32_t heads, int32_t d) {
  return {ptr(i), rnd(4) ? (int64_t)heads * d + 8 * rnd(20) : rnd(8) ? (int64_t)size() : INT64_MAX - rnd(9), rnd(30) ? heads : size()};
}
int main() {
  const float values[] = {0.0f, 0.1f, -2.0f, NAN, INFINITY, -INFINITY, 1e-40f, 1e-35f, 1e35f};
  for (int i = 0; i < 300000; ++i) {
    const int32_t ds[] = {-1, 0, 63, 64, 128, 128, 64, 256}, d = ds[rnd(8)], T = size();
    const int32_t Hq = rnd(4) ? 1 + (int32_t)rnd(50) : size(), Hk = rnd(4) ? 1 + (int32_t)rnd(50) : size();
    ts_rows r[6];
    for (int j = 0; j < 6; ++j) r[j] = rows(j, j & 1 ? Hk : Hq, d);
    const int32_t n0 = rnd(8) ? (int32_t)rnd(33) : size(), n1 = rnd(8) ? (int32_t)rnd(33) : size();
    const ts_rope rope{(const int32_t*)ptr(6), (const double*)ptr(7), {n0, n1, rnd(8) ? (int32_t)((int64_t)d / 2 - n0 - n1) : size()}, (int32_t)rnd(2)};
    const ts_rope* rp = rnd(4) ? &rope : nullptr;
    const float eps = rnd(4) ? 1e-6f : values[rnd(9)], scale = rnd(4) ? 0.1f : values[rnd(9)];
    auto some = [&](int j) { return rnd(30) ? &r[j] : nullptr; };
    float *wq = (float*)(rnd(3) ? ptr(8) : nullptr), *wk = (float*)(rnd(3) ? ptr(9) : nullptr);
    float *gq = (float*)(wq ? ptr(10) : nullptr), *gk = (float*)(wk ? ptr(11) : nullptr);
    const int64_t work = rnd(3) ? rnd((int64_t)1 << 31) << rnd(20) : -rnd(2);
    const int32_t nseq = size(), max_q = size(), max_k = size(), Tq = size(), Tk = size(), H = rnd(3) ? 1 + (int32_t)rnd(50) : size();
    const int32_t n = rnd(2) ? 0 : (int32_t)rnd(20) - 2;
    const int got[] = {ts_qk_rope(some(0), some(1), some(2), some(3), wq, wk, rp, T, d, eps, nullptr),
                       ts_qk_rope_bwd(some(0), some(1), some(2), some(3), some(4), some(5), wq, wk, gq, gk, rp, T, d, eps, ptr(12), work, nullptr),
                       ts_attn_bwd(ptr(0), ptr(1), ptr(2), ptr(3), ptr(4), (float*)ptr(5), ptr(6), ptr(7), ptr(8), (int32_t*)ptr(9), (int32_t*)ptr(10),
                                   nseq, max_q, max_k, Tq, Tk, H, d, scale, n, ptr(11), work, nullptr)};
    for (int s : got) CHECK(s >= TS_OK && s <= TS_ERR_SCRATCH);
    CHECK(ts_attn_bwd_workspace(nseq, max_q, max_k, Tq, Tk, H, d, n) >= 0);
    CHECK(ts_qk_rope_bwd_workspace(T, Hq, Hk, d) >= 0);
  }
  // divisions: what a call needs least always fits what the query says, a smaller workspace divides less, and the launch stays
  // within its grid
  for (int i = 0; i < 200000; ++i) {
    const int32_t H = 1 + (int32_t)rnd(64), d = rnd(2) ? 64 : 128, cus = rnd(4) ? 256 : 1 + (int32_t)rnd(400);
    const int32_t nseq = 1 + (int32_t)rnd(rnd(2) ? 3 : 200), mq = (int32_t)rnd(rnd(2) ? 40 : 40000), mk = (int32_t)rnd(rnd(2) ? 40 : 40000);
    const int32_t Tq = (int32_t)rnd((int64_t)mq * nseq + 1), Tk = (int32_t)rnd((int64_t)mk * nseq + 1), forced = rnd(2) ? 0 : 1 + (int32_t)rnd(16);
    const BwdParts most = bwd_parts(nseq, mq, mk, Tq, Tk, H, d, forced, INT64_MAX, cus);
    const int64_t least = bwd_least_workspace(nseq, mq, mk, Tq, Tk, H, d, forced);
    CHECK(most.bytes >= least && most.n_q >= 1 && most.n_q <= 16 && most.n_k >= 1 && most.n_k <= 16);
    CHECK(most.tile == 128 || (most.tile == 256 && d == 128));
    CHECK(most.stat_offset % 256 == 0 && most.q_offset % 256 == 0 && most.k_offset % 256 == 0);
    const int64_t tiles = bwd_tiles(nseq, mq, Tq, most.tile) * most.n_q + bwd_tiles(nseq, mk, Tk, most.tile) * most.n_k;
    CHECK((int64_t)sizeof(BwdPlan) + tiles * (int64_t)sizeof(BwdTile) <= most.stat_offset);
    if (forced > 0) { CHECK(most.n_q == forced && most.n_k == forced && most.bytes == least); continue; }
    const BwdParts same = bwd_parts(nseq, mq, mk, Tq, Tk, H, d, 0, most.bytes, cus);
    CHECK(same.n_q == most.n_q && same.n_k == most.n_k && same.bytes == most.bytes && same.tile == most.tile);
    const BwdParts less = bwd_parts(nseq, mq, mk, Tq, Tk, H, d, 0, least + rnd(most.bytes - least + 1), cus);
    CHECK(less.bytes <= most.bytes && less.n_q >= 1);
    CHECK(bwd_parts(nseq, mq, mk, Tq, Tk, H, d, 0, least, cus).bytes == least);
  }
  // an upper bound of the tiles, and no more than one too many a segment
  for (int i = 0; i < 20000; ++i) {
    int32_t lens[8], nseq = 1 + (int32_t)rnd(8), most = 0, total = 0, tile = rnd(2) ? 128 : 256;
    int64_t tiles = 0;
    for (int s = 0; s < nseq; ++s) {
      lens[s] = (int32_t)rnd(rnd(2) ? 3 : 1000);
      most = lens[s] > most ? lens[s] : most;
      total += lens[s];
      tiles += (lens[s] + tile - 1) / tile;
    }
    CHECK(bwd_tiles(nseq, most, total, tile) >= tiles && bwd_tiles(nseq, most, total, tile) <= tiles + nseq);
  }
  printf("failures %d\n", bad);
  return bad != 0;
}
"""


def build_and_run(tmp_path, source, *flags):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    src, exe = tmp_path / "driver.cpp", str(tmp_path / "driver")
    src.write_text(source)
    cmd = ["g++", "-std=c++17", "-O1", "-g", *flags, "-Wall", "-Wextra", "-Werror", "-Wno-missing-field-initializers", "-Wno-unused-variable",
           "-D__HIP_PLATFORM_AMD__", "-I" + os.path.join(ROCM, "include"), "-I" + os.path.join(ROOT, "include"), "-I" + CSRC, str(src),
           os.path.join(CSRC, "ts_block.cpp"), os.path.join(CSRC, "block_plan.cpp"), "-o", exe]
    if "-fsanitize=address,undefined" in flags:
        cmd += ["-L" + os.path.join(ROCM, "lib"), "-lamdhip64", "-Wl,-rpath," + os.path.join(ROCM, "lib")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "failures 0" in r.stdout


def test_a_device_s_first_call_under_capture_is_refused(tmp_path):
    build_and_run(tmp_path, CAPTURE.replace("#include <stdio.h>", "#include <stdio.h>\n#include <stdlib.h>"))


def test_the_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    build_and_run(tmp_path, SANITIZED, "-fno-omit-frame-pointer", "-fsanitize=address,undefined", "-fno-sanitize-recover=all")
