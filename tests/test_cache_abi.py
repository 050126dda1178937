"""The session cache's C ABI and binding without a GPU: exports, the header, and every refusal, which the host makes before
any HIP call (fake pointers are never dereferenced)."""
import ctypes
import math
import os
import re
import subprocess

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "ts_cache.h")

ts = pytest.importorskip("paper_2606_19271_amd")
from paper_2606_19271_amd import _lib  # noqa: E402
from paper_2606_19271_amd import cache as C  # noqa: E402

P = ctypes.c_void_p
MB = 1 << 20
# fake device addresses, far enough apart for the sizes below
AT = {n: (i + 1) << 32 for i, n in enumerate(("k", "v", "k_exp", "v_exp", "weight", "x", "y", "o", "lse", "cu", "table", "lens", "new",
                                             "new_table", "kept", "work", "out"))}
TOP = (1 << 31) - 1


@pytest.fixture(scope="module")
def lib():
    return C.load_cache()


def pool(k=AT["k"], v=AT["v"], k_exp=AT["k_exp"], v_exp=AT["v_exp"], weight=AT["weight"], pages=10, H=2, d=64):
    return C._Pool(k, v, k_exp, v_exp, weight, pages, H, d)


def append(lib, c=None, k=AT["x"], v=AT["y"], cu=AT["cu"], table=AT["table"], lens=AT["lens"], new=AT["new"], nseq=2, width=4,
           max_rows=10, total=20, **p):
    c = pool(**p) if c is None else c
    return lib.ts_cache_append(ctypes.byref(c), P(k), P(v), P(cu), P(table), P(lens), P(new), nseq, width, max_rows, total, P(None))


def attn(lib, q=AT["x"], o=AT["o"], lse=AT["lse"], cu=AT["cu"], table=AT["table"], lens=AT["lens"], nseq=2, width=4, max_rows=10,
         max_len=200, total=20, Hq=4, scale=0.1, n=0, work=None, bytes=0, **p):
    return lib.ts_cache_attn(ctypes.byref(pool(**p)), P(q), P(o), P(lse), P(cu), P(table), P(lens), nseq, width, max_rows, max_len, total,
                             Hq, scale, n, P(work), bytes, P(None))


def weigh(lib, q=AT["x"], lse=AT["lse"], cu=AT["cu"], table=AT["table"], lens=AT["lens"], out=AT["out"], nseq=2, width=4, max_rows=10,
          max_len=200, total=20, Hq=4, scale=0.1, **p):
    return lib.ts_cache_weigh(ctypes.byref(pool(**p)), P(q), P(lse), P(cu), P(table), P(lens), P(out), nseq, width, max_rows, max_len,
                              total, Hq, scale, P(None))


def evict(lib, table=AT["table"], lens=AT["lens"], new_table=AT["new_table"], new=AT["new"], kept=AT["kept"], nseq=2, width=4, new_width=2,
          max_len=200, keep=100, first=10, last=20, **p):
    return lib.ts_cache_evict(ctypes.byref(pool(**p)), P(table), P(lens), P(new_table), P(new), P(kept), nseq, width, new_width, max_len,
                              keep, first, last, P(None))


CALLS = {"append": append, "attn": attn, "weigh": weigh, "evict": evict}
# without a GPU a call that passes every check ends at the device
PASSES = (_lib.TS_ERR_UNSUPPORTED, _lib.TS_ERR_HIP)


def refused(rc, name):
    assert rc == getattr(_lib, name), (rc, name)


def test_exports_and_version(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(ts_cache_\w+)\s*\(", text)))
    assert names == ["ts_cache_abi_version", "ts_cache_append", "ts_cache_attn", "ts_cache_attn_workspace", "ts_cache_evict",
                     "ts_cache_weigh"]
    out = subprocess.run(["nm", "-D", "--defined-only", C.CACHE_LIB], capture_output=True, text=True, check=True).stdout
    assert sorted(re.findall(r"^[0-9a-fA-F]+ [A-Za-z] (\S+)$", out, flags=re.M)) == names
    assert lib.ts_cache_abi_version() == int(re.search(r"#define\s+TS_CACHE_ABI_VERSION\s+(\d+)", open(HEADER).read()).group(1))


def test_header_compiles_as_c_and_cxx(tmp_path):
    src = tmp_path / "use.c"
    src.write_text('#include "ts_cache.h"\nint main(void){ts_cache c; c.pages = TS_CACHE_PAGE; return ts_cache_abi_version() - c.pages;}\n')
    inc = "-I" + os.path.dirname(HEADER)
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-fsyntax-only", inc, str(src)], check=True)
    subprocess.run(["g++", "-std=c++11", "-Wall", "-Werror", "-fsyntax-only", "-x", "c++", inc, str(src)], check=True)


@pytest.mark.skipif(torch.cuda.is_available(), reason="would launch on fake pointers")
@pytest.mark.parametrize("name", CALLS)
def test_good_arguments_reach_the_device(lib, name):
    assert CALLS[name](lib) in PASSES
    assert lib.ts_cache_attn_workspace(2, 10, 200, 20, 2, 4, 64, 0) == 0  # the library's choice needs the device


@pytest.mark.parametrize("name", CALLS)
def test_pool_checks(lib, name):
    call = CALLS[name]
    for t in ("k", "v", "k_exp", "v_exp"):
        refused(call(lib, **{t: 0}), "TS_ERR_NULL")
    for bad in ({"pages": 0}, {"pages": -1}, {"H": 0}, {"H": -2}, {"H": TOP}, {"H": 1 << 17}):
        refused(call(lib, **bad), "TS_ERR_SHAPE")
    for d in (0, 32, 96, 256, -64):
        refused(call(lib, d=d), "TS_ERR_HEAD_DIM")
    for t in ("k", "v", "weight"):
        refused(call(lib, **{t: AT[t] + 8}), "TS_ERR_ALIGN")
    assert lib.ts_cache_append(None, *[P(AT["x"])] * 6, 1, 1, 1, 1, P(None)) == _lib.TS_ERR_NULL


@pytest.mark.parametrize("name", CALLS)
def test_size_checks(lib, name):
    call = CALLS[name]
    for bad in ({"nseq": -1}, {"width": -1}, {"width": TOP}, {"width": (1 << 31) // 64 // 64}):
        refused(call(lib, **bad), "TS_ERR_SHAPE")
    if name != "evict":
        for bad in ({"max_rows": -1}, {"total": -1}, {"max_rows": TOP}, {"max_rows": (1 << 31) // (2 * 64 * 2)}):
            refused(call(lib, **bad), "TS_ERR_SHAPE")
    if name != "append":
        for bad in ({"max_len": -1}, {"max_len": 257}, {"max_len": TOP}):
            refused(call(lib, **bad), "TS_ERR_SHAPE")
    # more workgroups than a launch takes
    refused(call(lib, nseq=1 << 24), "TS_ERR_SHAPE")
    refused(call(lib, nseq=TOP), "TS_ERR_SHAPE")
    # no sessions: nothing to do, whatever the pointers
    assert call(lib, nseq=0, table=0, lens=0) == _lib.TS_OK


def test_append_checks(lib):
    for t in ("k", "v"):
        refused(append(lib, c=pool(), **{t: 0}), "TS_ERR_NULL")
        refused(append(lib, c=pool(), **{t: AT["x"] + 2}), "TS_ERR_ALIGN")
    for t in ("cu", "table", "lens", "new"):
        refused(append(lib, **{t: 0}), "TS_ERR_NULL")
    refused(append(lib, new=AT["lens"]), "TS_ERR_ALIAS")
    refused(append(lib, new=AT["lens"] + 4), "TS_ERR_ALIAS")
    refused(append(lib, c=pool(), k=AT["k"] + 64), "TS_ERR_ALIAS")
    refused(append(lib, c=pool(v=AT["k"] + 16)), "TS_ERR_ALIAS")  # the pool's tensors overlap each other
    refused(append(lib, table=AT["weight"]), "TS_ERR_ALIAS")


def test_attn_checks(lib):
    for t in ("q", "o", "cu", "table", "lens"):
        refused(attn(lib, **{t: 0}), "TS_ERR_NULL")
    for t in ("q", "o"):
        refused(attn(lib, **{t: AT["x"] + 8}), "TS_ERR_ALIGN")
    refused(attn(lib, lse=AT["lse"] + 2), "TS_ERR_ALIGN")
    refused(attn(lib, work=AT["work"] + 64, bytes=MB), "TS_ERR_ALIGN")
    for s in (math.nan, math.inf, -math.inf):
        refused(attn(lib, scale=s), "TS_ERR_SCALE")
    for bad in ({"Hq": 0}, {"Hq": 3}, {"Hq": -2}, {"n": -1}, {"n": 65}, {"bytes": -1}, {"Hq": 1 << 23, "H": 1}, {"Hq": TOP, "H": 1}):
        refused(attn(lib, **bad), "TS_ERR_SHAPE")
    for bad in ({"o": AT["x"]}, {"o": AT["k"]}, {"lse": AT["o"] + 4}, {"lse": AT["v_exp"]}, {"work": AT["x"], "bytes": MB},
                {"work": AT["o"], "bytes": MB}, {"o": AT["lens"]}):
        refused(attn(lib, **bad), "TS_ERR_ALIAS")
    # 3 ranges: lse 3 * 20 * 4 floats rounded to 256 bytes, then O
    need = 1024 + 3 * 20 * 4 * 64 * 4
    assert lib.ts_cache_attn_workspace(2, 10, 200, 20, 2, 4, 64, 3) == need
    refused(attn(lib, n=3), "TS_ERR_SCRATCH")
    refused(attn(lib, n=3, work=AT["work"], bytes=need - 1), "TS_ERR_SCRATCH")
    refused(attn(lib, n=3, work=0, bytes=need), "TS_ERR_SCRATCH")
    for bad in ((0, 10, 200, 20, 2, 4, 64, 3), (2, 10, 200, 20, 3, 4, 64, 3), (2, 10, 200, 20, 2, 4, 65, 3), (2, 10, 200, 20, 2, 4, 64, 65),
                (2, TOP, 200, 20, 2, 4, 64, 3), (2, 10, 200, 20, 2, 4, 64, 1)):
        assert lib.ts_cache_attn_workspace(*bad) == 0
    # nothing to do
    assert attn(lib, total=0, q=0, o=0, lse=0) == _lib.TS_OK
    assert attn(lib, max_rows=0, q=0, o=0) == _lib.TS_OK


def test_weigh_checks(lib):
    for t in ("q", "lse", "cu", "table", "lens", "out", "weight"):
        refused(weigh(lib, **{t: 0}), "TS_ERR_NULL")
    refused(weigh(lib, q=AT["x"] + 8), "TS_ERR_ALIGN")
    refused(weigh(lib, lse=AT["lse"] + 1), "TS_ERR_ALIGN")
    refused(weigh(lib, out=AT["out"] + 4), "TS_ERR_ALIGN")
    refused(weigh(lib, scale=math.inf), "TS_ERR_SCALE")
    for bad in ({"Hq": 5}, {"Hq": 0}):
        refused(weigh(lib, **bad), "TS_ERR_SHAPE")
    for bad in ({"out": AT["weight"] + 256}, {"out": AT["k"]}, {"out": AT["lse"]}, {"out": AT["x"]}):
        refused(weigh(lib, **bad), "TS_ERR_ALIAS")
    assert weigh(lib, max_len=0) == _lib.TS_OK


def test_evict_checks(lib):
    for t in ("table", "lens", "new_table", "new", "kept", "weight"):
        refused(evict(lib, **{t: 0}), "TS_ERR_NULL")
    for bad in ({"keep": -1, "first": 0, "last": 0}, {"first": -1}, {"last": -1}, {"first": 50, "last": 51}, {"first": TOP, "last": TOP}, {"keep": 129},
                {"new_width": -1}, {"new_width": TOP}, {"nseq": 1 << 20, "H": 2}):
        refused(evict(lib, **bad), "TS_ERR_SHAPE")
    for bad in ({"new": AT["lens"]}, {"kept": AT["table"]}, {"new_table": AT["k"]}, {"kept": AT["weight"]}):
        refused(evict(lib, **bad), "TS_ERR_ALIAS")


def test_binding_refuses_what_does_not_fit():
    cpu = ts.session_cache(3, 2, 64, device="cpu")
    ints = torch.zeros(1, dtype=torch.int32)
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    for f in (lambda: ts.ts_cache_append(cpu, x, x, ints, 1, ints[None], ints), lambda: ts.ts_cache_attn(x, cpu, ints, 1, ints[None], ints, 1),
              lambda: ts.ts_cache_weigh(x, x, cpu, ints, 1, ints[None], ints, 1),
              lambda: ts.ts_cache_evict(cpu, ints[None], ints, 1, ints[None], 1)):
        with pytest.raises(ValueError):
            f()
    assert cpu.k.dtype == torch.float8_e4m3fn and tuple(cpu.k.shape) == (3, 2, 64, 64) and cpu.weight.shape == (3, 2, 64)
    assert ts.session_cache(1, 1, 128, device="cpu", weight=False).weight is None
