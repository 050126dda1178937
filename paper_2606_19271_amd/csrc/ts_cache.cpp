// ts_cache.cpp -- the C ABI of libts_cache.so (declared in include/ts_cache.h): argument checks, per-device
// set-up, validation mode, and the launches.
#include "ts_cache.h"

#include <hip/hip_runtime_api.h>
#include <math.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <atomic>
#include <memory>
#include <mutex>
#include <new>

#include "cache_launch.h"
#include "device_setup.h"

namespace {

using namespace tshost;

constexpr int64_t kByteLimit = (int64_t)1 << 31;

static_assert(tscache::kPage == TS_CACHE_PAGE, "page size");

struct DeviceState : DeviceSetup {
  std::atomic<int32_t> cus{0};  // compute units, or 0: not asked for yet
};

DeviceState g_dev[kMaxDevices];

void init_device(int dev, DeviceState* st) {
  hipDeviceProp_t p;
  if (hipGetDeviceProperties(&p, dev) != hipSuccess) { (void)hipGetLastError(); st->status = TS_ERR_HIP; return; }
  if (strncmp(p.gcnArchName, "gfx950", 6) != 0) { st->status = TS_ERR_UNSUPPORTED; return; }
  st->cus = p.multiProcessorCount;
  if (tscache::configure_kernels() != hipSuccess) { (void)hipGetLastError(); st->status = TS_ERR_HIP; return; }
  st->status = TS_OK;
}

// Compute units of the calling thread's current device, or 0.  Sets nothing up, so that it can be asked while a stream is
// being captured, the device's first call or not.
int32_t current_cus() {
  const int dev = current_index();
  if (dev < 0) return 0;
  int n = g_dev[dev].cus.load(std::memory_order_relaxed);
  if (n == 0) {
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) {
      (void)hipGetLastError();
      return 0;
    }
    g_dev[dev].cus.store(n, std::memory_order_relaxed);
  }
  return n;
}

DeviceState* current_device(int* status, hipStream_t s) { return tshost::current_device(g_dev, init_device, status, s); }

bool misaligned(const void* p, unsigned to) { return ((uintptr_t)p & (to - 1)) != 0; }

// A byte range of device memory that a call reads or writes.
struct Span {
  const void* p;
  int64_t bytes;
};

bool overlap(const Span& a, const Span& b) {
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  return a.p && b.p && a.bytes > 0 && b.bytes > 0 && x < y + (uintptr_t)b.bytes && y < x + (uintptr_t)a.bytes;
}

// Whether any of the written spans meets another of them or a read one.
template <int W, int R>
bool aliased(const Span (&written)[W], const Span (&read)[R]) {
  for (int i = 0; i < W; ++i) {
    for (int j = i + 1; j < W; ++j)
      if (overlap(written[i], written[j])) return true;
    for (int j = 0; j < R; ++j)
      if (overlap(written[i], read[j])) return true;
  }
  return false;
}

// Bytes of the pool's k (and v), and of its weights and exponents; the checks keep them below 2^63.
int64_t pool_bytes(const ts_cache* c) { return (int64_t)c->pages * c->H * TS_CACHE_PAGE * c->d; }
int64_t weight_bytes(const ts_cache* c) { return (int64_t)c->pages * c->H * TS_CACHE_PAGE * 4; }
int64_t exp_bytes(const ts_cache* c) { return (int64_t)c->pages * c->H; }

int check_pool(const ts_cache* c) {
  if (!c || !c->k || !c->v || !c->k_exp || !c->v_exp) return TS_ERR_NULL;
  if (c->pages < 1 || c->H < 1) return TS_ERR_SHAPE;
  if (c->d != 64 && c->d != 128) return TS_ERR_HEAD_DIM;
  // H * 64 * d * 4 bytes of a page's heads within 32 bits, so the pool's bytes are below 2^62
  if ((int64_t)c->H * TS_CACHE_PAGE * c->d * 4 >= kByteLimit) return TS_ERR_SHAPE;
  if (misaligned(c->k, 16) || misaligned(c->v, 16) || misaligned(c->weight, 16)) return TS_ERR_ALIGN;
  return TS_OK;
}

// Checks of the sessions: max_rows rows of row_bytes, tables of `width` pages, at most max_len tokens.
int check_sessions(const ts_cache* c, int32_t nseq, int32_t width, int32_t max_rows, int32_t max_len,
                   int32_t total, int64_t heads) {
  if (nseq < 0 || width < 0 || max_rows < 0 || max_len < 0 || total < 0) return TS_ERR_SHAPE;
  if (((int64_t)width * TS_CACHE_PAGE + 256) * c->d >= kByteLimit) return TS_ERR_SHAPE;
  if (max_len > (int64_t)width * TS_CACHE_PAGE) return TS_ERR_SHAPE;
  const int64_t row_bytes = heads * c->d * 2;
  if (row_bytes >= kByteLimit || (int64_t)max_rows + 256 > (kByteLimit - 1) / row_bytes) return TS_ERR_SHAPE;
  return TS_OK;
}

bool validate_mode() {
  const char* e = getenv("TS_ATTN_VALIDATE");
  return e && e[0] == '1';
}

tscache::Pool pool_of(const ts_cache* c) {
  return {(uint8_t*)c->k, (uint8_t*)c->v, c->k_exp, c->v_exp, c->weight, c->pages, c->H};
}

// Validation mode: the sessions' arrays on the host, after the work that is on the stream.  new_table, where
// there is one, has new_pages entries of use per session at most, of rows new_width apart.
int validate(const tscache::Sessions& ss, int32_t pages, bool append, const int32_t* new_table,
             int32_t new_width, int32_t keep, hipStream_t s) {
  const size_t n = (size_t)ss.nseq, tab = n * (size_t)ss.width, ntab = new_table ? n * (size_t)new_width : 0;
  std::unique_ptr<int32_t[]> buf(new (std::nothrow) int32_t[n + 1 + n + tab + ntab]);
  if (!buf) return TS_ERR_NOMEM;
  int32_t *cu = buf.get(), *lens = cu + n + 1, *table = lens + n, *to = table + tab;
  memset(cu, 0, (n + 1) * 4);
  const bool copied =
      (!ss.cu || hipMemcpyAsync(cu, ss.cu, (n + 1) * 4, hipMemcpyDeviceToHost, s) == hipSuccess) &&
      hipMemcpyAsync(lens, ss.lens, n * 4, hipMemcpyDeviceToHost, s) == hipSuccess &&
      (tab == 0 || hipMemcpyAsync(table, ss.table, tab * 4, hipMemcpyDeviceToHost, s) == hipSuccess) &&
      (ntab == 0 || hipMemcpyAsync(to, new_table, ntab * 4, hipMemcpyDeviceToHost, s) == hipSuccess);
  if (!copied || hipStreamSynchronize(s) != hipSuccess) {
    (void)hipGetLastError();
    return TS_ERR_HIP;
  }
  for (size_t i = 0; i < n; ++i) {
    int64_t len = lens[i];
    if (len < 0 || len > ss.max_len) return TS_ERR_SEGMENTS;
    if (ss.cu) {
      if (cu[i] < 0 || cu[i + 1] < cu[i] || cu[i + 1] > ss.total || cu[i + 1] - cu[i] > ss.max_rows)
        return TS_ERR_SEGMENTS;
      if (append) len += cu[i + 1] - cu[i];
    }
    if (len > (int64_t)ss.width * TS_CACHE_PAGE) return TS_ERR_SEGMENTS;
    for (int64_t p = 0; p < (len + TS_CACHE_PAGE - 1) / TS_CACHE_PAGE; ++p) {
      const int32_t page = table[i * ss.width + p];
      if (page < 0 || page >= pages) return TS_ERR_SEGMENTS;
    }
    if (new_table)
      for (int64_t p = 0; p < (std::min<int64_t>(len, keep) + TS_CACHE_PAGE - 1) / TS_CACHE_PAGE; ++p) {
        const int32_t page = to[i * new_width + p];
        if (page < 0 || page >= pages) return TS_ERR_SEGMENTS;
      }
  }
  return TS_OK;
}

int launched(hipError_t e) {
  if (e == hipSuccess) return TS_OK;
  (void)hipGetLastError();
  return TS_ERR_HIP;
}

}  // namespace

extern "C" {

int ts_cache_abi_version(void) { return TS_CACHE_ABI_VERSION; }

int ts_cache_append(const ts_cache* cache, const void* k, const void* v, const int32_t* cu,
                    const int32_t* table, const int32_t* lens, int32_t* new_lens, int32_t nseq,
                    int32_t width, int32_t max_rows, int32_t total, void* stream) {
  int rc = check_pool(cache);
  if (rc != TS_OK) return rc;
  rc = check_sessions(cache, nseq, width, max_rows, 0, total, cache->H);
  if (rc != TS_OK) return rc;
  if (tscache::append_items(nseq, max_rows, cache->H) >= tscache::kGridLimit) return TS_ERR_SHAPE;
  if (nseq == 0) return TS_OK;
  if (!cu || !lens || !new_lens || (width > 0 && !table) || (total > 0 && (!k || !v))) return TS_ERR_NULL;
  if (misaligned(k, 16) || misaligned(v, 16)) return TS_ERR_ALIGN;
  const int64_t row_bytes = (int64_t)cache->H * cache->d * 2;
  const Span written[] = {{cache->k, pool_bytes(cache)},         {cache->v, pool_bytes(cache)},
                          {cache->k_exp, exp_bytes(cache)},      {cache->v_exp, exp_bytes(cache)},
                          {cache->weight, weight_bytes(cache)},  {new_lens, (int64_t)nseq * 4}};
  const Span read[] = {{k, total * row_bytes},        {v, total * row_bytes},
                       {cu, ((int64_t)nseq + 1) * 4}, {table, (int64_t)nseq * width * 4},
                       {lens, (int64_t)nseq * 4}};
  if (aliased(written, read)) return TS_ERR_ALIAS;
  const hipStream_t s = (hipStream_t)stream;
  if (!current_device(&rc, s)) return rc;
  tscache::AppendArgs a{pool_of(cache), {cu, table, lens, nseq, width, max_rows, width * TS_CACHE_PAGE, total},
                        k, v, new_lens, cache->d};
  if (validate_mode() && !capturing(s) &&
      (rc = validate(a.ss, cache->pages, true, nullptr, 0, 0, s)) != TS_OK)
    return rc;
  return launched(tscache::launch_append(a, s));
}

int ts_cache_attn(const ts_cache* cache, const void* q, void* o, float* lse, const int32_t* cu,
                  const int32_t* table, const int32_t* lens, int32_t nseq, int32_t width,
                  int32_t max_rows, int32_t max_len, int32_t total, int32_t Hq, float scale,
                  int32_t num_splits, void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check_pool(cache);
  if (rc != TS_OK) return rc;
  if (Hq < 1 || Hq % cache->H != 0 || num_splits < 0 || num_splits > TS_CACHE_MAX_SPLITS || workspace_bytes < 0)
    return TS_ERR_SHAPE;
  rc = check_sessions(cache, nseq, width, max_rows, max_len, total, Hq);
  if (rc != TS_OK) return rc;
  const int32_t G = Hq / cache->H;
  const int tile = tscache::call_tile(nseq, (int64_t)max_rows * G, max_len, cache->H, cache->d, scale, num_splits);
  if (tscache::attn_items(nseq, max_rows, total, cache->H, G, tile) * std::max(1, num_splits) >= tscache::kGridLimit ||
      tscache::merge_blocks(nseq, max_rows, Hq, cache->d) >= tscache::kGridLimit)
    return TS_ERR_SHAPE;
  if (!isfinite(scale)) return TS_ERR_SCALE;
  if (nseq == 0 || total == 0 || max_rows == 0) return TS_OK;
  if (!q || !o || !cu || !lens || (width > 0 && !table)) return TS_ERR_NULL;
  if (misaligned(q, 16) || misaligned(o, 16) || misaligned(lse, 4) || misaligned(workspace, 256))
    return TS_ERR_ALIGN;
  const int64_t row_bytes = (int64_t)Hq * cache->d * 2;
  if (!workspace) workspace_bytes = 0;
  const Span written[] = {{o, total * row_bytes}, {lse, (int64_t)total * Hq * 4}, {workspace, workspace_bytes}};
  const Span read[] = {{q, total * row_bytes},
                       {cache->k, pool_bytes(cache)},
                       {cache->v, pool_bytes(cache)},
                       {cache->k_exp, exp_bytes(cache)},
                       {cache->v_exp, exp_bytes(cache)},
                       {cu, ((int64_t)nseq + 1) * 4},
                       {table, (int64_t)nseq * width * 4},
                       {lens, (int64_t)nseq * 4}};
  if (aliased(written, read)) return TS_ERR_ALIAS;
  const tscache::Sessions ss{cu, table, lens, nseq, width, max_rows, max_len, total};
  auto parts_on = [&](int32_t cus) {
    return tscache::attn_parts(ss, cache->H, G, cache->d, tile, num_splits, workspace_bytes, cus);
  };
  if (num_splits > 0 && parts_on(1).bytes > workspace_bytes) return TS_ERR_SCRATCH;  // (as asked for, on any device)
  const hipStream_t s = (hipStream_t)stream;
  DeviceState* st = current_device(&rc, s);
  if (!st) return rc;
  const tscache::Parts parts = parts_on(st->cus);
  const tscache::AttnArgs a{pool_of(cache), ss, q, o, lse, (float*)((char*)workspace + parts.o_offset), (float*)workspace,
                            cache->d, G, tile, parts.n_split, parts.shares, scale};
  if (validate_mode() && !capturing(s) &&
      (rc = validate(a.ss, cache->pages, false, nullptr, 0, 0, s)) != TS_OK)
    return rc;
  return launched(tscache::launch_attn(a, s));
}

int64_t ts_cache_attn_workspace(int32_t nseq, int32_t max_rows, int32_t max_len, int32_t total,
                                int32_t H, int32_t Hq, int32_t d, int32_t num_splits) {
  if (nseq < 1 || max_rows < 1 || max_len < 0 || total < 1 || H < 1 || Hq < 1 || Hq % H != 0 ||
      (d != 64 && d != 128) || num_splits < 0 || num_splits > TS_CACHE_MAX_SPLITS)
    return 0;
  if ((int64_t)max_rows + 256 > (kByteLimit - 1) / ((int64_t)Hq * d * 2)) return 0;
  const int32_t cus = num_splits == 0 ? current_cus() : 1;  // (forced ranges are the same on any device)
  if (cus == 0) return 0;
  const tscache::Sessions ss{nullptr, nullptr, nullptr, nseq, 0, max_rows, max_len, total};
  const int tile = tscache::call_tile(nseq, (int64_t)max_rows * (Hq / H), max_len, H, d, 1.0f, num_splits);
  return tscache::attn_parts(ss, H, Hq / H, d, tile, num_splits, INT64_MAX, cus).bytes;
}

int ts_cache_weigh(const ts_cache* cache, const void* q, const float* lse, const int32_t* cu,
                   const int32_t* table, const int32_t* lens, float* weight_out, int32_t nseq,
                   int32_t width, int32_t max_rows, int32_t max_len, int32_t total, int32_t Hq,
                   float scale, void* stream) {
  int rc = check_pool(cache);
  if (rc != TS_OK) return rc;
  if (!cache->weight || !weight_out) return TS_ERR_NULL;
  if (Hq < 1 || Hq % cache->H != 0) return TS_ERR_SHAPE;
  rc = check_sessions(cache, nseq, width, max_rows, max_len, total, Hq);
  if (rc != TS_OK) return rc;
  if (tscache::weigh_items(nseq, max_len, cache->H) >= tscache::kGridLimit) return TS_ERR_SHAPE;
  if (!isfinite(scale)) return TS_ERR_SCALE;
  if (nseq == 0 || max_len == 0) return TS_OK;
  if ((total > 0 && (!q || !lse)) || !cu || !lens || (width > 0 && !table)) return TS_ERR_NULL;
  if (misaligned(q, 16) || misaligned(lse, 4) || misaligned(weight_out, 16)) return TS_ERR_ALIGN;
  const int64_t row_bytes = (int64_t)Hq * cache->d * 2;
  const Span written[] = {{weight_out, weight_bytes(cache)}};
  const Span read[] = {{q, total * row_bytes},
                       {lse, (int64_t)total * Hq * 4},
                       {cache->k, pool_bytes(cache)},
                       {cache->v, pool_bytes(cache)},
                       {cache->k_exp, exp_bytes(cache)},
                       {cache->v_exp, exp_bytes(cache)},
                       {weight_out == cache->weight ? nullptr : cache->weight, weight_bytes(cache)},
                       {cu, ((int64_t)nseq + 1) * 4},
                       {table, (int64_t)nseq * width * 4},
                       {lens, (int64_t)nseq * 4}};
  if (aliased(written, read)) return TS_ERR_ALIAS;
  const hipStream_t s = (hipStream_t)stream;
  DeviceState* st = current_device(&rc, s);
  if (!st) return rc;
  tscache::WeighArgs a{pool_of(cache), {cu, table, lens, nseq, width, max_rows, max_len, total}, q, lse,
                       weight_out, cache->d, Hq / cache->H, scale, st->cus};
  if (validate_mode() && !capturing(s) &&
      (rc = validate(a.ss, cache->pages, false, nullptr, 0, 0, s)) != TS_OK)
    return rc;
  return launched(tscache::launch_weigh(a, s));
}

int ts_cache_evict(const ts_cache* cache, const int32_t* table, const int32_t* lens,
                   const int32_t* new_table, int32_t* new_lens, int32_t* kept, int32_t nseq,
                   int32_t width, int32_t new_width, int32_t max_len, int32_t keep, int32_t first,
                   int32_t last, void* stream) {
  int rc = check_pool(cache);
  if (rc != TS_OK) return rc;
  if (!cache->weight) return TS_ERR_NULL;
  rc = check_sessions(cache, nseq, width, 0, max_len, 0, cache->H);
  if (rc != TS_OK) return rc;
  if (new_width < 0 || keep < 0 || first < 0 || last < 0 || (int64_t)first + last > keep ||
      keep > (int64_t)new_width * TS_CACHE_PAGE || ((int64_t)new_width * TS_CACHE_PAGE + 256) * cache->d >= kByteLimit)
    return TS_ERR_SHAPE;
  // before any size is formed from them; the first kernel's workgroups are 1024 threads
  if ((int64_t)nseq * cache->H >= tscache::kGridLimit / 4 ||
      tscache::gather_items(nseq, keep, cache->H) >= tscache::kGridLimit)
    return TS_ERR_SHAPE;
  if (nseq == 0) return TS_OK;
  if (!lens || !new_lens || (width > 0 && !table) || (keep > 0 && (!new_table || !kept))) return TS_ERR_NULL;
  const Span written[] = {{cache->k, pool_bytes(cache)},
                          {cache->v, pool_bytes(cache)},
                          {cache->k_exp, exp_bytes(cache)},
                          {cache->v_exp, exp_bytes(cache)},
                          {cache->weight, weight_bytes(cache)},
                          {new_lens, (int64_t)nseq * 4},
                          {kept, (int64_t)nseq * cache->H * keep * 4}};
  const Span read[] = {{table, (int64_t)nseq * width * 4},
                       {new_table, (int64_t)nseq * new_width * 4},
                       {lens, (int64_t)nseq * 4}};
  if (aliased(written, read)) return TS_ERR_ALIAS;
  const hipStream_t s = (hipStream_t)stream;
  if (!current_device(&rc, s)) return rc;
  tscache::EvictArgs a{pool_of(cache), {nullptr, table, lens, nseq, width, 0, max_len, 0}, new_table, new_lens,
                       kept, cache->d, new_width, keep, first, last};
  if (validate_mode() && !capturing(s) &&
      (rc = validate(a.ss, cache->pages, false, new_table, new_width, keep, s)) != TS_OK)
    return rc;
  return launched(tscache::launch_evict(a, s));
}

}  // extern "C"
