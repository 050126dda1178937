// ts_block.cpp -- the C ABI of libts_block.so (declared in include/ts_block.h): argument checks, per-device set-up,
// validation mode, and the launches.
#include "ts_block.h"

#include <float.h>
#include <hip/hip_runtime_api.h>
#include <math.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <atomic>
#include <memory>
#include <new>

#include "block_launch.h"
#include "device_setup.h"

namespace {

using namespace tshost;

constexpr int64_t kByteLimit = (int64_t)1 << 31;

struct DeviceState : DeviceSetup {
  std::atomic<int32_t> cus{0};  // compute units, or 0: not asked for yet
};

DeviceState g_dev[kMaxDevices];

void init_device(int dev, DeviceState* st) {
  hipDeviceProp_t p;
  if (hipGetDeviceProperties(&p, dev) != hipSuccess) { (void)hipGetLastError(); st->status = TS_ERR_HIP; return; }
  if (strncmp(p.gcnArchName, "gfx950", 6) != 0) { st->status = TS_ERR_UNSUPPORTED; return; }
  st->cus = p.multiProcessorCount;
  if (tsblock::configure_kernels() != hipSuccess) { (void)hipGetLastError(); st->status = TS_ERR_HIP; return; }
  st->status = TS_OK;
}

// Compute units of the calling thread's current device, or 0.  Sets nothing up, so that it can be asked while a stream is
// being captured.
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

int launched(hipError_t e) {
  if (e == hipSuccess) return TS_OK;
  (void)hipGetLastError();
  return TS_ERR_HIP;
}

// Device memory that a call reads or writes: `bytes` at p, every `stride` bytes, `rows` times.
struct Span {
  const void* p;
  int64_t bytes, stride, rows;
};

Span flat(const void* p, int64_t bytes) { return {p, bytes, bytes, 1}; }

bool overlap(const Span& a, const Span& b) {
  if (!a.p || !b.p || a.bytes <= 0 || b.bytes <= 0 || a.rows <= 0 || b.rows <= 0) return false;
  const uintptr_t x = (uintptr_t)a.p, y = (uintptr_t)b.p;
  const uintptr_t x_end = x + (uintptr_t)((a.rows - 1) * a.stride + a.bytes), y_end = y + (uintptr_t)((b.rows - 1) * b.stride + b.bytes);
  if (x >= y_end || y >= x_end) return false;
  if (a.stride != b.stride || a.rows == 1 || b.rows == 1) return true;
  // rows of one stride side by side, as those of a fused projection
  const int64_t to_b = (int64_t)((y - x) % (uintptr_t)a.stride), ahead = y >= x ? to_b : a.stride - (int64_t)((x - y) % (uintptr_t)a.stride);
  const int64_t d = ahead % a.stride;
  return d < a.bytes || d + b.bytes > a.stride;
}

bool same(const Span& a, const Span& b) { return a.p == b.p && a.bytes == b.bytes && (a.stride == b.stride || a.rows <= 1); }

// Whether written span i meets another written one, or a read one that is not its own memory where it may be.
template <int W, int R>
bool aliased(const Span (&written)[W], const Span (&read)[R], const bool (&in_place)[W][R]) {
  for (int i = 0; i < W; ++i) {
    for (int j = i + 1; j < W; ++j)
      if (overlap(written[i], written[j])) return true;
    for (int j = 0; j < R; ++j)
      if (overlap(written[i], read[j]) && !(in_place[i][j] && same(written[i], read[j]))) return true;
  }
  return false;
}

// Checks of one set of rows, or of none.
int check_rows(const ts_rows* x, int32_t T, int32_t d) {
  if (!x) return TS_OK;
  if (x->heads < 1 || x->stride < (int64_t)x->heads * d || x->stride >= ((int64_t)1 << 30)) return TS_ERR_SHAPE;
  if (x->stride % 8 != 0 || misaligned(x->p, 16)) return TS_ERR_ALIGN;
  return T > 0 && !x->p ? TS_ERR_NULL : TS_OK;
}

Span span_of(const ts_rows* x, int32_t T, int32_t d) {
  if (!x) return {nullptr, 0, 0, 0};
  return {x->p, (int64_t)x->heads * d * 2, x->stride * 2, T};
}

tsblock::Rows rows_of(const ts_rows* x) { return x ? tsblock::Rows{x->p, x->stride, x->heads} : tsblock::Rows{nullptr, 0, 0}; }

// What ts_qk_rope and its gradients check alike, in this order: sizes, values, pointers.
int check_rope(const ts_rope* r, int32_t T, int32_t d, int64_t heads, float eps) {
  if (d != 64 && d != 128) return TS_ERR_HEAD_DIM;
  if (T < 0 || heads * std::max(T, 1) >= kByteLimit - 65536) return TS_ERR_SHAPE;
  if (!(eps >= FLT_MIN) || !isfinite(eps)) return TS_ERR_SCALE;
  if (!r) return TS_OK;
  if (r->axes[0] < 0 || r->axes[1] < 0 || r->axes[2] < 0 || (int64_t)r->axes[0] + r->axes[1] + r->axes[2] != d / 2) return TS_ERR_SHAPE;
  if ((T > 0 && !r->pos) || !r->freq) return TS_ERR_NULL;
  if (misaligned(r->pos, 4) || misaligned(r->freq, 8)) return TS_ERR_ALIGN;
  return TS_OK;
}

tsblock::Rope rope_of(const ts_rope* r) {
  if (!r) return {nullptr, nullptr, 0, 0, 0};
  return {r->pos, r->freq, r->axes[0], r->axes[0] + r->axes[1], r->interleaved != 0};
}

bool validate_mode() {
  const char* e = getenv("TS_ATTN_VALIDATE");
  return e && e[0] == '1';
}

// Validation mode: the offsets on the host, after the work that is on the stream.
int validate(const int32_t* cu_q, const int32_t* cu_k, int32_t nseq, int32_t max_q, int32_t max_k, int32_t total_q, int32_t total_k,
             hipStream_t s) {
  const size_t n = (size_t)nseq + 1;
  std::unique_ptr<int32_t[]> buf(new (std::nothrow) int32_t[2 * n]);
  if (!buf) return TS_ERR_NOMEM;
  if (hipMemcpyAsync(buf.get(), cu_q, n * 4, hipMemcpyDeviceToHost, s) != hipSuccess ||
      hipMemcpyAsync(buf.get() + n, cu_k, n * 4, hipMemcpyDeviceToHost, s) != hipSuccess || hipStreamSynchronize(s) != hipSuccess) {
    (void)hipGetLastError();
    return TS_ERR_HIP;
  }
  for (int side = 0; side < 2; ++side) {
    const int32_t* cu = buf.get() + side * n;
    const int32_t most = side ? max_k : max_q, total = side ? total_k : total_q;
    if (cu[0] != 0 || cu[nseq] != total) return TS_ERR_SEGMENTS;
    for (int32_t i = 0; i < nseq; ++i)
      if (cu[i + 1] < cu[i] || (int64_t)cu[i + 1] - cu[i] > most) return TS_ERR_SEGMENTS;
  }
  return TS_OK;
}

constexpr float kLeastScale = 0x1p-100f, kMostScale = 0x1p100f;

constexpr int kLeastTile = 128;  // held rows of a workgroup, at least
constexpr int64_t kItemLimit = (int64_t)1 << 23;  // workgroups of a launch (x 512 threads < 2^32)

// Sizes of an attention gradient call.
int check_sizes(int32_t nseq, int32_t max_q, int32_t max_k, int32_t total_q, int32_t total_k, int32_t H, int32_t d, int32_t num_splits) {
  if (d != 64 && d != 128) return TS_ERR_HEAD_DIM;
  if (nseq < 0 || max_q < 0 || max_k < 0 || total_q < 0 || total_k < 0 || H < 1 || num_splits < 0 || num_splits > TS_ATTN_BWD_MAX_SPLITS)
    return TS_ERR_SHAPE;
  const int64_t row_bytes = (int64_t)H * d * 2;
  if (row_bytes >= kByteLimit || std::max(max_q, max_k) + (int64_t)256 > (kByteLimit - 1) / row_bytes) return TS_ERR_SHAPE;
  // H < 2^24 and tiles < 2^24 from here on, so the products below are within 64 bits
  const int64_t tiles = (int64_t)max_q / kLeastTile + max_k / kLeastTile + 2;
  if ((int64_t)nseq * H >= (int64_t)1 << 26 || (int64_t)nseq * H * tiles >= (int64_t)1 << 26) return TS_ERR_SHAPE;
  if (H * ((int64_t)std::max(total_q, total_k) / kLeastTile + nseq) >= (int64_t)1 << 19) return TS_ERR_SHAPE;
  // (undivided calls have less than 2^20 workgroups by that, and the library divides only those of a few rounds of the device)
  if (num_splits > 1 && tsblock::bwd_forced_items(nseq, max_q, max_k, total_q, total_k, H, d, num_splits) >= kItemLimit) return TS_ERR_SHAPE;
  return TS_OK;
}

}  // namespace

extern "C" {

int ts_block_abi_version(void) { return TS_BLOCK_ABI_VERSION; }

int ts_qk_rope(const ts_rows* q, const ts_rows* k, const ts_rows* q_out, const ts_rows* k_out, const float* q_weight,
               const float* k_weight, const ts_rope* rope, int32_t T, int32_t d, float eps, void* stream) {
  if (!q || !q_out || (k != nullptr) != (k_out != nullptr)) return TS_ERR_NULL;
  const int64_t heads = (int64_t)q->heads + (k ? k->heads : 0);
  int rc = check_rope(rope, T, d, heads, eps);
  if (rc != TS_OK) return rc;
  if (q_out->heads != q->heads || (k && k_out->heads != k->heads)) return TS_ERR_SHAPE;
  for (const ts_rows* x : {q, k, q_out, k_out})
    if ((rc = check_rows(x, T, d)) != TS_OK) return rc;
  if (misaligned(q_weight, 4) || misaligned(k_weight, 4)) return TS_ERR_ALIGN;
  if (T == 0) return TS_OK;
  const Span written[] = {span_of(q_out, T, d), span_of(k_out, T, d)};
  const Span read[] = {span_of(q, T, d), span_of(k, T, d), flat(q_weight, d * 4), flat(k_weight, d * 4),
                       flat(rope ? rope->pos : nullptr, (int64_t)T * 12), flat(rope ? rope->freq : nullptr, d * 4)};
  const bool in_place[2][6] = {{true}, {false, true}};
  if (aliased(written, read, in_place)) return TS_ERR_ALIAS;
  const hipStream_t s = (hipStream_t)stream;
  if (!current_device(&rc, s)) return rc;
  return launched(tsblock::launch_rope({rows_of(q), rows_of(k), rows_of(q_out), rows_of(k_out), q_weight, k ? k_weight : nullptr,
                                        rope_of(rope), T, d, eps}, s));
}

int64_t ts_qk_rope_bwd_workspace(int32_t T, int32_t q_heads, int32_t k_heads, int32_t d) {
  if (T < 0 || q_heads < 1 || k_heads < 0 || (d != 64 && d != 128) ||
      ((int64_t)q_heads + k_heads) * std::max(T, 1) >= kByteLimit - 65536)
    return 0;
  return (int64_t)tsblock::rope_bwd_blocks(T, q_heads, k_heads, d) * 2 * d * 4;
}

int ts_qk_rope_bwd(const ts_rows* dq_out, const ts_rows* dk_out, const ts_rows* q, const ts_rows* k, const ts_rows* dq,
                   const ts_rows* dk, const float* q_weight, const float* k_weight, float* dq_weight, float* dk_weight,
                   const ts_rope* rope, int32_t T, int32_t d, float eps, void* workspace, int64_t workspace_bytes,
                   void* stream) {
  if (!dq_out || !dq || (dk_out != nullptr) != (dk != nullptr)) return TS_ERR_NULL;
  const int64_t heads = (int64_t)dq->heads + (dk ? dk->heads : 0);
  int rc = check_rope(rope, T, d, heads, eps);
  if (rc != TS_OK) return rc;
  if ((q_weight && !q) || (k_weight && dk && !k) || (q_weight != nullptr) != (dq_weight != nullptr) ||
      (k_weight != nullptr) != (dk_weight != nullptr) || (k_weight && !dk))
    return TS_ERR_NULL;
  if (!q_weight) q = nullptr;  // not read
  if (!k_weight) k = nullptr;
  if (dq_out->heads != dq->heads || (dk && dk_out->heads != dk->heads) || (q && q->heads != dq->heads) || (k && k->heads != dk->heads))
    return TS_ERR_SHAPE;
  for (const ts_rows* x : {dq_out, dk_out, q, k, dq, dk})
    if ((rc = check_rows(x, T, d)) != TS_OK) return rc;
  if (misaligned(q_weight, 4) || misaligned(k_weight, 4) || misaligned(dq_weight, 4) || misaligned(dk_weight, 4) ||
      misaligned(workspace, 256))
    return TS_ERR_ALIGN;
  const bool weights = q_weight || k_weight;
  const int64_t need = weights ? ts_qk_rope_bwd_workspace(T, dq->heads, dk ? dk->heads : 0, d) : 0;
  if (workspace_bytes < 0) return TS_ERR_SHAPE;
  if (need > 0 && (!workspace || workspace_bytes < need)) return TS_ERR_SCRATCH;
  if (T == 0 && !weights) return TS_OK;
  const Span written[] = {span_of(dq, T, d), span_of(dk, T, d), flat(dq_weight, d * 4), flat(dk_weight, d * 4), flat(workspace, need)};
  const Span read[] = {span_of(dq_out, T, d), span_of(dk_out, T, d), span_of(q, T, d), span_of(k, T, d), flat(q_weight, d * 4),
                       flat(k_weight, d * 4), flat(rope ? rope->pos : nullptr, (int64_t)T * 12),
                       flat(rope ? rope->freq : nullptr, d * 4)};
  const bool in_place[5][8] = {{true, false, true}, {false, true, false, true}};
  if (aliased(written, read, in_place)) return TS_ERR_ALIAS;
  const hipStream_t s = (hipStream_t)stream;
  if (!current_device(&rc, s)) return rc;
  return launched(tsblock::launch_rope_bwd({rows_of(dq_out), rows_of(dk_out), rows_of(q), rows_of(k), rows_of(dq), rows_of(dk),
                                            q_weight, k_weight, dq_weight, dk_weight, weights ? (float*)workspace : nullptr,
                                            rope_of(rope), T, d, eps}, s));
}

int ts_attn_bwd(const void* d_o, const void* q, const void* k, const void* v, const void* o, const float* lse, void* dq,
                void* dk, void* dv, const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, int32_t nseq,
                int32_t max_seqlen_q, int32_t max_seqlen_k, int32_t total_q, int32_t total_k, int32_t H, int32_t d,
                float scale, int32_t num_splits, void* workspace, int64_t workspace_bytes, void* stream) {
  int rc = check_sizes(nseq, max_seqlen_q, max_seqlen_k, total_q, total_k, H, d, num_splits);
  if (rc != TS_OK) return rc;
  if (workspace_bytes < 0) return TS_ERR_SHAPE;
  if (!isfinite(scale) || (scale != 0.0f && (fabsf(scale) < kLeastScale || fabsf(scale) > kMostScale))) return TS_ERR_SCALE;
  if (total_q == 0 && total_k == 0) return TS_OK;
  if (nseq == 0) return validate_mode() && !capturing((hipStream_t)stream) ? TS_ERR_SEGMENTS : TS_OK;
  if ((total_q > 0 && (!q || !d_o || !o || !lse || !dq)) || (total_k > 0 && (!k || !v || !dk || !dv)) || !cu_seqlens_q || !cu_seqlens_k)
    return TS_ERR_NULL;
  for (const void* p : {d_o, q, k, v, o, (const void*)dq, (const void*)dk, (const void*)dv})
    if (misaligned(p, 16)) return TS_ERR_ALIGN;
  if (misaligned(lse, 4) || misaligned(cu_seqlens_q, 4) || misaligned(cu_seqlens_k, 4) || misaligned(workspace, 256)) return TS_ERR_ALIGN;
  const int64_t bytes_q = (int64_t)total_q * H * d * 2, bytes_k = (int64_t)total_k * H * d * 2, bytes_cu = ((int64_t)nseq + 1) * 4;
  if (!workspace) workspace_bytes = 0;
  const Span written[] = {flat(dq, bytes_q), flat(dk, bytes_k), flat(dv, bytes_k), flat(workspace, workspace_bytes)};
  const Span read[] = {flat(d_o, bytes_q), flat(q, bytes_q),  flat(k, bytes_k), flat(v, bytes_k),
                       flat(o, bytes_q),   flat(lse, (int64_t)total_q * H * 4), flat(cu_seqlens_q, bytes_cu), flat(cu_seqlens_k, bytes_cu)};
  const bool in_place[4][8] = {};
  if (aliased(written, read, in_place)) return TS_ERR_ALIAS;
  if (tsblock::bwd_least_workspace(nseq, max_seqlen_q, max_seqlen_k, total_q, total_k, H, d, num_splits) > workspace_bytes)
    return TS_ERR_SCRATCH;
  const hipStream_t s = (hipStream_t)stream;
  DeviceState* st = current_device(&rc, s);
  if (!st) return rc;
  if (validate_mode() && !capturing(s) &&
      (rc = validate(cu_seqlens_q, cu_seqlens_k, nseq, max_seqlen_q, max_seqlen_k, total_q, total_k, s)) != TS_OK)
    return rc;
  const tsblock::BwdParts p =
      tsblock::bwd_parts(nseq, max_seqlen_q, max_seqlen_k, total_q, total_k, H, d, num_splits, workspace_bytes, st->cus);
  char* const w = (char*)workspace;
  return launched(tsblock::launch_attn_bwd({d_o, q, k, v, o, lse, dq, dk, dv, cu_seqlens_q, cu_seqlens_k, (tsblock::BwdPlan*)w,
                                            (float*)(w + p.stat_offset), (float*)(w + p.q_offset), (float*)(w + p.k_offset), nseq, max_seqlen_q, max_seqlen_k,
                                            total_q, total_k, H, d, p.n_q, p.n_k, p.tile, scale}, s));
}

int64_t ts_attn_bwd_workspace(int32_t nseq, int32_t max_seqlen_q, int32_t max_seqlen_k, int32_t total_q,
                              int32_t total_k, int32_t H, int32_t d, int32_t num_splits) {
  if (check_sizes(nseq, max_seqlen_q, max_seqlen_k, total_q, total_k, H, d, num_splits) != TS_OK || nseq == 0) return 0;
  const int32_t cus = num_splits == 0 ? current_cus() : 1;  // (forced ranges are the same on any device)
  if (cus == 0) return 0;
  return tsblock::bwd_parts(nseq, max_seqlen_q, max_seqlen_k, total_q, total_k, H, d, num_splits, INT64_MAX, cus).bytes;
}

}  // extern "C"
