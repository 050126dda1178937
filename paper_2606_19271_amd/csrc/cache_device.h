// cache_device.h -- device code shared by the session cache's kernels: sessions, pages and the 8-bit format.
#pragma once
#include <float.h>
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "attn_tile.h"
#include "cache_launch.h"

namespace tscache {

using namespace tsattn;  // the types and products of attn_tile.h

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

// One session of a call, read by every workgroup that works on it.  ok: it is worked on at all (every
// bound is checked before a difference is formed, so nothing wraps).
struct Session {
  int q0, rows, len;
  bool ok;
};

__device__ __forceinline__ Session session_of(const Sessions& ss, int s) {
  Session r;
  r.q0 = 0, r.rows = 0;
  r.len = ss.lens[s];
  r.ok = r.len >= 0 && r.len <= ss.max_len;
  if (ss.cu != nullptr) {
    const int a = ss.cu[s], b = ss.cu[s + 1];
    r.ok = r.ok && a >= 0 && b <= ss.total && b >= a && b - a <= ss.max_rows;
    r.q0 = a, r.rows = r.ok ? b - a : 0;
  }
  return r;
}

// The bits of the float 2^(exp - 127); exponent 255 and pages outside the pool (bad) give infinity, with
// which the conversion below makes every element NaN.
__device__ __forceinline__ float scale_of(unsigned exp, bool bad) {
  return __uint_as_float((bad ? 255u : exp) << 23);
}

// A page's exponent `down` lower.  Values are widened to 2^-down of their size, and a row's sums scaled back with the division:
// products of the largest values with weights of 1 and less, added up over a row's keys, would pass the largest float.
// The smallest element of a page, 2^-109, stays a normal bfloat16 up to 17.
__device__ __forceinline__ unsigned value_exp(unsigned exp, unsigned down) { return exp < 255 ? max(exp, down) - down : exp; }

// Four e4m3 bytes as four bfloat16, times the scale's power of two (exact for the exponents that this
// library writes: e4m3 has 4 significant bits, and 2^-9 2^-100 is a normal bfloat16).
__device__ __forceinline__ bf16x4 widen4(unsigned x, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, true);
  return bf16x4{a[0], a[1], b[0], b[1]};
}

__device__ __forceinline__ bf16x8 widen8(unsigned x, unsigned y, float scale) {
  const bf16x4 a = widen4(x, scale), b = widen4(y, scale);
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Four floats, already scaled, rounded to nearest even e4m3.  |x| <= 448 here but for infinities and NaN,
// which both become NaN.
__device__ __forceinline__ unsigned narrow4(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  return (unsigned)r;
}

// Four bytes of a page with the largest exponent.  There a magnitude of 1.9375 * 2^127 or more is rounded to 256 * 2^120, which
// is no bfloat16: it becomes the element before, 240 * 2^120.
constexpr int kTopExp = 247;
__device__ __forceinline__ unsigned in_bf16(unsigned bytes) {
  const unsigned off = (bytes & 0x7f7f7f7fu) ^ 0x78787878u;  // 0 where the byte is +-256
  return bytes - (~(off + 0x7f7f7f7fu) >> 7 & 0x01010101u);
}

// The largest finite magnitude of packed bfloat16 bits, as bits (a positive bfloat16 orders as its bits).
__device__ __forceinline__ unsigned amax_bits(unsigned amax, unsigned packed) {
  const unsigned lo = packed & 0x7fffu, hi = packed >> 16 & 0x7fffu;
  amax = max(amax, lo < 0x7f80u ? lo : 0u);
  return max(amax, hi < 0x7f80u ? hi : 0u);
}

// The biased exponent of a page whose largest magnitude has these bfloat16 bits: 448 = 1.75 * 2^8, so
// 1.m * 2^x <= 448 * 2^n from n = x - 8 on where 1.m <= 1.75 (m <= 96 of 128), else one more; n >= -100.
__device__ __forceinline__ int exponent_of(unsigned amax) {
  const int x = (int)(amax >> 7), m = (int)(amax & 127u);
  return max(x - 8 + (m > 96 ? 1 : 0), 27);
}

// LDS DMA: lane i's 16 bytes at `offset` of the buffer land at to + 16 i.
__device__ __forceinline__ void dma16(__amdgpu_buffer_rsrc_t rsrc, lds_char* to, int offset) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)to, 16, offset, 0, 0, 0);
}

// threadIdx.x, of which nothing is derived ahead of the call: what a loop over items would keep in registers through
// all of them is formed for each anew.
__device__ __forceinline__ int thread_anew() {
  int t = threadIdx.x;
  __asm__ volatile("" : "+v"(t));
  return t;
}

// Bytes from a page's start to its head h, and the page itself; a page number outside the pool reads
// page 0 (in bounds, and poisoned through its scale).
__device__ __forceinline__ int64_t page_offset(int page, bool bad, int H, int h, int bytes) {
  return ((int64_t)(bad ? 0 : page) * H + h) * bytes;
}

// Row r of (session, cached head h) in q and o, in units of d elements (and in lse): the rows are the
// session's tokens, and of each the G query heads of h.
__device__ __forceinline__ int64_t row_of(const Session& se, int r, int h, int H, int G) {
  const int t = G == 1 ? r : r / G;
  return ((int64_t)se.q0 + t) * (H * G) + h * G + (r - t * G);
}

// |scale| log2(e); of the largest scales the largest float, since infinity times a score of 0 would be NaN.
inline float log2_scale(float scale) { return fminf(fabsf(scale) * kLog2e, FLT_MAX); }

// What the attention kernels take.
struct RowArgs {
  Pool pool;
  Sessions ss;
  const __bf16* q;
  __bf16* o;
  float* lse;
  float* part_o;
  float* part_lse;
  int G, n_split;
  int shares;     // equal shares of the work (cache_tiles_kernel), or 0
  int tiles;      // row tiles of a session at most (cache_rows_kernel)
  bool few;       // up to 64 rows in 256-row tiles (call_tile)
  float c;        // log2_scale
  unsigned flip;  // sign bits of Q to invert (negative scales)
};

// What becomes of an item's rows: they are the result, or one of n_split ranges' part of it (part_o[n_split][total][Hq]),
// or the part of it that a share of the work has (part_o[slots][256], kTileRows rows each).
enum Out { kResult, kSlab, kSlot };

constexpr float kPartDown = 1.0f / 1024;  // of up to that many parts: their sum stays below the largest float

// The 8 channels from `ch` on of a row whose n parts lie at rows part(0) .. part(n - 1) of part_o and part_lse:
// O = sum_i exp(lse_i - lse) O_i with lse = ln sum_i exp(lse_i), kBatch parts loaded at once.
template <int D, int kBatch, typename Part>
__device__ __forceinline__ void join_parts(const RowArgs& a, int n, Part&& part, int64_t row, int ch) {
  float big = -INFINITY, sum = 0.0f;
  f32x4 x = {}, y = {};
  for (int n0 = 0; n0 < n; n0 += kBatch) {
    float e[kBatch];
    f32x4 px[kBatch], py[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {  // (past the last part: that one's again, with no weight)
      const int64_t at = part(min(n0 + k, n - 1));
      const float l = a.part_lse[at];
      e[k] = n0 + k < n ? l : -INFINITY;
      const f32x4* const src = (const f32x4*)(a.part_o + at * D + ch);
      px[k] = src[0], py[k] = src[1];
    }
    float top = big;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) top = fmaxf(top, e[k]);
    const float old = big == top ? 1.0f : __builtin_amdgcn_exp2f((big - top) * kLog2e);
    big = top, sum *= old, x *= old, y *= old;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const bool none = e[k] == -INFINITY;  // a part without keys has no O
      const float w = none ? 0.0f : e[k] == big ? 1.0f : __builtin_amdgcn_exp2f((e[k] - big) * kLog2e);
      sum += w;
      const float f = w * kPartDown;
#pragma unroll
      for (int c = 0; c < 4; ++c) x[c] += none ? 0.0f : f * px[k][c], y[c] += none ? 0.0f : f * py[k][c];
    }
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / (sum * kPartDown);
  bf16x8 r;
#pragma unroll
  for (int c = 0; c < 4; ++c) r[c] = (__bf16)(x[c] * inv), r[4 + c] = (__bf16)(y[c] * inv);
  *(bf16x8*)(a.o + row * D + ch) = r;
  if (a.lse != nullptr && ch == 0) a.lse[row] = sum == 0.0f ? -INFINITY : big + log2f(sum) * kLn2;
}

// cache_tiles.hip
hipError_t configure_tiles();
hipError_t configure_pages();
void launch_tiles(const RowArgs& r, int d, int64_t items, hipStream_t st);

}  // namespace tscache
