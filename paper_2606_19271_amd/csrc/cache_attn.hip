// cache_attn.hip -- gfx950 kernels that read the session cache's pages: attention, and the weight that
// its queries give to each cached token.
//
// For every session s, query row t of it, query head hq (of cached head h = hq / G):
//   O[t,hq,:] = softmax_j(scale <Q[t,hq,:], K[j,h,:]>) V[j,h,:]   over the session's cached tokens j.
// Elements of a page are e4m3 times a power of two, so each is exact in bfloat16: the products run on the
// bf16 matrix cores with fp32 accumulation, on exactly the cached values.
//
// The G query heads of a cached head are further rows of the same problem (row_of).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_launch.h"
#include "cache_rows.h"

namespace tscache {

// ---- attention of few query rows: a tile of 16 NB of them over a range of pages, one workgroup of four waves.
constexpr int kRowThreads = 256;
constexpr int kRowWaves = kRowThreads / 64;

template <int D, int NB, bool kPartial>
__global__ void __launch_bounds__(kRowThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
cache_rows_kernel(RowArgs a) {
  __shared__ __attribute__((aligned(16))) char smem[RowGeo<D, NB, kRowWaves>::kLds];
  // consecutive workgroups: the page ranges of a tile, then the tiles of a head
  int b = blockIdx.x;
  const int split = b % a.n_split;
  b /= a.n_split;
  const int tile = b % a.tiles;
  b /= a.tiles;
  const int h = b % a.pool.H, s = b / a.pool.H;
  const Session se = session_of(a.ss, s);
  const int rows = se.rows * a.G, row0 = tile * 16 * NB;
  if (!se.ok || row0 >= rows) return;
  const int pages = (se.len + kPage - 1) / kPage;
  const int per = (pages + a.n_split - 1) / a.n_split;
  const int begin = __builtin_amdgcn_readfirstlane(min(pages, split * per));
  const int end = __builtin_amdgcn_readfirstlane(min(pages, begin + per));
  rows_item<D, NB, kRowWaves, kPartial>(a, se, a.ss.table + (int64_t)s * a.ss.width, h, row0, rows, begin, end, split,
                                        smem);
}

// Joins the page ranges of a split call: O = sum_i exp(lse_i - lse) O_i with lse = ln sum_i exp(lse_i).  One
// thread per 8 channels of a row, per_session workgroups to a session.
template <int D>
__global__ void __launch_bounds__(kMergeThreads) cache_merge_kernel(RowArgs a, int per_session) {
  constexpr int kChunks = D / 8;
  const int s = blockIdx.x / per_session, Hq = a.pool.H * a.G;
  const Session se = session_of(a.ss, s);
  const int64_t i = (int64_t)(blockIdx.x % per_session) * kMergeThreads + threadIdx.x;
  if (!se.ok || i / kChunks >= (int64_t)se.rows * Hq) return;
  const int64_t row = (int64_t)se.q0 * Hq + i / kChunks, all = (int64_t)a.ss.total * Hq;
  const int ch = (int)(i % kChunks) * 8;
  float big = -INFINITY;
  for (int n = 0; n < a.n_split; ++n) big = fmaxf(big, a.part_lse[n * all + row]);
  f32x4 x = {}, y = {};
  float sum = 0.0f;
  for (int n = 0; n < a.n_split; ++n) {
    const float e = a.part_lse[n * all + row];
    if (e == -INFINITY) continue;  // a range without keys has no O
    const float w = e == big ? 1.0f : __builtin_amdgcn_exp2f((e - big) * kLog2e);
    const f32x4* const src = (const f32x4*)(a.part_o + (n * all + row) * D + ch);
    sum += w;
    x += w * src[0];
    y += w * src[1];
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  bf16x8 r;
#pragma unroll
  for (int c = 0; c < 4; ++c) r[c] = (__bf16)(x[c] * inv), r[4 + c] = (__bf16)(y[c] * inv);
  *(bf16x8*)(a.o + row * D + ch) = r;
  if (a.lse != nullptr && ch == 0) a.lse[row] = sum == 0.0f ? -INFINITY : big + log2f(sum) * kLn2;
}

// ---- the weight that the queries give to each cached token: column sums of the softmax, one workgroup
// per (session, page, head).  A wave holds the page's keys as MFMA operands and takes every fourth tile of 32
// query rows: S^T = K Q^T on 32x32x16 MFMAs (lane: query row lane & 31), weights against the rows' lse, and
// their sums over the rows in the lane, across the lanes at the end.
template <int D>
__global__ void __launch_bounds__(kRowThreads)
cache_weigh_kernel(Pool pool, Sessions ss, const __bf16* __restrict__ q, const float* __restrict__ lse,
                   float* __restrict__ out, int G, int page_slots, float c, unsigned flip) {
  constexpr int kKK = D / 16;
  __shared__ float sums[kRowWaves][kPage];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, hb = lane >> 5;
  const int H = pool.H;
  int b = blockIdx.x;
  const int p = b % page_slots;
  b /= page_slots;
  const int h = b % H, s = b / H;
  const Session se = session_of(ss, s);
  if (!se.ok || p * kPage >= se.len) return;
  const int page = ss.table[(int64_t)s * ss.width + p];
  if ((unsigned)page >= (unsigned)pool.pages) return;
  const int64_t ph = (int64_t)page * H + h;
  const float ks = scale_of(pool.k_exp[ph], false);
  bf16x8 kf[2][kKK];
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int x = 0; x < kKK / 2; ++x) {
      const u32x4 y = *(const u32x4*)(pool.k + ph * (kPage * D) + (32 * kb + col) * D + D / 2 * hb + 16 * x);
      kf[kb][2 * x] = widen8(y[0], y[1], ks);
      kf[kb][2 * x + 1] = widen8(y[2], y[3], ks);
    }
  const int rows = se.rows * G;
  f32x16 acc[2] = {};
  for (int r0 = 32 * wave; r0 < rows; r0 += 32 * kRowWaves) {
    const int r = r0 + col;
    const int64_t at = row_of(se, min(r, rows - 1), h, H, G);
    const float ls = r < rows ? lse[at] * kLog2e : INFINITY;  // rows past the end weigh nothing
    f32x16 sc[2] = {};
#pragma unroll
    for (int kk = 0; kk < kKK; ++kk) {
      const bf16x8 qf = __builtin_bit_cast(
          bf16x8, *(const u32x4*)(q + at * D + D / 2 * hb + 8 * kk) ^ u32x4{flip, flip, flip, flip});
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) sc[kb] = mfma32(kf[kb][kk], qf, sc[kb]);
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[kb][i], c, -ls));
        acc[kb][i] += r < rows ? w : 0.0f;
      }
  }
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      float x = acc[kb][i];
#pragma unroll
      for (int m = 1; m < 32; m <<= 1) x += __shfl_xor(x, m);
      if (col == 0) sums[wave][32 * kb + 8 * (i >> 2) + 4 * hb + (i & 3)] = x;
    }
  __syncthreads();
  if (tid < kPage && p * kPage + tid < se.len) {
    float x = pool.weight[ph * kPage + tid];
#pragma unroll
    for (int w = 0; w < kRowWaves; ++w) x += sums[w][tid];
    out[ph * kPage + tid] = x;
  }
}

// ---------------------------------------------------------------------------------------------
// host-side launchers

template <int D, bool kPartial>
static void launch_rows(const RowArgs& r, int tile, unsigned grid, hipStream_t st) {
  auto kern = tile == 16 ? cache_rows_kernel<D, 1, kPartial> : cache_rows_kernel<D, 2, kPartial>;
  hipLaunchKernelGGL(kern, dim3(grid), dim3(kRowThreads), 0, st, r);
}

template <int D>
static hipError_t launch_attn_d(const AttnArgs& a, hipStream_t st) {
  const int64_t rows = (int64_t)a.ss.max_rows * a.G;
  const int tile = row_tile(rows, a.scale);
  RowArgs r{a.pool, a.ss, (const __bf16*)a.q, (__bf16*)a.o, a.lse, a.part_o, a.part_lse, a.G, a.n_split,
            (int)((rows + tile - 1) / tile), fabsf(a.scale) * kLog2e, a.scale < 0.0f ? 0x80008000u : 0u};
  const int64_t items = attn_items(a.ss.nseq, a.ss.max_rows, a.ss.total, a.pool.H, a.G, tile) * a.n_split;
  if (tile == kTileRows) launch_tiles(r, D, items, st);
  else if (a.n_split > 1) launch_rows<D, true>(r, tile, (unsigned)items, st);
  else launch_rows<D, false>(r, tile, (unsigned)items, st);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_split == 1) return e;
  const int64_t blocks = merge_blocks(a.ss.nseq, a.ss.max_rows, a.pool.H * a.G, D);
  hipLaunchKernelGGL(cache_merge_kernel<D>, dim3((unsigned)blocks), dim3(kMergeThreads), 0, st, r,
                     (int)(blocks / a.ss.nseq));
  return hipGetLastError();
}

hipError_t launch_attn(const AttnArgs& a, hipStream_t st) {
  return a.d == 64 ? launch_attn_d<64>(a, st) : launch_attn_d<128>(a, st);
}

hipError_t launch_weigh(const WeighArgs& a, hipStream_t st) {
  const int64_t items = weigh_items(a.ss.nseq, a.ss.max_len, a.pool.H);
  auto kern = a.d == 64 ? cache_weigh_kernel<64> : cache_weigh_kernel<128>;
  hipLaunchKernelGGL(kern, dim3((unsigned)items), dim3(kRowThreads), 0, st, a.pool, a.ss, (const __bf16*)a.q,
                     a.lse, a.out, a.G, (a.ss.max_len + kPage - 1) / kPage, fabsf(a.scale) * kLog2e,
                     a.scale < 0.0f ? 0x80008000u : 0u);
  return hipGetLastError();
}

hipError_t configure_kernels() { return configure_tiles(); }

}  // namespace tscache
