// cache_attn.hip -- attention over the session cache's pages: the kernel for few query rows, the merge of split
// calls, and the choice between the kernels.
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

template <int D, int NB, Out kOut>
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
  const int32_t* const table = a.ss.table + (int64_t)s * a.ss.width;
  const int id = first_ids<kRowWaves>(table, a.ss.width, split, a.n_split);
  const Session se = session_of(a.ss, s);
  const int rows = se.rows * a.G, row0 = tile * 16 * NB;
  if (!se.ok || row0 >= rows) return;
  const PageRange range{split, a.n_split, (se.len + kPage - 1) / kPage};
  rows_item<D, NB, kRowWaves, kOut>(a, se, table, h, row0, rows, range, id, split, smem);
}

// Joins the page ranges of a split call: O = sum_i exp(lse_i - lse) O_i with lse = ln sum_i exp(lse_i).  One
// thread per 8 channels of a row, per_session workgroups to a session.  Bound by latency: one round trip after the
// sessions' rows, 8 ranges of 48 rows 2.6 us (7.2 us with a range loaded after the other).
constexpr int kMergeBatch = 8;  // ranges whose results are loaded at once

template <int D>
__global__ void __launch_bounds__(kMergeThreads) cache_merge_kernel(RowArgs a, int per_session) {
  constexpr int kChunks = D / 8;
  const int s = blockIdx.x / per_session, Hq = a.pool.H * a.G;
  const Session se = session_of(a.ss, s);
  const int64_t i = (int64_t)(blockIdx.x % per_session) * kMergeThreads + threadIdx.x;
  if (!se.ok || i / kChunks >= (int64_t)se.rows * Hq) return;
  const int64_t row = (int64_t)se.q0 * Hq + i / kChunks, all = (int64_t)a.ss.total * Hq;
  const int ch = (int)(i % kChunks) * 8;
  join_parts<D, kMergeBatch>(a, a.n_split, [&](int n) { return n * all + row; }, row, ch);
}

// ---------------------------------------------------------------------------------------------
// host-side launchers

template <int D, Out kOut>
static void launch_rows(const RowArgs& r, int tile, unsigned grid, hipStream_t st) {
  auto kern = tile == 16 ? cache_rows_kernel<D, 1, kOut> : cache_rows_kernel<D, 2, kOut>;
  hipLaunchKernelGGL(kern, dim3(grid), dim3(kRowThreads), 0, st, r);
}

template <int D>
static hipError_t launch_attn_d(const AttnArgs& a, hipStream_t st) {
  const int64_t rows = (int64_t)a.ss.max_rows * a.G;
  const int tile = a.tile;
  RowArgs r{a.pool, a.ss, (const __bf16*)a.q, (__bf16*)a.o, a.lse, a.part_o, a.part_lse, a.G, a.n_split, a.shares,
            (int)((rows + tile - 1) / tile), tile == kTileRows && rows <= 64, log2_scale(a.scale), a.scale < 0.0f ? 0x80008000u : 0u};
  const int64_t items = attn_items(a.ss.nseq, a.ss.max_rows, a.ss.total, a.pool.H, a.G, tile) * a.n_split;
  if (tile == kTileRows) launch_tiles(r, D, items, st);
  else if (a.n_split > 1) launch_rows<D, kSlab>(r, tile, (unsigned)items, st);
  else launch_rows<D, kResult>(r, tile, (unsigned)items, st);
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

hipError_t configure_kernels() {
  const hipError_t e = configure_tiles();
  return e != hipSuccess ? e : configure_pages();
}

}  // namespace tscache
