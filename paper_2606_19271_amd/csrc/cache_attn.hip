// cache_attn.hip -- gfx950 kernels that read the session cache's pages: attention, and the weight that
// its queries give to each cached token.
//
// For every session s, query row t of it, query head hq (of cached head h = hq / G):
//   O[t,hq,:] = softmax_j(scale <Q[t,hq,:], K[j,h,:]>) V[j,h,:]   over the session's cached tokens j.
// Elements of a page are e4m3 times a power of two, so each is exact in bfloat16: the products run on the
// bf16 matrix cores with fp32 accumulation, on exactly the cached values.
//
// The G query heads of a cached head are further rows of the same problem: row r of (session, h) is token
// r / G, query head h * G + r % G.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_launch.h"
#include "cache_device.h"

namespace tscache {

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// ---- attention of a tile of 16 NB query rows over a range of pages, one workgroup of four waves.
//
// The waves take the pages in turn and share nothing until the end, so there is no barrier in the loop.
// Per page a wave computes S^T = K Q^T on 16x16x32 MFMAs (lane: query row lane & 15, keys 4 (lane >> 4) +
// 0..3 of each 16), keeps a running maximum and sum per row, and accumulates O^T += V^T P^T, whose B operand
// is the lane's own weights, once the 32 keys of a step are taken in the order in which two score blocks
// hold them.  K goes from memory to MFMA operands in registers: a lane loads D / 4 consecutive channels of
// a key, and the sum over channels takes them in that order on both sides.  V passes through the wave's
// own LDS for the 8-bit transpose read (16-byte chunks XORed with the row so that its rows spread over the
// banks).
constexpr int kRowThreads = 256;
constexpr int kRowWaves = kRowThreads / 64;

template <int D>
__device__ __forceinline__ constexpr int v_chunk(int row, int chunk) {
  return D == 128 ? chunk ^ (row >> 1 & 7) : chunk ^ (row >> 2 & 3);
}

template <int D, int NB, bool kPartial>
__global__ void __launch_bounds__(kRowThreads) cache_rows_kernel(RowArgs a) {
  constexpr int kKK = D / 32;                     // MFMA steps over the channels
  constexpr int kCB = D / 16;                     // 16-channel blocks of O
  constexpr int kVLoads = kPage * D / 1024;       // 16-byte loads of V per lane and page
  constexpr int kKLoads = D / 64;                 // and of K per 16 keys
  constexpr int kVBytes = kPage * D;
  constexpr int kObuf = kRowWaves * 16 * D * 4;
  constexpr int kLds = kRowWaves * kVBytes > kObuf ? kRowWaves * kVBytes : kObuf;
  __shared__ __attribute__((aligned(16))) char smem[kLds];
  __shared__ float ml[2][kRowWaves][16];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i16 = lane & 15, g = lane >> 4;
  const int H = a.pool.H, G = a.G;
  // consecutive workgroups: the page ranges of a tile, then the tiles of a head
  int b = blockIdx.x;
  const int split = b % a.n_split;
  b /= a.n_split;
  const int tile = b % a.tiles;
  b /= a.tiles;
  const int h = b % H, s = b / H;
  const Session se = session_of(a.ss, s);
  const int rows = se.rows * G, row0 = tile * 16 * NB;
  if (!se.ok || row0 >= rows) return;
  const int pages = (se.len + kPage - 1) / kPage;
  const int per = (pages + a.n_split - 1) / a.n_split;
  const int begin = split * per, end = min(pages, begin + per);
  const int32_t* const table = a.ss.table + (int64_t)s * a.ss.width;

  bf16x8 qf[NB][kKK];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const int r = row0 + 16 * n + i16;
    const __bf16* const src = a.q + row_of(se, min(r, rows - 1), h, H, G) * D + D / 4 * g;
#pragma unroll
    for (int kk = 0; kk < kKK; ++kk)
      qf[n][kk] = __builtin_bit_cast(bf16x8, *(const u32x4*)(src + 8 * kk) ^ u32x4{a.flip, a.flip, a.flip, a.flip});
  }
  f32x4 o[NB][kCB] = {};
  float m[NB], l[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) m[n] = -INFINITY, l[n] = 0.0f;

  u32x4 kx[4][kKLoads], vx[kVLoads];
  float ks = 0.0f, vs = 0.0f;
  auto load = [&](int p) {
    const int page = table[p];
    const bool bad = (unsigned)page >= (unsigned)a.pool.pages;
    const int64_t ph = page_offset(page, bad, H, h, 1);
    const uint8_t* const k = a.pool.k + ph * kVBytes;
    const uint8_t* const v = a.pool.v + ph * kVBytes;
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
#pragma unroll
      for (int x = 0; x < kKLoads; ++x)
        kx[kb][x] = *(const u32x4*)(k + (16 * kb + i16) * D + D / 4 * g + 16 * x);
#pragma unroll
    for (int x = 0; x < kVLoads; ++x) vx[x] = *(const u32x4*)(v + 1024 * x + 16 * lane);
    ks = scale_of(a.pool.k_exp[ph], bad);
    vs = scale_of(a.pool.v_exp[ph], bad);
  };
  lds_char* const vbuf = (lds_char*)smem + wave * kVBytes;
  int p = begin + wave;
  if (p < end) load(p);
  for (; p < end; p += kRowWaves) {
    const int valid = se.len - p * kPage;  // keys of this page (64 or more: all)
    // V to LDS; its rows past the session's end as zeros, which meet weights of zero
#pragma unroll
    for (int x = 0; x < kVLoads; ++x) {
      const int row = (64 * x + lane) / (D / 16), chunk = lane % (D / 16);
      u32x4 y = vx[x];
      if (row >= valid) y = u32x4{};
      *(lds_u32x4*)(vbuf + row * D + v_chunk<D>(row, chunk) * 16) = y;
    }
    const float v_scale = vs;
    f32x4 sc[NB][4] = {};
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
#pragma unroll
      for (int kk = 0; kk < kKK; ++kk) {
        const bf16x8 kf = widen8(kx[kb][kk / 2][2 * (kk & 1)], kx[kb][kk / 2][2 * (kk & 1) + 1], ks);
#pragma unroll
        for (int n = 0; n < NB; ++n) sc[n][kb] = mfma16(kf, qf[n][kk], sc[n][kb]);
      }
    if (p + kRowWaves < end) load(p + kRowWaves);
    bf16x8 pf[NB][2];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      float mt = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (16 * kb + 4 * g + r < valid) mt = fmaxf(mt, sc[n][kb][r]);
      mt = fmaxf(mt, __shfl_xor(mt, 16));
      mt = fmaxf(mt, __shfl_xor(mt, 32));
      // scores that are all NaN leave the maximum as it is; their weights are NaN
      const float m_new = fmaxf(m[n], mt * a.c);
      const float alpha = m[n] == m_new ? 1.0f : __builtin_amdgcn_exp2f(m[n] - m_new);
      m[n] = m_new;
      float sum = 0.0f;
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          float w = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][kb][r], a.c, -m_new));
          if (16 * kb + 4 * g + r >= valid) w = 0.0f;
          sum += w;
          // the weights enter the product in 16 bits (its operands' type), the row sum in 32
          pf[n][kb / 2][4 * (kb & 1) + r] = (__bf16)w;
        }
      l[n] = l[n] * alpha + sum;
#pragma unroll
      for (int cb = 0; cb < kCB; ++cb) o[n][cb] *= alpha;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int cb = 0; cb < kCB; ++cb) {
        // lane 2 R + c of 16 addresses bytes 8 c of key row R; it gets channel lane & 15 of the 8 rows:
        // keys 4 g + 0..3 of the step's first 16, then of its second
        const int R = i16 >> 1;
        const int row = 32 * u + (R & 4) * 4 + 4 * g + (R & 3);
        const i32x2 x = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
            (lds_i32x2*)(vbuf + row * D + v_chunk<D>(row, cb) * 16 + 8 * (i16 & 1)));
        const bf16x8 vf = widen8((unsigned)x[0], (unsigned)x[1], v_scale);
#pragma unroll
        for (int n = 0; n < NB; ++n) o[n][cb] = mfma16(vf, pf[n][u], o[n][cb]);
      }
  }

  // join the waves: O = sum_w 2^(m_w - M) O_w / sum_w 2^(m_w - M) l_w
  float* const obuf = (float*)smem;
  constexpr int kCh = D / 16;  // channels of a thread
  const int orow = tid / 16, och = tid % 16 * kCh;
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    float ln = l[n];
    ln += __shfl_xor(ln, 16);
    ln += __shfl_xor(ln, 32);
    __syncthreads();
#pragma unroll
    for (int cb = 0; cb < kCB; ++cb) *(f32x4*)(obuf + (wave * 16 + i16) * D + 16 * cb + 4 * g) = o[n][cb];
    if (g == 0) ml[0][wave][i16] = m[n], ml[1][wave][i16] = ln;
    __syncthreads();
    const int r = row0 + 16 * n + orow;
    if (r >= rows) continue;
    float big = -INFINITY, sum = 0.0f, acc[kCh] = {};
#pragma unroll
    for (int w = 0; w < kRowWaves; ++w) big = fmaxf(big, ml[0][w][orow]);
#pragma unroll
    for (int w = 0; w < kRowWaves; ++w) {
      const float mw = ml[0][w][orow], lw = ml[1][w][orow];
      if (lw == 0.0f) continue;  // no keys
      const float f = mw == big ? 1.0f : __builtin_amdgcn_exp2f(mw - big);
      sum += f * lw;
#pragma unroll
      for (int x = 0; x < kCh; ++x) acc[x] += f * obuf[(w * 16 + orow) * D + och + x];
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    const float lse = sum == 0.0f ? -INFINITY : (big + log2f(sum)) * kLn2;
    const int64_t at = row_of(se, r, h, H, G);
    if constexpr (kPartial) {
      const int64_t part = (int64_t)split * a.ss.total * (H * G) + at;
      if (sum != 0.0f)
#pragma unroll
        for (int x = 0; x < kCh; x += 4)
          *(f32x4*)(a.part_o + part * D + och + x) = f32x4{acc[x] * inv, acc[x + 1] * inv, acc[x + 2] * inv, acc[x + 3] * inv};
      if (och == 0) a.part_lse[part] = lse;
    } else {
#pragma unroll
      for (int x = 0; x < kCh; x += 4)
        *(bf16x4*)(a.o + at * D + och + x) =
            bf16x4{(__bf16)(acc[x] * inv), (__bf16)(acc[x + 1] * inv), (__bf16)(acc[x + 2] * inv), (__bf16)(acc[x + 3] * inv)};
      if (a.lse != nullptr && och == 0) a.lse[at] = lse;
    }
  }
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
  const unsigned grid =
      (unsigned)(attn_items(a.ss.nseq, a.ss.max_rows, a.ss.total, a.pool.H, a.G, tile) * a.n_split);
  if (tile == kTileRows) launch_tiles(r, D, grid, a.cus, st);
  else if (a.n_split > 1) launch_rows<D, true>(r, tile, grid, st);
  else launch_rows<D, false>(r, tile, grid, st);
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
