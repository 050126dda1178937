// cache_weigh.hip -- the weight that queries give to each token of the session cache.
//
// For cached token j of head h, over the query rows r of its session (tokens x the G query heads of h):
//   weight[j,h] += sum_r exp(scale <Q_r, K_j> - lse_r),
// the column sums of the attention's softmax, whose row statistics (lse) are known.  Half the products of
// attention and as many exponentials: per 64 keys x 32 rows a wave has 16 32x32x16 MFMAs (512 clocks at d = 128) and
// 32 exponentials a lane with their multiply-adds and sums (768 clocks), which bound it.
//
// S^T = K Q^T (lane: row lane & 31, keys in the accumulator), with the keys as MFMA operands in registers, widened
// once: the rows' lse is one number a lane, and a key's sum over the rows grows in a register and is joined across
// the lanes at the end.  Rows arrive by LDS DMA.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn_tile.h"
#include "cache_device.h"
#include "cache_launch.h"
#include "cache_rows.h"

namespace tscache {

// 16-byte chunk c of a staged row r lies at chunk position c ^ row_swz(r): 16 rows' reads fall on distinct banks.
template <int D>
__device__ __forceinline__ constexpr int row_swz(int r) {
  return D == 128 ? r & 15 : (r >> 1) & 7;
}

// Sums of 32 values over 32 lanes (both halves of the wave by themselves): lane i gets the sum of x[i], halving the
// values with the lanes.
__device__ __forceinline__ float sum_over_lanes(float (&x)[32], int lane) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    // lanes 16..31 of x[i] against lanes 0..15 of x[i + 16]
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x[i]), __float_as_uint(x[i + 16]), false, false);
    x[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
#pragma unroll
  for (int m = 8; m > 0; m >>= 1)
#pragma unroll
    for (int i = 0; i < m; ++i) {
      const bool up = (lane & m) != 0;
      const float a = x[i], b = x[i + m];  // (values: a conditional of the elements themselves indexes registers)
      x[i] = (up ? b : a) + __shfl_xor(up ? a : b, m);
    }
  return x[0];
}

// The query rows of (session, head): DMA of staged rows, and the rows' lse.
struct Rows {
  __amdgpu_buffer_rsrc_t q, lse;
  int n, G, token_bytes, token_lse;

  __device__ __forceinline__ Rows(const Session& se, const __bf16* qp, const float* lp, int h, int H, int G, int D) : G(G) {
    n = __builtin_amdgcn_readfirstlane(se.rows * G);
    token_bytes = H * G * D * 2, token_lse = H * G * 4;
    const int last = max(n - 1, 0), t = __builtin_amdgcn_readfirstlane(last / G);
    const int64_t first = (int64_t)se.q0 * (H * G) + h * G;
    q = make_rsrc(qp + first * D, n > 0 ? (uint32_t)t * (uint32_t)token_bytes + (uint32_t)(last - t * G + 1) * (D * 2) : 0u);
    lse = make_rsrc(lp + first, n > 0 ? (uint32_t)t * (uint32_t)token_lse + (uint32_t)(last - t * G + 1) * 4 : 0u);
  }
  // Where row `row` of a stage of `stage` rows lies, in units of `token` for its token and `head` for its query head, and
  // `first`, that of stage 0, moved to stage t: where the group divides the stage, a stage is a whole number of tokens.
  __device__ __forceinline__ int place(int row, int token, int head) const {
    const int tok = row / G;
    return tok * token + (row - tok * G) * head;
  }
  __device__ __forceinline__ int place(int first, int t, int stage, int row, int token, int head) const {
    return stage % G == 0 ? first + t * (stage / G) * token : place(stage * t + row, token, head);
  }
  // the lse of a row as it is, and in log2 units, infinite (a weight of zero) past the end
  __device__ __forceinline__ float load_lse(int offset) const {
    return __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(lse, offset, 0, 0));
  }
  __device__ __forceinline__ float lse_of(float x, int t, int stage, int row) const {
    return stage * t + row < n ? x * kLog2e : INFINITY;
  }
};

// A page's keys as MFMA operands: (kb, kk) has key 32 kb + (lane & 31), channels D / 2 * (lane >> 5) + 8 kk .. + 7.  The sign
// bits in `flip` are inverted for a negative scale.
template <int D>
struct PageKeys {
  bf16x8 f[2][D / 16];

  __device__ __forceinline__ void set(const u32x4 (&raw)[2][D / 32], float scale, unsigned flip) {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int x = 0; x < D / 32; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y)
          f[kb][2 * x + y] = __builtin_bit_cast(
              bf16x8, __builtin_bit_cast(u32x4, widen8(raw[kb][x][2 * y], raw[kb][x][2 * y + 1], scale)) ^ u32x4{flip, flip, flip, flip});
  }
};

template <int D>
__device__ __forceinline__ void load_keys(u32x4 (&raw)[2][D / 32], const uint8_t* page, int lane) {
#pragma unroll
  for (int kb = 0; kb < 2; ++kb)
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
      raw[kb][x] = *(const u32x4*)(page + (32 * kb + (lane & 31)) * D + D / 2 * (lane >> 5) + 16 * x);
}

// Operand kk of a staged row is chunk D / 16 * (lane >> 5) + kk, at a position that differs from operand 0's by kk's
// bits: an address and an XOR.
template <int D>
__device__ __forceinline__ int row_at(int row, int lane) {
  return row * (D * 2) + ((D / 16 * (lane >> 5) ^ row_swz<D>(row)) << 4);
}
__device__ __forceinline__ bf16x8 row_operand(int at, int kk) {
  return *(const lds_bf16x8*)(uintptr_t)(unsigned)(at ^ kk << 4);
}

// Key of the page whose sum sum_over_lanes leaves in this lane: accumulator register i = lane & 31 is block i / 16, key
// 8 (i % 16 / 4) + 4 (lane >> 5) + i % 4 of it.
__device__ __forceinline__ int key_of_lane(int lane) {
  const int i = lane & 31;
  return 32 * (i >> 4) + 8 * ((i & 15) >> 2) + 4 * (lane >> 5) + (i & 3);
}

// ---- many keys.  A workgroup of four waves, one page each, walks over the rows, 64 at a time; two workgroups share a CU.
// A wave forms the weights of 32 rows while its MFMAs form the products of the next 32: between every two MFMAs two
// scores are weighed, and an operand is read again, for the rows after the next, when its second MFMA has it.  1560 rows x
// 32760 keys x 12 heads, d = 128: 153 us (1.03 PFLOP/s), against 177 us for two waves that take turns at a SIMD, one with
// its MFMAs and the other with its weights (the attention kernels' schedule): without the sums of a second product to
// form, a lone wave's exponentials take longer than the MFMAs they are to hide, and two waves fill each other's gaps.
//
// In iteration g (rows 64 g .. + 63 are weighed) the operands come from stage g + 1, fetched in iteration g - 1 and waited for
// at its end, and stage g + 2 is fetched over stage g - 1, whose operands iteration g - 1 has used.
template <int D>
struct WeighGeo {
  static constexpr int kThreads = 256;
  static constexpr int kRows = 64;                        // of a stage
  static constexpr int kStage = kRows * D * 2;
  static constexpr int kDma = kStage / 1024 / 4;          // DMA instructions per wave and stage
  static constexpr int kStages = 3;
};

template <int D>
__global__ void __launch_bounds__(WeighGeo<D>::kThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
cache_weigh_kernel(Pool pool, Sessions ss, const __bf16* __restrict__ q, const float* __restrict__ lse,
                   float* __restrict__ out, int G, int share, float c, unsigned flip) {
  using W = WeighGeo<D>;
  constexpr int kKK = D / 16;
  __shared__ __attribute__((aligned(1024))) char smem[W::kStages * W::kStage];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // An XCD (workgroup b runs on XCD b % 8) takes a consecutive eighth of each session's items, so that its L2 holds
  // the queries of the few heads that it works on; `share` workgroups of each XCD to a session.
  const int xcd = blockIdx.x & 7, s = (int)(blockIdx.x >> 3) / share, at = (int)(blockIdx.x >> 3) % share;
  const Session se = session_of(ss, s);
  if (!se.ok || se.len == 0) return;
  const int groups = (se.len + 4 * kPage - 1) / (4 * kPage);
  const int per_xcd = (pool.H * groups + 7) / 8, item = xcd * per_xcd + at;
  if (at >= per_xcd || item >= pool.H * groups) return;
  const int h = __builtin_amdgcn_readfirstlane(item / groups);
  const int p = __builtin_amdgcn_readfirstlane((item - h * groups) * 4 + wave);
  const int32_t* const table = ss.table + (int64_t)s * ss.width;
  const int number = p * kPage < se.len ? table[p] : -1;
  const int page = __builtin_amdgcn_readfirstlane((unsigned)number < (unsigned)pool.pages ? number : -1);
  const int64_t ph = (int64_t)max(page, 0) * pool.H + h;
  const Rows rows(se, q, lse, h, pool.H, G, D);
  const int stages = (rows.n + W::kRows - 1) / W::kRows;
  lds_char* const lds = (lds_char*)smem;

  int row_of[W::kDma], chunk[W::kDma], first[W::kDma];  // of the lane's 16-byte chunks of a stage
#pragma unroll
  for (int n = 0; n < W::kDma; ++n) {
    const int i = (4 * n + wave) * 64 + lane;
    row_of[n] = i / (D / 8);
    chunk[n] = (i % (D / 8) ^ row_swz<D>(row_of[n])) * 16;
    first[n] = rows.place(row_of[n], rows.token_bytes, D * 2);
    __asm__ volatile("" : "+v"(first[n]), "+v"(chunk[n]));  // (not formed again for every stage)
  }
  auto fetch = [&](int slot, int t) {
#pragma unroll
    for (int n = 0; n < W::kDma; ++n)
      dma16(rows.q, lds + slot * W::kStage + (4 * n + wave) * 1024,
            rows.place(first[n], t, W::kRows, row_of[n], rows.token_bytes, D * 2) + chunk[n]);
  };
  const int my_row = lane & 31;
  int first_lse[2] = {rows.place(my_row, rows.token_lse, 4), rows.place(32 + my_row, rows.token_lse, 4)};
  __asm__ volatile("" : "+v"(first_lse[0]), "+v"(first_lse[1]));
  auto load_lse = [&](int t, int half) {
    return rows.load_lse(rows.place(first_lse[half], t, W::kRows, 32 * half + my_row, rows.token_lse, 4));
  };
  const int at0 = (int)(uintptr_t)lds + row_at<D>(my_row, lane);  // of rows 32 .. 63: 32 rows on

  fetch(0, 0);
  fetch(1, 1);
  u32x4 raw[2][D / 32];
  load_keys<D>(raw, pool.k + ph * (kPage * D), lane);
  float next_lse[2] = {load_lse(0, 0), load_lse(0, 1)};
  PageKeys<D> keys;
  keys.set(raw, scale_of(pool.k_exp[ph], false), flip);
  wait_vmem<0>();
  block_sync();

  float acc[32] = {};
  bf16x8 qf[kKK];
  f32x16 x[2], y[2];
#pragma unroll
  for (int kk = 0; kk < kKK; ++kk) qf[kk] = row_operand(at0, kk);
  x[0] = x[1] = f32x16{};
#pragma unroll
  for (int kk = 0; kk < kKK; ++kk) {
    x[0] = mfma32(keys.f[0][kk], qf[kk], x[0]);
    x[1] = mfma32(keys.f[1][kk], qf[kk], x[1]);
  }
#pragma unroll
  for (int kk = 0; kk < kKK; ++kk) qf[kk] = row_operand(at0 + 32 * D * 2, kk);

  // weighs the scores `now` of rows with -lse `ls`, forms those of the next rows, and reads the operands at `from` for
  // the ones after
  auto step = [&](f32x16 (&now)[2], f32x16 (&next)[2], float ls, int from) {
    next[0] = next[1] = f32x16{};
#pragma unroll
    for (int kk = 0; kk < kKK; ++kk) {
      next[0] = mfma32(keys.f[0][kk], qf[kk], next[0]);
      next[1] = mfma32(keys.f[1][kk], qf[kk], next[1]);
      qf[kk] = row_operand(from, kk);
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) acc[i] += __builtin_amdgcn_exp2f(__builtin_fmaf(now[i >> 4][i & 15], c, ls));
#pragma unroll
    for (int i = 0; i < 2 * kKK; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);             // an MFMA
      if (i & 1) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);  // a read
      __builtin_amdgcn_sched_group_barrier(0x402, 48 / kKK, 0);      // the weighing of 32 / (2 kKK) scores
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) __asm__ volatile("" : "+v"(acc[i]));  // here, not where the sums are used next
  };
  int slot = 0;
  for (int g = 0; g < stages; ++g) {
    const int s1 = slot == W::kStages - 1 ? 0 : slot + 1, s2 = s1 == W::kStages - 1 ? 0 : s1 + 1;
    const float ls[2] = {-rows.lse_of(next_lse[0], g, W::kRows, my_row), -rows.lse_of(next_lse[1], g, W::kRows, 32 + my_row)};
    fetch(s2, g + 2);  // (past the last row, zeros that nobody reads)
    next_lse[0] = load_lse(g + 1, 0);
    next_lse[1] = load_lse(g + 1, 1);
    step(x, y, ls[0], at0 + s1 * W::kStage);
    step(y, x, ls[1], at0 + s1 * W::kStage + 32 * D * 2);
    wait_vmem<0>();
    block_sync();
    slot = s1;
  }
  const float sum = sum_over_lanes(acc, lane);
  const int key = key_of_lane(lane);
  if (page >= 0 && p * kPage + key < se.len) out[ph * kPage + key] = pool.weight[ph * kPage + key] + sum;
}

// ---- few keys: one page to a workgroup of four waves, which take 32 rows each of a stage of 128.
template <int D>
struct FewGeo {
  static constexpr int kThreads = 256;
  static constexpr int kRows = 128;
  static constexpr int kStage = kRows * D * 2;
  static constexpr int kDma = kStage / 1024 / 4;
  static constexpr int kSums = 2 * kStage;                // each wave's sums of the page
  static constexpr int kLds = kSums + 4 * kPage * 4;
};

template <int D>
__global__ void __launch_bounds__(FewGeo<D>::kThreads) __attribute__((amdgpu_waves_per_eu(1, 2)))
cache_weigh_few_kernel(Pool pool, Sessions ss, const __bf16* __restrict__ q, const float* __restrict__ lse,
                       float* __restrict__ out, int G, int slots, float c, unsigned flip) {
  using W = FewGeo<D>;
  constexpr int kKK = D / 16;
  __shared__ __attribute__((aligned(1024))) char smem[W::kLds];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int p = (int)blockIdx.x % slots, sh = (int)blockIdx.x / slots, h = sh % pool.H, s = sh / pool.H;
  const Session se = session_of(ss, s);
  if (!se.ok || p * kPage >= se.len) return;
  const int page = ss.table[(int64_t)s * ss.width + p];
  if ((unsigned)page >= (unsigned)pool.pages) return;
  const int64_t ph = (int64_t)page * pool.H + h;
  const Rows rows(se, q, lse, h, pool.H, G, D);
  const int stages = (rows.n + W::kRows - 1) / W::kRows;
  lds_char* const lds = (lds_char*)smem;  // (one object: the compiler has reads of a second one wait for all DMA in flight)
  float* const sums = (float*)(smem + W::kSums);
  auto fetch = [&](int t) {
#pragma unroll
    for (int n = 0; n < W::kDma; ++n) {
      const int i = (4 * n + wave) * 64 + lane;  // 16-byte chunk of the stage
      const int row = i / (D / 8), chunk = i % (D / 8) ^ row_swz<D>(row);
      dma16(rows.q, lds + (t & 1) * W::kStage + (4 * n + wave) * 1024,
            rows.place(W::kRows * t + row, rows.token_bytes, D * 2) + chunk * 16);
    }
  };
  fetch(0);
  u32x4 raw[2][D / 32];
  load_keys<D>(raw, pool.k + ph * (kPage * D), lane);
  PageKeys<D> keys;
  keys.set(raw, scale_of(pool.k_exp[ph], false), flip);
  const int row = 32 * wave + (lane & 31), at0 = (int)(uintptr_t)lds + row_at<D>(row, lane);
  float acc[32] = {};
  for (int t = 0; t < stages; ++t) {
    const float ls = rows.lse_of(rows.load_lse(rows.place(W::kRows * t + row, rows.token_lse, 4)), t, W::kRows, row);
    wait_vmem<0>();
    block_sync();  // stage t is there, and every wave is done with stage t - 1
    if (t + 1 < stages) fetch(t + 1);
    f32x16 x[2] = {};
#pragma unroll
    for (int kk = 0; kk < kKK; ++kk) {
      const bf16x8 qf = row_operand(at0 + (t & 1) * W::kStage, kk);
      x[0] = mfma32(keys.f[0][kk], qf, x[0]);
      x[1] = mfma32(keys.f[1][kk], qf, x[1]);
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) acc[i] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[i >> 4][i & 15], c, -ls));
    wait_lds();
  }
  sums[wave * kPage + key_of_lane(lane)] = sum_over_lanes(acc, lane);
  __syncthreads();
  if (wave != 0 || p * kPage + lane >= se.len) return;
  const int64_t to = ph * kPage + lane;
  out[to] = pool.weight[to] + ((sums[lane] + sums[kPage + lane]) + (sums[2 * kPage + lane] + sums[3 * kPage + lane]));
}

// ---- few rows (up to 16 NB of a cached head, a token or two of each session): bound by reading the keys.  A wave walks
// over pages of one (session, head), first, first + step, ...; S^T = K Q^T on 16x16x32 MFMAs with the keys straight from memory (as
// rows_item has them: lane: row lane & 15, keys 4 (lane >> 4) + 0..3 of each 16), the next page asked for a step ahead.
// 32 single tokens over 16384 keys x 8 heads take 116 us at d = 128 (4.6 TB/s) and 50 at d = 64, and 251 and 147 by the
// kernel for many keys; 32 times 64 rows 130 and 81 instead of 238 and 149.
template <int D, int NB>
__global__ void __launch_bounds__(256) cache_weigh_rows_kernel(Pool pool, Sessions ss, const __bf16* __restrict__ q,
                                                               const float* __restrict__ lse, float* __restrict__ out, int G,
                                                               int split, float c, unsigned flip) {
  constexpr int kKK = D / 32, kKLoads = D / 64, kW = 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i16 = lane & 15, g = lane >> 4, H = pool.H;
  const int b = blockIdx.x, sh = b / split, h = sh % H, s = sh / H;
  const PageRange range{b % split, split, 0};
  const int32_t* const table = ss.table + (int64_t)s * ss.width;
  int id = first_ids<kW>(table, ss.width, range.first, split);
  const Session se = session_of(ss, s);
  if (!se.ok) return;
  const int rows = se.rows * G, len = __builtin_amdgcn_readfirstlane(se.len);
  const int left = (len + kPage - 1) / kPage - range.page(wave), apart = kW * split;
  const int mine = left > 0 ? (left + apart - 1) / apart : 0;
  if (mine == 0) return;

  struct Page {
    u32x4 k[4][kKLoads];
    float weight;
  };
  int i0 = 0, now = min(mine, 64), kexp = 0;
  unsigned long long good = 0;  // of the lanes' pages, those in the pool
  auto exponents = [&] {
    const bool ok = (unsigned)id < (unsigned)pool.pages;
    good = __builtin_amdgcn_ballot_w64(ok && lane < now);
    id = ok ? id : 0;
    kexp = pool.k_exp[(int64_t)id * H + h];
  };
  auto load = [&](int i, Page& p) {  // page i0 + i of the wave; past the last of them, one of the pool's
    const int64_t ph = (int64_t)__builtin_amdgcn_readlane(id, i & 63) * H + h;
    const uint8_t* const from = pool.k + ph * (kPage * D) + i16 * D + D / 4 * g;
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
#pragma unroll
      for (int x = 0; x < kKLoads; ++x) p.k[kb][x] = *(const u32x4*)(from + 16 * kb * D + 16 * x);
    p.weight = pool.weight[ph * kPage + lane];
  };
  exponents();
  u32x4 qraw[NB][kKK];
  float ls[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const int r = 16 * n + i16;
    const int64_t at = row_of(se, r, h, H, G);
#pragma unroll
    for (int kk = 0; kk < kKK; ++kk) qraw[n][kk] = u32x4{};  // rows past the last one: zeros, with weights of zero
    ls[n] = INFINITY;
    if (r < rows) {
#pragma unroll
      for (int kk = 0; kk < kKK; ++kk) qraw[n][kk] = *(const u32x4*)(q + at * D + D / 4 * g + 8 * kk);
      ls[n] = lse[at];
    }
  }
  Page p0, p1;
  load(0, p0);
  bf16x8 qf[NB][kKK];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
#pragma unroll
    for (int kk = 0; kk < kKK; ++kk) qf[n][kk] = __builtin_bit_cast(bf16x8, qraw[n][kk] ^ u32x4{flip, flip, flip, flip});
    ls[n] *= kLog2e;
  }
  auto page = [&](int i, Page& p, Page& next) {
    load(i + 1, next);
    __builtin_amdgcn_sched_barrier(0);  // the products stay behind those loads
    const float ks = __uint_as_float((unsigned)__builtin_amdgcn_readlane(kexp, i) << 23);
    f32x4 sc[NB][4] = {};
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
#pragma unroll
      for (int kk = 0; kk < kKK; ++kk) {
        const bf16x8 kf = widen8(p.k[kb][kk / 2][2 * (kk & 1)], p.k[kb][kk / 2][2 * (kk & 1) + 1], ks);
#pragma unroll
        for (int n = 0; n < NB; ++n) sc[n][kb] = mfma16(kf, qf[n][kk], sc[n][kb]);
      }
    float x[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      x[j] = 0.0f;
#pragma unroll
      for (int n = 0; n < NB; ++n) x[j] += __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][j >> 2][j & 3], c, -ls[n]));
    }
#pragma unroll
    for (int m = 8; m > 0; m >>= 1)
#pragma unroll
      for (int j = 0; j < m; ++j) {
        const bool up = (lane & m) != 0;
        const float lo = x[j], hi = x[j + m];
        x[j] = (up ? hi : lo) + __shfl_xor(up ? lo : hi, m);
      }
    // lane 16 g + i has the sum of key 16 (i / 4) + 4 g + i % 4; from there to the lane that has this key's weight
    const float sum = __shfl(x[0], (lane >> 2 & 3) * 16 + (lane >> 4) * 4 + (lane & 3));
    const int at = range.page(wave + kW * (i0 + i)) * kPage;
    if ((good >> i & 1) && at + lane < len)  // (without rows, weights as they were, those of NaN keys too)
      out[((int64_t)__builtin_amdgcn_readlane(id, i) * H + h) * kPage + lane] = rows > 0 ? p.weight + sum : p.weight;
  };
  for (; i0 < mine; i0 += 64) {
    if (i0 > 0) {
      now = min(mine - i0, 64);
      id = lane < now ? table[range.page(wave + kW * (i0 + lane))] : -1;
      exponents();
      load(0, p0);
    }
    for (int i = 0; i < now; i += 2) {
      page(i, p0, p1);
      if (i + 1 < now) page(i + 1, p1, p0);
    }
  }
}

// ---------------------------------------------------------------------------------------------
// host-side launcher

hipError_t launch_weigh(const WeighArgs& a, hipStream_t st) {
  const float c = log2_scale(a.scale);
  const unsigned flip = a.scale < 0.0f ? 0x80008000u : 0u;
  if (const int split = weigh_rows(a.ss.nseq, a.ss.max_rows, a.ss.max_len, a.pool.H, a.G, a.cus)) {
    const int64_t rows = (int64_t)a.ss.max_rows * a.G;
    auto kern = a.d == 64 ? (rows <= 16   ? cache_weigh_rows_kernel<64, 1>
                             : rows <= 32 ? cache_weigh_rows_kernel<64, 2>
                                          : cache_weigh_rows_kernel<64, 4>)
                          : (rows <= 16   ? cache_weigh_rows_kernel<128, 1>
                             : rows <= 32 ? cache_weigh_rows_kernel<128, 2>
                                          : cache_weigh_rows_kernel<128, 4>);
    hipLaunchKernelGGL(kern, dim3((unsigned)(a.ss.nseq * a.pool.H * split)), dim3(256), 0, st, a.pool, a.ss, (const __bf16*)a.q,
                       a.lse, a.out, a.G, split, c, flip);
    return hipGetLastError();
  }
  if (weigh_few(a.ss.nseq, a.ss.max_len, a.pool.H, a.cus)) {
    const int slots = (a.ss.max_len + kPage - 1) / kPage;
    auto kern = a.d == 64 ? cache_weigh_few_kernel<64> : cache_weigh_few_kernel<128>;
    hipLaunchKernelGGL(kern, dim3((unsigned)(a.ss.nseq * a.pool.H * slots)), dim3(FewGeo<64>::kThreads), 0, st, a.pool, a.ss,
                       (const __bf16*)a.q, a.lse, a.out, a.G, slots, c, flip);
    return hipGetLastError();
  }
  const int64_t share = weigh_share(a.ss.max_len, a.pool.H);
  auto kern = a.d == 64 ? cache_weigh_kernel<64> : cache_weigh_kernel<128>;
  hipLaunchKernelGGL(kern, dim3((unsigned)(8 * a.ss.nseq * share)), dim3(WeighGeo<64>::kThreads), 0, st, a.pool, a.ss,
                     (const __bf16*)a.q, a.lse, a.out, a.G, (int)share, c, flip);
  return hipGetLastError();
}

}  // namespace tscache
