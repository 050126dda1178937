// attn_bwd.hip -- the gradients of packed attention (ts_attn_bwd): D and the scaled log-sum-exp of each row, then dq and
// dk, dv on the matrix cores.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>
#include <utility>

#include "attn_tile.h"
#include "block_launch.h"

namespace tsblock {

using namespace tsattn;

// The rows of one side are held in registers (dq: queries and d_o; dk, dv: keys and values), 32 by a wave, and those of
// the other stream through LDS, kBN of them at a time.  With X1, X2 the streamed pair (dq: k, v; dk, dv: q, d_o)
// and Y1, Y2 the held one, a wave computes for 32 streamed rows
//   S = X1 Y1^T,  T = X2 Y2^T - D       (32 x 32: streamed rows in registers, held ones over the lanes)
//   P = exp(scale S - lse),  R = P T
//   acc1^T += X1^T R   (dq or dk),      acc2^T += X2^T P   (dv)
// where P and R, as they lie, are the B operands of the last two products, whose A operands are transposed reads of
// the same LDS rows.  Where the streamed rows are queries, S and T start at their -lse / scale and -D, which come with them.
//
// R is rounded to bfloat16 once for dk, and for dq taken in two parts, R and what its rounding leaves, each times the keys from the
// same registers.  The R of a query sum to 0 but for D's rounding, so that dq loses what its keys have in common while
// an error of R does not: with one part dq is off by 0.0029 of its norm where the keys' mean is as large as their
// spread, by 0.013 where it is 8 times that, with two by 0.0017, its own rounding.  (Less the sum of R's errors times a mean
// of keys it would be 0.0024, 10 % sooner, but keys of no weight that lie far out, as masked ones do, then put it off by more
// than its norm, and with a mean that no such key can move the gain is gone where signs are mixed.)
//
// Both gradients of a score tile recompute S and T: eight products of a tile in all where six would do if dq were added up
// in memory across the key tiles.  Those sums would have to be atomic, in no fixed order, or wait for each other, and the scores
// would have to be laid out anew for them through LDS, which has no time to spare (a read of 1 KiB feeds one MFMA of a SIMD:
// 8 clocks of the LDS' 8).
//
// LDS layout of a streamed tile: rows in groups of four, so that both the row reads (b128: 16 rows, the same 16-byte
// chunk) and the transposed ones (b64: 4 rows x 64 bytes) fall on distinct banks, with offsets that are sums of a
// lane's own and an immediate.  At d = 128 the four rows are 320 bytes apart, at d = 64 at 0, 128, 320 and 448.  (No bank
// conflicts were counted in these reads.)
template <int D, int W>  // W waves to a workgroup
struct Bwd {
  static constexpr int kThreads = 64 * W;
  static constexpr int kTileRows = 32 * W;
  static constexpr int kBN = bwd_step(D, kTileRows);
  static constexpr int kGroup = D == 128 ? 1232 : 592;  // bytes of a group of four rows, 16 mod 64
  static constexpr int kTile = (kBN / 4 * kGroup + 1023) / 1024 * 1024;
  static constexpr int kDma = kTile / 1024;  // DMA instructions of a tile
  static constexpr int kDmaMax = (kDma + W - 1) / W, kDmaMin = kDma / W;  // of a wave
  static constexpr int kStat = 2 * kTile;  // the two statistics, after X1 and X2
  static constexpr int kStatRow = kBN < 64 ? 256 : kBN * 4;  // bytes of one: a DMA instruction fills 256
  static constexpr int kStatDma = kStatRow / 256;
  static constexpr int kStage = 2 * kTile + 2 * kStatRow;
  static constexpr int kStages = D == 64 ? 2 : 3;
  static constexpr int kLds = kStages * kStage;
  static_assert(bwd_groups(D, kTileRows) * kLds <= 160 * 1024, "LDS of a CU");
  static_assert(2 * kStatDma <= W, "a wave fetches one part of the statistics");
  __host__ __device__ static constexpr int row_offset(int r) {
    return (r >> 2) * kGroup + (D == 128 ? 320 * (r & 3) : 128 * (r & 1) + 320 * ((r >> 1) & 1));
  }
};

struct BwdCall {
  const __bf16* d_o;
  const __bf16* q;
  const __bf16* k;
  const __bf16* v;
  const float* stat;
  __bf16* dq;
  __bf16* dk;
  __bf16* dv;
  float* part_q;
  float* part_k;
  const BwdPlan* plan;
  int total_q, total_k, H, n_q, n_k;
  float scale, c;  // c: log2(e) times the scale, or log2(e) for a scale of 0
};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// An item of a call: which head, tile and range, of which segment's rows.
struct Item {
  int h, tile, split;
  int held0, held_len, str0, str_len;
};

// Item `at` of the list of entry t, of a side with n ranges.  Its head, range and tile go by the list's own order over the XCDs,
// so that each of them gets an equal part of every list, and neighbours on it stream the same rows.
__device__ __forceinline__ Item find_item(const BwdTile& t, int at, int heads, int n) {
  at = remap_block(at - t.first * heads, t.tiles * n * heads, 32);
  const int j = at / t.tiles;
  return Item{j / n, at - j * t.tiles, j % n, t.held0, t.held_len, t.str0, t.str_len};
}

typedef __attribute__((address_space(3))) f32x4 lds_f32x4;

// The LDS reads of a step take their address as a restrict pointer: the compiler then knows that they do not wait for the
// DMA of the steps ahead.

// A operand of a product with 32 rows of X1 or X2: 16 of their channels.
__device__ __forceinline__ bf16x8 rows_operand(const lds_char* __restrict__ x) { return *(const lds_bf16x8*)x; }

// A operand of a product with the columns of X1 or X2: 32 channels of 16 rows.
template <int kGroup>
__device__ __forceinline__ bf16x8 columns_operand(const lds_char* __restrict__ x) {
  const bf16x4 a0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)x);
  const bf16x4 a1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(x + 2 * kGroup));
  return bf16x8{a0[0], a0[1], a0[2], a0[3], a1[0], a1[1], a1[2], a1[3]};
}

// The statistics of a block's 32 queries, as the rows of an accumulator.
__device__ __forceinline__ f32x16 row_statistics(const lds_char* __restrict__ x, int hb) {
  f32x16 to;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const f32x4 y = *(const lds_f32x4*)(x + 32 * g + 16 * hb);
#pragma unroll
    for (int r = 0; r < 4; ++r) to[4 * g + r] = y[r];
  }
  return to;
}

// f(0), f(1) .. f(N - 1), each a constant of its type, for a loop that is too long to be unrolled by the compiler.
template <int... I, typename F>
__device__ __forceinline__ void for_each(std::integer_sequence<int, I...>, F&& f) { (f(std::integral_constant<int, I>{}), ...); }

__device__ __forceinline__ f32x16 splat(float x) { return f32x16{x, x, x, x, x, x, x, x, x, x, x, x, x, x, x, x}; }

// A wave's 32 rows of results leave through LDS, in pieces of 128 bytes a row: straight from the accumulators every
// store would touch 32 rows with 16 bytes each (six odd clips at d = 64 82 us instead of 75, 1560 x 32760 x 12 heads 1003 instead
// of 965).  Rows past the segment's end are dropped by the range check.
constexpr int kOutRow = 128 + 16;  // bytes
constexpr int kOutWave = 32 * kOutRow;

template <int D>
__device__ __forceinline__ void write_rows(const f32x16 (&acc)[D / 32], float f, __bf16* to, int row0, int len, int H, lds_char* out,
                                           int lane) {
  const int row_bytes = H * D * 2, hb = lane >> 5, r = lane >> 3, chunk = lane & 7;
  const __amdgpu_buffer_rsrc_t rsrc = make_rsrc(to, (uint32_t)(len - 1) * (uint32_t)row_bytes + D * 2);
  lds_char* const put = out + (lane & 31) * kOutRow + 8 * hb;
  const lds_char* const get = out + r * kOutRow + 16 * chunk;
  auto in_order = [] { __asm__ volatile("" ::: "memory"); };  // (the accesses of a wave are in order in the LDS)
#pragma unroll
  for (int d0 = 0; d0 < D / 32; d0 += 2) {
#pragma unroll
    for (int db = d0; db < d0 + 2; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 x = {acc[db][4 * g] * f, acc[db][4 * g + 1] * f, acc[db][4 * g + 2] * f, acc[db][4 * g + 3] * f};
        *(lds_u32x2*)(put + 64 * (db - d0) + 16 * g) = __builtin_bit_cast(u32x2, __builtin_convertvector(x, bf16x4));
      }
    in_order();
#pragma unroll
    for (int u = 0; u < 4; ++u)
      __builtin_amdgcn_raw_buffer_store_b128(*(const lds_u32x4*)(get + 8 * u * kOutRow), rsrc,
                                             (row0 + r + 8 * u) * row_bytes + 64 * d0 + 16 * chunk, 0, 0);
    in_order();
  }
}

// The same in 32 bits, of one range.
template <int D>
__device__ __forceinline__ void write_part(const f32x16 (&acc)[D / 32], float* to, int row0, int len, int H, lds_char* out, int lane) {
  // (offsets of up to twice those of 16-bit rows, unsigned)
  const uint32_t row_bytes = (uint32_t)(H * D) * 4u;
  const int hb = lane >> 5, r = lane >> 3, chunk = lane & 7;
  const __amdgpu_buffer_rsrc_t rsrc = make_rsrc(to, (uint32_t)(len - 1) * row_bytes + D * 4);
  lds_char* const put = out + (lane & 31) * kOutRow + 16 * hb;
  const lds_char* const get = out + r * kOutRow + 16 * chunk;
  auto in_order = [] { __asm__ volatile("" ::: "memory"); };
#pragma unroll
  for (int db = 0; db < D / 32; ++db) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 x = {acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]};
      *(lds_u32x4*)(put + 32 * g) = __builtin_bit_cast(u32x4, x);
    }
    in_order();
#pragma unroll
    for (int u = 0; u < 4; ++u)
      __builtin_amdgcn_raw_buffer_store_b128(*(const lds_u32x4*)(get + 8 * u * kOutRow), rsrc,
                                             __builtin_bit_cast(int, (uint32_t)(row0 + r + 8 * u) * row_bytes + 128u * db + 16u * chunk), 0, 0);
    in_order();
  }
}

// One item of the dq (kKeys = false) or the dk, dv side.
template <int D, int W, bool kKeys>
__device__ __forceinline__ void run_item(const BwdCall& a, const Item& w, lds_char* lds) {
  using G = Bwd<D, W>;
  constexpr int kBN = G::kBN;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int col = lane & 31, hb = lane >> 5;
  const int row_bytes = a.H * D * 2;
  const int held_len = w.held_len, len = w.str_len;  // rows of the segment
  const int64_t held0 = ((int64_t)w.held0 * a.H + w.h) * D, str0 = ((int64_t)w.str0 * a.H + w.h) * D;
  const int row0 = w.tile * G::kTileRows + 32 * wave;  // this wave's first held row

  // the range's steps; ranges are of 64 rows, whatever a step has, so that their sums do not go by the tile
  const int steps_all = (len + kBN - 1) / kBN, n = kKeys ? a.n_k : a.n_q, units = (len + 63) / 64;
  const int begin = (int)((int64_t)units * w.split / n) * (64 / kBN);
  const int end = min((int)((int64_t)units * (w.split + 1) / n) * (64 / kBN), steps_all);
  const int steps = end - begin;

  f32x16 acc1[D / 32], acc2[kKeys ? D / 32 : 1];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) acc1[i] = f32x16{};
#pragma unroll
  for (int i = 0; i < (kKeys ? D / 32 : 1); ++i) acc2[i] = f32x16{};

  int slot = 0;  // stage of the step to come
  if (steps > 0) {
    const uint32_t held_bytes = (uint32_t)(held_len - 1) * (uint32_t)row_bytes + D * 2;
    const uint32_t str_bytes = (uint32_t)(len - 1) * (uint32_t)row_bytes + D * 2;
    const __amdgpu_buffer_rsrc_t ry1 = make_rsrc((kKeys ? a.k : a.q) + held0, held_bytes);
    const __amdgpu_buffer_rsrc_t ry2 = make_rsrc((kKeys ? a.v : a.d_o) + held0, held_bytes);
    const __amdgpu_buffer_rsrc_t rx1 = make_rsrc((kKeys ? a.q : a.k) + str0, str_bytes);
    const __amdgpu_buffer_rsrc_t rx2 = make_rsrc((kKeys ? a.d_o : a.v) + str0, str_bytes);
    // the head's statistics of the segment's queries
    const float* const stat = a.stat + (int64_t)w.h * a.total_q + (kKeys ? w.str0 : w.held0);
    const uint32_t stat_bytes = (uint32_t)(kKeys ? len : held_len) * 4;
    const __amdgpu_buffer_rsrc_t ra = make_rsrc(stat, stat_bytes);
    const __amdgpu_buffer_rsrc_t rd = make_rsrc(stat + (int64_t)a.H * a.total_q, stat_bytes);

    // DMA: instruction i = wave + W u of a tile fills LDS bytes [1024 i, 1024 i + 1024), lane l 16 of them; lanes of the
    // pads fetch a row's first chunk again
    int off[G::kDmaMax];
#pragma unroll
    for (int u = 0; u < G::kDmaMax; ++u) {
      const int b = 1024 * (wave + W * u) + 16 * lane;
      const int g = b / G::kGroup, rem = b % G::kGroup;
      int r, byte;
      if (D == 128) {
        r = rem / 320;
        byte = rem - 320 * r;
      } else {
        const int half = rem / 320, in = rem - 320 * half;
        r = 2 * half + min(in / 128, 1);
        byte = in - 128 * (r & 1);
      }
      const int row = 4 * g + r;
      off[u] = (row < kBN ? row : 0) * row_bytes + (byte < D * 2 ? byte : 0);
    }
    // Rows past the segment's end read as zeros.  The fetches after the range's last step bring its first one again.
    auto fetch = [&](int j, lds_char* stage) {
      const int step = begin + (j < steps ? j : 0), skip = step * kBN * row_bytes;
#pragma unroll
      for (int u = 0; u < G::kDmaMax; ++u) {
        const int i = wave + W * u;
        if (u < G::kDmaMin || i < G::kDma) {
          __builtin_amdgcn_raw_ptr_buffer_load_lds(rx1, (lds_void*)(stage + 1024 * i), 16, off[u] + skip, 0, 0, 0);
          __builtin_amdgcn_raw_ptr_buffer_load_lds(rx2, (lds_void*)(stage + G::kTile + 1024 * i), 16, off[u] + skip, 0, 0, 0);
        }
      }
      if (kKeys && wave < 2 * G::kStatDma) {
        const int part = wave % G::kStatDma;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(wave < G::kStatDma ? ra : rd, (lds_void*)(stage + G::kStat + 256 * wave), 4,
                                                 (step * kBN + 64 * part + lane) * 4, 0, 0, 0);
      }
    };
#pragma unroll
    for (int j = 0; j < G::kStages - 1; ++j) fetch(j, lds + j * G::kStage);

    // held rows as B operands: row col, channels 16 kk + 8 hb + 0..7 (by way of LDS in whole lines, as the results, they come no
    // more than 1 % of a small call sooner)
    bf16x8 y1[D / 16], y2[D / 16];
    const bool zero = a.scale == 0.0f;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      const int at = (row0 + col) * row_bytes + kk * 32 + hb * 16;
      u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(ry1, at, 0, 0);
      y1[kk] = __builtin_bit_cast(bf16x8, zero ? u32x4{} : x);
      y2[kk] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(ry2, at, 0, 0));
    }
    float la = 0, ld = 0;  // dq: the lane's query's statistics
    if (!kKeys) {
      la = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(ra, (row0 + col) * 4, 0, 0)) * a.c;
      ld = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rd, (row0 + col) * 4, 0, 0));
    }

    const int row_lane = G::row_offset(col) + hb * 16;
    const int tr_lane = G::row_offset(4 * (lane >> 5) + ((lane & 15) >> 2)) + 32 * ((lane >> 4) & 1) + 16 * ((lane & 3) >> 1) + 8 * (lane & 1);
    const float c = a.c;
    const bool active = row0 < held_len;

    // One step.  The order of its products and reads is pinned: each operand is read a product before it is used (more ahead
    // measured the same), and the vector work on a product's result goes between products that do not wait for it.  Left to the
    // compiler's order 32760 x 32760 x 12 heads took 2 % longer, as 16380 x 16380 x 24 heads of d = 64 did (before R came in two
    // parts).  ragged: rows from `left` on are past the segment's end; their P and R are 0.
    constexpr int kM = D / 16;  // MFMAs of a product
    constexpr bool kPair = !kKeys && kBN >= 64;  // dq: two blocks at a time
    constexpr int kBlocks = kBN / (kPair ? 64 : 32), kPer = (kKeys ? 4 : kPair ? 6 : 3) * kM, kAll = kBlocks * kPer;
    auto step_of = [&](const lds_char* stage, auto ragged, int left) {
      const lds_char* const xr = stage + row_lane;
      const lds_char* const xt = stage + tr_lane;
      const lds_char* const st = stage + G::kStat;
      auto operand = [&](int i) {
        const int b = i / kPer, phase = i % kPer / kM, m = i % kM;
        const int column = 4 * (m / (D / 32)) * G::kGroup + 64 * (m % (D / 32));
        if (kKeys) {
          const int block = 8 * b * G::kGroup;
          if (phase < 2) return rows_operand(xr + block + phase * G::kTile + 32 * m);
          return columns_operand<G::kGroup>(xt + block + (phase == 2 ? G::kTile : 0) + column);
        }
        const int block = (8 * (kPair ? 2 : 1) * b + (kPair && (phase == 2 || phase == 3 || phase == 5) ? 8 : 0)) * G::kGroup;
        if (phase < (kPair ? 4 : 2)) return rows_operand(xr + block + (phase & 1) * G::kTile + 32 * m);
        return columns_operand<G::kGroup>(xt + block + column);
      };
      f32x16 s[kKeys ? 1 : 2], t[kKeys ? 1 : 2];
      bf16x8 p[2], ds[kKeys ? 1 : 2][2], dl[kKeys ? 1 : 2][2];
      auto weight = [&](int w, int r, int row) {  // s becomes P
        float x = s[w][r];
        x = __builtin_amdgcn_exp2f(kKeys ? x * c : __builtin_fmaf(x, c, la));
        if (decltype(ragged)::value && row + 8 * (r >> 2) + 4 * hb + (r & 3) >= left) x = 0.0f;
        s[w][r] = x;
        if (kKeys) p[r >> 3][r & 7] = (__bf16)x;
      };
      auto residual = [&](int w, int r, int row) {
        float x = s[w][r] * t[w][r];
        if (decltype(ragged)::value && row + 8 * (r >> 2) + 4 * hb + (r & 3) >= left) x = 0.0f;
        const __bf16 hi = (__bf16)x;
        ds[w][r >> 3][r & 7] = hi;
        // (P is 0 past the end; a fused operation in every kernel, so that all have the same bits)
        if (!kKeys) dl[w][r >> 3][r & 7] = (__bf16)__builtin_fmaf(s[w][r], t[w][r], -(float)hi);
      };
      // element range of slot m of a phase: nothing in the first, whose product waits for the result
      auto from = [](int m) { return m < 1 ? 0 : 2 * ((8 * (m - 1) + kM - 2) / (kM - 1)); };
      if (kKeys) {
        s[0] = row_statistics(st, hb);
        t[0] = row_statistics(st + G::kStatRow, hb);
      }
      bf16x8 next = operand(0);
      for_each(std::make_integer_sequence<int, kAll>{}, [&](auto at) __attribute__((always_inline)) {
        constexpr int i = at, b = i / kPer, phase = i % kPer / kM, m = i % kM;
        const bf16x8 x = next;
        if (i + 1 < kAll) next = operand(i + 1);
        if constexpr (kKeys) {
          if (phase == 0) s[0] = mfma32(x, y1[m], s[0]);
          else if (phase == 1) t[0] = mfma32(x, y2[m], t[0]);
          else if (phase == 2) acc2[m % (D / 32)] = mfma32(x, p[m / (D / 32)], acc2[m % (D / 32)]);
          else acc1[m % (D / 32)] = mfma32(x, ds[0][m / (D / 32)], acc1[m % (D / 32)]);
#pragma unroll
          for (int r = from(m); r < from(m + 1); ++r) {
            if (phase == 1) weight(0, r, 32 * b);
            if (phase == 2) residual(0, r, 32 * b);
          }
          if (phase == 3 && b + 1 < kBlocks) {
            if (m == 0) s[0] = row_statistics(st + 128 * (b + 1), hb);
            if (m == 1) t[0] = row_statistics(st + 128 * (b + 1) + G::kStatRow, hb);
          }
        } else {
          const int w = kPair && (phase == 2 || phase == 3 || phase == 5);
          if (phase == 0 || (kPair && phase == 2)) s[w] = mfma32(x, y1[m], m == 0 ? f32x16{} : s[w]);
          else if (phase == 1 || (kPair && phase == 3)) t[w] = mfma32(x, y2[m], m == 0 ? splat(ld) : t[w]);
          else {
            acc1[m % (D / 32)] = mfma32(x, ds[w][m / (D / 32)], acc1[m % (D / 32)]);
            acc1[m % (D / 32)] = mfma32(x, dl[w][m / (D / 32)], acc1[m % (D / 32)]);
          }
#pragma unroll
          for (int r = from(m); r < from(m + 1); ++r) {
            if (phase == 1) weight(0, r, (kPair ? 64 : 32) * b);
            if (kPair && phase == 2) residual(0, r, 64 * b);
            if (kPair && phase == 3) weight(1, r, 64 * b + 32);
            if (kPair && phase == 4) residual(1, r, 64 * b + 32);
          }
          if (!kPair && phase == 1 && m == kM - 1) {
#pragma unroll
            for (int r = 0; r < 16; ++r) residual(0, r, 32 * b);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      });
    };

    auto open_step = [&](int j) {  // step j's stage, complete; the next fetch, into the stage that step j - 1 was read from
      wait_lds();
      wait_vmem<(G::kStages - 2) * 2 * G::kDmaMin>();  // step j is here, step j + 1 of three may be on its way
      block_sync();
      const lds_char* const stage = lds + slot * G::kStage;
      fetch(j + G::kStages - 1, lds + (slot == 0 ? G::kStages - 1 : slot - 1) * G::kStage);
      slot = slot == G::kStages - 1 ? 0 : slot + 1;
      return stage;
    };
    const int whole = min(steps, len / kBN - begin);  // steps without rows past the segment's end: all but the last one
    if (active) {
      for (int j = 0; j < whole; ++j) step_of(open_step(j), std::false_type{}, kBN);
      if (whole < steps) step_of(open_step(whole), std::true_type{}, len - (begin + whole) * kBN);
    } else {
      for (int j = 0; j < steps; ++j) open_step(j);
    }
    wait_lds();
    wait_vmem<0>();
    block_sync();
  }

  // The results: registers 4 g + r of block db are channels 32 db + 8 g + 4 hb + r of the lane's row.  (All of LDS is free.)
  lds_char* const out = lds + wave * kOutWave;
  static_assert(W * kOutWave <= G::kLds, "the waves' output fits LDS");
  if (n > 1) {
    const int64_t rows = (int64_t)(kKeys ? a.total_k : a.total_q) * a.H * D;
    const int64_t at = w.split * rows + held0;
    write_part<D>(acc1, (kKeys ? a.part_k : a.part_q) + at, row0, held_len, a.H, out, lane);
    if constexpr (kKeys) write_part<D>(acc2, a.part_k + a.n_k * rows + at, row0, held_len, a.H, out, lane);
  } else {
    write_rows<D>(acc1, a.scale, (kKeys ? a.dk : a.dq) + held0, row0, held_len, a.H, out, lane);
    if constexpr (kKeys) write_rows<D>(acc2, 1.0f, a.dv + held0, row0, held_len, a.H, out, lane);
  }
}

// Bound by the matrix cores under the power cap: 32760 x 32760 x 12 heads (d = 128) 20.2 ms, in which its eight products
// run at 1300 TFLOP/s, what a large library product reaches on the same device; MFMA busy 68 % of 36.9 M clocks.  16380 x
// 16380 x 24 heads of d = 64 5.75 ms, 1150 TFLOP/s: exponentials and sums take as many clocks there as the products, which two
// of the three workgroups of a CU have to hide.  Each CU takes one item after the other; small calls are bound by the
// last ones, and by what each takes beside its products, 3 to 5 us (1024 x 1024 x 2 heads of d = 64: 12 us in this kernel).
template <int D, int W>
__global__ __launch_bounds__(64 * W, bwd_groups(D, 32 * W) * W / 4) void attn_bwd_kernel(BwdCall a) {
  extern __shared__ char smem[];
  const int item = blockIdx.x;
  const BwdTile t = ((const BwdTile*)(a.plan + 1))[item / a.H];  // (any of the item's list; read with the plan's length)
  if (item >= a.plan->tiles * a.H) return;
  if (t.keys) run_item<D, W, true>(a, find_item(t, item, a.H, a.n_k), (lds_char*)smem);
  else run_item<D, W, false>(a, find_item(t, item, a.H, a.n_q), (lds_char*)smem);
}

// The plan: the tiles of all segments' queries (for dq) and keys (for dk and dv), each once for every range of its
// streamed side.  Of these lists, one for each segment and side, the one with the longest items comes first, where
// there are up to kSorted of them; more keep their order.  One workgroup makes it.  Offsets that break the rules leave it
// empty.
constexpr int kPlanThreads = 256, kSorted = 1024;

__device__ __forceinline__ int wave_sum_to(int x, int lane) {  // inclusive prefix sum over the lanes
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  return x;
}

__device__ void make_plan(BwdPlan* plan, BwdOffsets f, int n_q, int n_k, int tile) {
  __shared__ int cost[kSorted], order[kSorted], part[kPlanThreads / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lists = 2 * f.nseq;
  bool bad = false;
  for (int s = tid; s < f.nseq; s += kPlanThreads) {
    const int q0 = f.cu_q[s], q1 = f.cu_q[s + 1], k0 = f.cu_k[s], k1 = f.cu_k[s + 1];
    // (differences of offsets within 0 and the totals do not overflow)
    bad |= q0 < 0 || q1 < q0 || q1 > f.total_q || k0 < 0 || k1 < k0 || k1 > f.total_k;
    if (!bad) {
      bad |= q1 - q0 > f.max_q || k1 - k0 > f.max_k;
      bad |= s == 0 && (q0 != 0 || k0 != 0);
      bad |= s == f.nseq - 1 && (q1 != f.total_q || k1 != f.total_k);
    }
  }
  if (__syncthreads_or(bad)) {
    if (tid == 0) plan->tiles = 0;
    return;
  }
  // list i: the keys of segment i / 2 for an even i, else its queries
  auto list = [&](int i, BwdTile& t) {
    const int s = i >> 1;
    t.keys = !(i & 1);
    t.held0 = t.keys ? f.cu_k[s] : f.cu_q[s];
    t.str0 = t.keys ? f.cu_q[s] : f.cu_k[s];
    t.held_len = (t.keys ? f.cu_k[s + 1] : f.cu_q[s + 1]) - t.held0;
    t.str_len = (t.keys ? f.cu_q[s + 1] : f.cu_k[s + 1]) - t.str0;
    t.tiles = (t.held_len + tile - 1) / tile;
  };
  const bool sorted = lists <= kSorted;
  if (sorted) {  // by the rows that stream past an item (as many products of each on either side)
    for (int i = tid; i < lists; i += kPlanThreads) {
      BwdTile t;
      list(i, t);
      cost[i] = t.tiles ? t.str_len / (t.keys ? n_k : n_q) : -1;
    }
    __syncthreads();
    for (int i = tid; i < lists; i += kPlanThreads) {
      const int mine = cost[i];
      int rank = 0;
      for (int j = 0; j < lists; ++j) rank += cost[j] > mine || (cost[j] == mine && j < i);
      order[rank] = i;
    }
    __syncthreads();
  }
  BwdTile* const to = (BwdTile*)(plan + 1);
  int before = 0;  // tiles of the lists before this round's
  for (int i0 = 0; i0 < lists; i0 += kPlanThreads) {
    const int i = i0 + tid;
    BwdTile t{};
    if (i < lists) list(sorted ? order[i] : i, t);
    const int n = t.tiles * (t.keys ? n_k : n_q);
    const int upto = wave_sum_to(n, lane);
    __syncthreads();  // (the round before has read its sums)
    if (lane == 63) part[wave] = upto;
    __syncthreads();
    t.first = before + upto - n;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
      if (w < wave) t.first += part[w];
      before += part[w];
    }
    for (int j = 0; j < n; ++j) to[t.first + j] = t;
  }
  if (tid == 0) plan->tiles = before;
}

// Before the gradients, as fast as memory takes it (40 us for 32760 x 12 heads, d = 128) or in 5 us of latency: the plan, by
// workgroup 0, and by the others -lse / scale and -D of every query and head,
// [2][H][total_q], 64 tokens of one head to a workgroup and a row of d bf16 to d / 8 lanes.
template <int D>
__global__ __launch_bounds__(kPlanThreads) void bwd_prepare_kernel(const __bf16* d_o, const __bf16* o, const float* lse, float* stat,
                                                                   int T, int H, float inv, BwdPlan* plan, BwdOffsets f, int n_q, int n_k, int tile) {
  if (blockIdx.x == 0) return make_plan(plan, f, n_q, n_k, tile);
  constexpr int kLanes = D / 8, kRows = kPlanThreads / kLanes;
  const int h = (blockIdx.x - 1) % H, t0 = (blockIdx.x - 1) / H * 64;
  const int r = threadIdx.x / kLanes, i = threadIdx.x % kLanes;
#pragma unroll
  for (int u = 0; u < 64 / kRows; ++u) {
    const int t = t0 + kRows * u + r;
    if (t >= T) continue;  // (all lanes of a row together)
    const int64_t at = ((int64_t)t * H + h) * D + 8 * i;
    const bf16x8 x = *(const bf16x8*)(d_o + at), y = *(const bf16x8*)(o + at);
    float sum = 0;
#pragma unroll
    for (int m = 0; m < 8; ++m) sum = __builtin_fmaf((float)x[m], (float)y[m], sum);
#pragma unroll
    for (int s = kLanes / 2; s > 0; s >>= 1) sum += __shfl_xor(sum, s);
    if (i == 0) {
      // of a query that saw no key, or none but of score -infinity, P is 0: its exponent is -infinity whatever the score
      const float l = lse[(int64_t)t * H + h];
      stat[(int64_t)h * T + t] = l == -INFINITY ? __builtin_copysignf(INFINITY, -inv) : -l * inv;
      stat[((int64_t)H + h) * T + t] = -sum;
    }
  }
}

// Sums of the ranges' partial gradients, in order: 16 rows of a head to a workgroup, 4 channels to a thread.  (A plan that is not empty
// covers all rows.)
constexpr int kJoinRows = 16;

template <int D>
__global__ __launch_bounds__(256) void bwd_join_kernel(BwdCall a, int blocks_k) {
  if (a.plan->tiles == 0) return;
  const bool keys = (int)blockIdx.x < blocks_k;
  const int b = keys ? blockIdx.x : blockIdx.x - blocks_k, n = keys ? a.n_k : a.n_q;
  const int64_t all = (int64_t)(keys ? a.total_k : a.total_q) * a.H, row0 = (int64_t)b * kJoinRows;
  constexpr int kLanes = D / 4, kRows = 256 / kLanes;
  const int64_t step = all * D;
  auto sum = [&](const float* p) {
    f32x4 x = *(const f32x4*)p;
    int i = 1;
    for (; i + 3 < n; i += 4) {  // four reads under way
      const f32x4 y0 = *(const f32x4*)(p + i * step), y1 = *(const f32x4*)(p + (i + 1) * step),
                  y2 = *(const f32x4*)(p + (i + 2) * step), y3 = *(const f32x4*)(p + (i + 3) * step);
      x = x + y0 + y1 + y2 + y3;
    }
    for (; i < n; ++i) x += *(const f32x4*)(p + i * step);
    return x;
  };
  auto narrow = [](f32x4 x, float f) { return bf16x4{(__bf16)(x[0] * f), (__bf16)(x[1] * f), (__bf16)(x[2] * f), (__bf16)(x[3] * f)}; };
#pragma unroll
  for (int u = 0; u < kJoinRows / kRows; ++u) {
    const int64_t row = row0 + kRows * u + threadIdx.x / kLanes;
    if (row >= all) return;
    const int64_t at = row * D + 4 * (threadIdx.x % kLanes);
    if (keys) {
      *(bf16x4*)(a.dk + at) = narrow(sum(a.part_k + at), a.scale);
      *(bf16x4*)(a.dv + at) = narrow(sum(a.part_k + n * step + at), 1.0f);
    } else {
      *(bf16x4*)(a.dq + at) = narrow(sum(a.part_q + at), a.scale);
    }
  }
}

template <int D>
hipError_t launch(const BwdArgs& x, hipStream_t st) {
  const float s = x.scale == 0.0f ? 1.0f : x.scale;
  const BwdCall a{(const __bf16*)x.d_o, (const __bf16*)x.q, (const __bf16*)x.k, (const __bf16*)x.v, x.stat,
                  (__bf16*)x.dq, (__bf16*)x.dk, (__bf16*)x.dv, x.part_q, x.part_k, x.plan,
                  x.total_q, x.total_k, x.H, x.n_q, x.n_k, x.scale, s * kLog2e};
  // (each kernel reads what the one before wrote: none goes out after one that was refused)
  const int64_t stats = ((int64_t)x.total_q + 63) / 64 * x.H;
  bwd_prepare_kernel<D><<<(unsigned)(1 + stats), kPlanThreads, 0, st>>>(
      a.d_o, (const __bf16*)x.o, x.lse, x.stat, x.total_q, x.H, 1.0f / s, x.plan,
      BwdOffsets{x.cu_q, x.cu_k, x.nseq, x.max_q, x.max_k, x.total_q, x.total_k}, x.n_q, x.n_k, x.tile);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t items = bwd_items(x.nseq, x.max_q, x.max_k, x.total_q, x.total_k, x.H, x.n_q, x.n_k, x.tile);
  if (items > 0 && x.tile == 128) attn_bwd_kernel<D, 4><<<(unsigned)items, Bwd<D, 4>::kThreads, Bwd<D, 4>::kLds, st>>>(a);
  if constexpr (D == 128)
    if (items > 0 && x.tile == 256) attn_bwd_kernel<D, 8><<<(unsigned)items, Bwd<D, 8>::kThreads, Bwd<D, 8>::kLds, st>>>(a);
  if (items > 0 && (e = hipGetLastError()) != hipSuccess) return e;
  const int64_t join_k = x.n_k > 1 ? ((int64_t)x.total_k * x.H + kJoinRows - 1) / kJoinRows : 0;
  const int64_t join_q = x.n_q > 1 ? ((int64_t)x.total_q * x.H + kJoinRows - 1) / kJoinRows : 0;
  if (join_k + join_q == 0) return hipSuccess;
  bwd_join_kernel<D><<<(unsigned)(join_k + join_q), 256, 0, st>>>(a, (int)join_k);
  return hipGetLastError();
}

hipError_t launch_attn_bwd(const BwdArgs& a, hipStream_t st) {
  return a.d == 64 ? launch<64>(a, st) : launch<128>(a, st);
}

hipError_t configure_kernels() {
  auto allow = [](const void* f, int bytes) { return hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, bytes); };
  hipError_t e = allow((const void*)attn_bwd_kernel<64, 4>, Bwd<64, 4>::kLds);
  if (e == hipSuccess) e = allow((const void*)attn_bwd_kernel<128, 4>, Bwd<128, 4>::kLds);
  if (e == hipSuccess) e = allow((const void*)attn_bwd_kernel<128, 8>, Bwd<128, 8>::kLds);
  return e;
}

}  // namespace tsblock
