// cache_rows.h -- attention of up to 32 query rows of one cached head over a range of its session's pages, by a
// workgroup whose waves take the pages in turn.  Used for calls of few rows (cache_attn.hip) and, once or twice, for the last, thin
// tile of a session's rows (cache_tiles.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_device.h"

namespace tscache {

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Waits until at most N of this wave's vector-memory operations are outstanding (gfx9 encoding: the count's upper
// two bits are 15:14), and keeps memory accesses from moving across.
template <int N>
__device__ __forceinline__ void wait_vmem_in_order() {
  static_assert(N >= 0 && N < 64, "vmcnt field");
  __asm__ volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0F70 | (N & 15) | (N >> 4) << 14);
  __asm__ volatile("" ::: "memory");
}

// The waves share nothing until the end, so there is no barrier in the loop.  Per page a wave computes S^T = K Q^T
// on 16x16x32 MFMAs (lane: query row lane & 15, keys 4 (lane >> 4) + 0..3 of each 16), keeps a running maximum and
// sum per row, and accumulates O^T += V^T P^T, whose B operand is the lane's own weights once the 32 keys of a step
// are taken in the order in which two score blocks hold them.  K goes from memory to MFMA operands in registers: a
// lane loads D / 4 consecutive channels of a key, and the sum over channels takes them in that order on both sides.
// V's bytes go by LDS DMA to the wave's own two buffers, in an order (v_chunk) in which the 8-bit transpose reads
// spread over the banks; both arrive a page ahead of their use.  Bound by HBM: 32 single tokens x 8 heads x 5 over 32760 to
// 6193 keys, d = 128, 215 us, 1.28 GB at 5.9 TB/s (one page's keys in registers at a time: 219); short calls by the round trips
// from the lengths to the pages' numbers, to their bytes, to the result: 9.4 us for a page a wave.
template <int D, int NB, int kW>
struct RowGeo {
  static constexpr int kKK = D / 32;                     // MFMA steps over the channels
  static constexpr int kCB = D / 16;                     // 16-channel blocks of O
  static constexpr int kVLoads = kPage * D / 1024;       // LDS DMA instructions of V per page
  static constexpr int kKLoads = D / 64;                 // 16-byte loads of K per lane and 16 keys
  static constexpr int kPageBytes = kPage * D;
  static constexpr bool kEarly = D * NB < 256;           // room for two pages' keys in registers
  static constexpr int kVBufs = kW * 2 * kPageBytes;
  static constexpr int kObuf = kW * 16 * D * 4;          // over the V buffers, at the end
  static constexpr int kMl = kVBufs > kObuf ? kVBufs : kObuf;  // float [2][kW][16]: maxima and sums
  static constexpr int kLds = kMl + 2 * kW * 16 * 4;
  // channels of a thread when the waves' results are joined, 16 rows at a time
  static constexpr int kCh = D / (4 * kW) < 4 ? 4 : D / (4 * kW);
};

constexpr int kRowsDown = 17;  // value_exp: sums of weights of up to 1, of 2^17 keys

// f over the lanes that differ in bits 4 and 5.
template <typename F>
__device__ __forceinline__ float across(float x, F&& f) {
  x = f(x, __shfl_xor(x, 16));
  return f(x, __shfl_xor(x, 32));
}

// Position of 16-byte chunk `chunk` of V row `row` in LDS.
template <int D>
__device__ __forceinline__ constexpr int v_chunk(int row, int chunk) {
  return D == 128 ? chunk ^ (row >> 1 & 7) : chunk ^ (row >> 2 & 3);
}

// A range of a session's pages: first, first + step, ... < end.  Wave w of kW takes the pages number w, w + kW, ...
struct PageRange {
  int first, step, end;
  __device__ __forceinline__ int page(int i) const { return first + step * i; }
};

// The first table entries of a wave's pages, one a lane.  Asked for before the session's length is known, they arrive
// with it: entries past the last page are read (inside the table) and not used.
template <int kW>
__device__ __forceinline__ int first_ids(const int32_t* table, int width, int first, int step) {
  const int tid = thread_anew(), p = first + step * ((tid >> 6) + kW * (tid & 63));
  return p < width ? table[p] : 0;
}

// Rows [row0, row0 + 16 NB) of `rows` (see row_of) over a range of pages, `id` its first_ids; kW waves, RowGeo::kLds
// bytes of LDS.  `to`: of kSlab the range's number; of kSlot the first row's place in the slots, or -1 for a result.
template <int D, int NB, int kW, Out kOut>
__device__ __forceinline__ void rows_item(const RowArgs& a, const Session& se, const int32_t* table, int h, int row0,
                                          int rows, const PageRange& range, int id, int to, char* smem) {
  using R = RowGeo<D, NB, kW>;
  constexpr int kKK = R::kKK, kCB = R::kCB, kVLoads = R::kVLoads, kKLoads = R::kKLoads, kPageBytes = R::kPageBytes;
  const int tid = thread_anew(), lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int i16 = lane & 15, g = lane >> 4;
  const int H = a.pool.H, G = a.G;
  lds_char* const lds = (lds_char*)smem;
  lds_char* const vbuf = lds + wave * 2 * kPageBytes;

  // ---- the wave's pages; lane i has the number and exponents of the i-th of 64 of them
  const int left = range.end - range.page(wave), apart = kW * range.step;
  const int mine = left > 0 ? (left + apart - 1) / apart : 0;
  int kexp = 0, vexp = 0;
  auto exponents = [&] {
    const bool bad = (unsigned)id >= (unsigned)a.pool.pages;
    id = bad ? 0 : id;
    kexp = a.pool.k_exp[(int64_t)id * H + h];
    vexp = a.pool.v_exp[(int64_t)id * H + h];
    if (bad) kexp = vexp = 255;  // reads as NaN
    vexp = value_exp(vexp, kRowsDown);
  };
  typedef u32x4 Keys[4][kKLoads];
  const int koff = i16 * D + D / 4 * g;
  int i0 = 0, now = min(mine, 64);  // the pages whose numbers the lanes have: i0, ... i0 + now - 1 of the wave's
  auto load = [&](int i, Keys& kx, lds_char* to) {  // page i0 + i; past the last of them, nothing
    const int64_t at = ((int64_t)__builtin_amdgcn_readlane(id, i & 63) * H + h) * kPageBytes;
    // rows past the session's end as zeros: scores that are masked, values that meet weights of zero
    const int n = __builtin_amdgcn_readfirstlane(i < now ? min(kPage, se.len - range.page(wave + kW * (i0 + i)) * kPage) : 0);
    __amdgpu_buffer_rsrc_t rk = make_rsrc(a.pool.k + at, (uint32_t)(n * D));
    __amdgpu_buffer_rsrc_t rv = make_rsrc(a.pool.v + at, (uint32_t)(n * D));
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
#pragma unroll
      for (int x = 0; x < kKLoads; ++x)
        kx[kb][x] = __builtin_amdgcn_raw_buffer_load_b128(rk, koff + 16 * kb * D + 16 * x, 0, 0);
#pragma unroll
    for (int x = 0; x < kVLoads; ++x) {
      const int row = (64 * x + lane) / (D / 16);
      dma16(rv, to + 1024 * x, row * D + v_chunk<D>(row, lane % (D / 16)) * 16);
    }
    __asm__ volatile("" ::: "memory");
  };
  if (mine > 0) exponents();

  u32x4 qraw[NB][kKK];
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const int r = row0 + 16 * n + i16;
    const __bf16* const src = a.q + row_of(se, min(r, rows - 1), h, H, G) * D + D / 4 * g;
#pragma unroll
    for (int kk = 0; kk < kKK; ++kk) qraw[n][kk] = *(const u32x4*)(src + 8 * kk);
  }
  lds_char *const v0 = vbuf, *const v1 = vbuf + kPageBytes;
  Keys k0, k1;
  if (mine > 0) load(0, k0, v0);  // before the queries are waited for
  bf16x8 qf[NB][kKK];
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int kk = 0; kk < kKK; ++kk)
      qf[n][kk] = __builtin_bit_cast(bf16x8, qraw[n][kk] ^ u32x4{a.flip, a.flip, a.flip, a.flip});
  f32x4 o[NB][kCB] = {};
  float m[NB], l[NB];
#pragma unroll
  for (int n = 0; n < NB; ++n) m[n] = -INFINITY, l[n] = 0.0f;

  // Page i0 + i, its keys in kx; the next page's go to `next`, before this one's are waited for (R::kEarly) or once they are used.
  // `from` holds the page's values, `to` takes the next page's: told that they are apart, the compiler does not have the
  // transpose reads wait for every DMA in flight.
  auto page = [&](int i, Keys& kx, Keys& next, lds_char* __restrict to, const lds_char* __restrict from) {
    const int valid = se.len - range.page(wave + kW * (i0 + i)) * kPage;  // keys of this page (64 or more: all)
    if (R::kEarly) load(i + 1, next, to);
    // (after those loads: the first page's exponents may still be on their way)
    const float ks = __uint_as_float((unsigned)__builtin_amdgcn_readlane(kexp, i) << 23);
    const float v_scale = __uint_as_float((unsigned)__builtin_amdgcn_readlane(vexp, i) << 23);
    if (R::kEarly) __builtin_amdgcn_sched_barrier(0);  // the products stay behind those loads
    f32x4 sc[NB][4] = {};
#pragma unroll
    for (int kb = 0; kb < 4; ++kb)
#pragma unroll
      for (int kk = 0; kk < kKK; ++kk) {
        const bf16x8 kf = widen8(kx[kb][kk / 2][2 * (kk & 1)], kx[kb][kk / 2][2 * (kk & 1) + 1], ks);
#pragma unroll
        for (int n = 0; n < NB; ++n) sc[n][kb] = mfma16(kf, qf[n][kk], sc[n][kb]);
      }
    if (!R::kEarly) load(i + 1, next, to);
    bf16x8 pf[NB][2];
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      float mt = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (16 * kb + 4 * g + r < valid) mt = fmaxf(mt, sc[n][kb][r]);
      mt = across(mt, [](float x, float y) { return fmaxf(x, y); });
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
    // this page's V: all but the next page's loads are done
    wait_vmem_in_order<4 * kKLoads + kVLoads>();
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int cb = 0; cb < kCB; ++cb) {
        // lane 2 R + c of 16 addresses bytes 8 c of key row R; it gets channel lane & 15 of the 8 rows:
        // keys 4 g + 0..3 of the step's first 16, then of its second
        const int r8 = i16 >> 1;
        const int row = 32 * u + (r8 & 4) * 4 + 4 * g + (r8 & 3);
        const i32x2 x = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
            (lds_i32x2*)(from + row * D + v_chunk<D>(row, cb) * 16 + 8 * (i16 & 1)));
        const bf16x8 vf = widen8((unsigned)x[0], (unsigned)x[1], v_scale);
#pragma unroll
        for (int n = 0; n < NB; ++n) o[n][cb] = mfma16(vf, pf[n][u], o[n][cb]);
      }
    // the reads have left the buffer before the next but one page's DMA comes into it
    wait_lds();
    __asm__ volatile("" ::: "memory");
  };
  for (; i0 < mine; i0 += 64) {
    if (i0 > 0) {
      now = min(mine - i0, 64);
      id = lane < now ? table[range.page(wave + kW * (i0 + lane))] : 0;
      exponents();
      load(0, k0, v0);
    }
    if constexpr (R::kEarly) {
      for (int i = 0; i < now; i += 2) {
        page(i, k0, k1, v1, v0);
        if (i + 1 < now) page(i + 1, k1, k0, v0, v1);
      }
    } else {
      for (int i = 0; i < now; ++i) page(i, k0, k0, i & 1 ? v0 : v1, i & 1 ? v1 : v0);
    }
    wait_vmem_in_order<0>();  // (nothing lands in the buffers any more)
  }

  // ---- join the waves: O = sum_w 2^(m_w - M) O_w / sum_w 2^(m_w - M) l_w, 16 rows at a time
  typedef __attribute__((address_space(3))) float lds_float;
  typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
  lds_float* const obuf = (lds_float*)lds;
  lds_float* const ml = (lds_float*)(lds + R::kMl);
  constexpr int kCh = R::kCh;
  const int orow = tid / (D / kCh), och = tid % (D / kCh) * kCh;
#pragma unroll
  for (int n = 0; n < NB; ++n) {
    const float ln = across(l[n], [](float x, float y) { return x + y; });
    __syncthreads();
#pragma unroll
    for (int cb = 0; cb < kCB; ++cb) *(lds_f32x4*)(obuf + (wave * 16 + i16) * D + 16 * cb + 4 * g) = o[n][cb];
    if (g == 0) ml[wave * 16 + i16] = m[n], ml[(kW + wave) * 16 + i16] = ln;
    __syncthreads();
    const int r = row0 + 16 * n + orow;
    if (orow >= 16 || r >= rows) continue;
    float big = -INFINITY, sum = 0.0f;
    f32x4 acc[kCh / 4] = {};
#pragma unroll
    for (int w = 0; w < kW; ++w) big = fmaxf(big, ml[w * 16 + orow]);
#pragma unroll
    for (int w = 0; w < kW; ++w) {
      const float mw = ml[w * 16 + orow], lw = ml[(kW + w) * 16 + orow];
      if (lw == 0.0f) continue;  // no keys
      const float f = mw == big ? 1.0f : __builtin_amdgcn_exp2f(mw - big);
      sum += f * lw;
#pragma unroll
      for (int x = 0; x < kCh / 4; ++x) acc[x] += f * *(const lds_f32x4*)(obuf + (w * 16 + orow) * D + och + 4 * x);
    }
    const float inv = sum == 0.0f ? 0.0f : (float)(1 << kRowsDown) / sum;
    const float lse = sum == 0.0f ? -INFINITY : (big + __builtin_amdgcn_logf(sum)) * kLn2;
    const int64_t at = row_of(se, r, h, H, G);
    if (kOut == kSlab || (kOut == kSlot && to >= 0)) {
      const int64_t part = kOut == kSlot ? (int64_t)to + (r - row0) : (int64_t)to * a.ss.total * (H * G) + at;
      if (sum != 0.0f)
#pragma unroll
        for (int x = 0; x < kCh / 4; ++x) *(f32x4*)(a.part_o + part * D + och + 4 * x) = acc[x] * inv;
      if (och == 0) a.part_lse[part] = lse;
    } else {
#pragma unroll
      for (int x = 0; x < kCh / 4; ++x)
        *(bf16x4*)(a.o + at * D + och + 4 * x) = __builtin_convertvector(acc[x] * inv, bf16x4);
      if (a.lse != nullptr && och == 0) a.lse[at] = lse;
    }
  }
}

}  // namespace tscache
