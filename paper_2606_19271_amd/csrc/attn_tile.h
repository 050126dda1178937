// attn_tile.h -- device code shared by the attention kernels (attn_kernels.hip) and those over the session
// cache (cache_tiles.hip): the LDS layout of K and V tiles, the MFMA products that read it, the order of
// workgroups over the XCDs, waits and barriers.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn_launch.h"

namespace tsattn {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
typedef __attribute__((address_space(3))) bf16x8 lds_bf16x8;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) u32x2 lds_u32x2;
typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) void lds_void;

constexpr int kBM = kQueryTile;  // queries per work item
constexpr int kWaves = 8;      // waves per workgroup, 32 queries each
constexpr int kThreads = kWaves * 64;
constexpr float kLog2e = 1.4426950408889634f;
constexpr unsigned kRsrcWord3 = 0x00020000u;  // raw buffer, 32-bit data format (gfx9 family)

// LDS layout: a ring of three V tiles (first, so every V address fits the 16-bit immediate of a
// DS instruction), then a ring of four K tiles; V_j sits in stage j % 3 and K_j in j % 4.  Tiles arrive by
// LDS DMA (buffer_load ... lds: lane i of an instruction lands at base + 16 i), 1 KiB per
// instruction.
//  * K rows are padded by one 16-byte chunk (stride 2d + 16 bytes), so the 16 rows one b128 K
//    read touches per 16 lanes fall on distinct banks.  DMA lanes that land in a pad chunk fetch
//    a harmless duplicate.
//  * V rows are unpadded; the 16-byte chunk c of row r is stored at chunk position c ^ vswz(r),
//    which keeps the transposed V reads free of bank conflicts.
template <int D>
struct Geo {
  // Keys per K/V tile.  A matrix step costs the same number of MFMA clocks at both head widths
  // (32 32x32x16 MFMAs per wave): 64 keys at d = 128, 128 keys at d = 64, so the fixed costs of
  // a step (two barriers, the DMA issue, the waits) weigh the same against its matrix work.
  static constexpr int kBN = key_tile(D);
  static constexpr int kChunks = D / 8;                  // 16-byte chunks per row of d bf16
  static constexpr int kKRow = D * 2 + 16;               // padded K row stride (bytes)
  static constexpr int kVRow = D * 2;                    // V row stride (bytes)
  static constexpr int kKTile = kBN * kKRow;
  static constexpr int kVTile = kBN * kVRow;
  static constexpr int kKStages = 4;                     // K_j in stage j % 4
  static constexpr int kVStages = 3;                     // V_j in stage j % 3
  static constexpr int kVRing = 0;                       // byte offset of the V ring
  static constexpr int kKRing = kVStages * kVTile;       // byte offset of the K ring
  static constexpr int kRings = kKStages * kKTile + kVStages * kVTile;
  // Q staging of the prologue: 32 rows of each wave, in the K stage that no prologue fetch fills
  // and the space after the rings (and, for the one wave that does not fit there, in the last V
  // stage, unused until the first vector step as well).
  static constexpr int kQWave = 32 * D * 2;              // bytes of one wave's query rows
  static constexpr int kQBase = kKRing + (kKStages - 1) * kKTile;
  static constexpr int kQFit = 7;                        // waves staged from kQBase on
  static constexpr int kQLast = kVRing + (kVStages - 1) * kVTile;
  // Output staging of the epilogue, after the rings: 32 rows of 128 bytes per wave, padded by one
  // 16-byte chunk (both sides of the transposition then spread over the banks).
  static constexpr int kORow = 128 + 16;
  static constexpr int kOBase = kRings;
  static constexpr int kOWave = 32 * kORow;
  static constexpr int kLdsQ = kQBase + kQFit * kQWave;
  static constexpr int kLdsO = kOBase + kWaves * kOWave;
  static constexpr int kLds = kLdsQ > kLdsO ? kLdsQ : kLdsO;
  static constexpr int kGroupWaves = kWaves / 2;
  static constexpr int kKDma = kKTile / 1024;            // DMA instructions per K tile (17 / 18)
  static constexpr int kVDma = kVTile / 1024;            // per V tile (16 / 16)
  static constexpr int kKDmaMax = (kKDma + kGroupWaves - 1) / kGroupWaves;  // per wave, at most
  static constexpr int kKDmaMin = kKDma / kGroupWaves;                      // per wave, at least
  static constexpr int kVDmaPerWave = kVDma / kGroupWaves;
  // Pair steps of the softmax's exp work (16 per tile at d = 128, 32 at d = 64) between two of
  // the vector step's DMA instructions.  Issued back to back, the four vector-step waves of a CU
  // queue 16 KiB at once on its 64 B/clk address path, and each wave's exp work waits behind
  // its own share of that queue.
  static constexpr int kDmaEvery = 4;
  static_assert(kKTile % 1024 == 0 && kVTile % 1024 == 0 && kVDma % kGroupWaves == 0, "DMA split");
  static_assert(kVStages * kVTile <= 65536, "V addresses must fit the DS immediate");
  static_assert(kLds <= 160 * 1024, "LDS of a CU");
  static_assert(kQWave <= kVTile && kQFit == kWaves - 1, "the last wave's queries fit a V stage");
  __host__ __device__ static constexpr int vswz(int r) {
    return D == 128 ? (((r & 3) << 2) | ((r >> 2) & 3)) : ((((r >> 1) & 1) << 2) | ((r >> 2) & 3));
  }
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, (int)bytes,
                                           (int)kRsrcWord3);
}

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// max over the two 32-lane halves of the wave (lane l and lane l^32).
__device__ __forceinline__ float half_max(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

constexpr float kLn2 = 0.6931471805599453f;

// XCD-aware order: workgroup b runs on XCD b % 8; consecutive workgroups of one XCD take
// `chunk` consecutive items, and every 8*chunk workgroups cover 8*chunk consecutive items,
// so the global order is kept at that granularity.  The r items after the last whole span are
// dealt the same way: XCD x takes a contiguous block of its ceil((r - x) / 8) of them.
// Bijective on [0, total).
__device__ __forceinline__ int remap_block(int b, int total, int chunk) {
  const int span = 8 * chunk;
  const int full = (total / span) * span;
  const int x = b & 7;
  if (b < full) {
    const int j = b >> 3;
    return (j / chunk) * span + x * chunk + (j % chunk);
  }
  const int r = total - full, j = (b - full) >> 3;  // j-th tail workgroup of XCD x
  const int q = r >> 3, rem = r & 7;                // XCD x has q + (x < rem) of them
  return full + x * q + min(x, rem) + j;
}

// S^T = K Q^T for one key tile: 32-key blocks (two at d = 128, four at d = 64), each an
// accumulation over d in steps of 16.  Accumulator register r of block kb holds key
// 32*kb + 8*(r/4) + 4*hb + r%4 of the tile for the lane's query (lane & 31).  The blocks' MFMAs
// alternate, so that each Q fragment is the B operand of consecutive MFMAs: under the power cap
// an operand held over consecutive MFMAs costs less switching energy, and the clock rises
// accordingly (measured +0.6 % for two).  MFMA i uses the K fragment (kk, kb) = (i / nkb, i % nkb)
// with nkb blocks per tile; the first kPreReads of them were read ahead into kp.
constexpr int kPreReads = 8;

template <int D>
__device__ __forceinline__ const lds_char* k_frag(const lds_char* kt, int kk, int kb, int lane) {
  using G = Geo<D>;
  return kt + (32 * kb + (lane & 31)) * G::kKRow + (lane >> 5) * 16 + kk * 32;
}

// The K fragments of a tile's first kPreReads S MFMAs.
template <int D, int kPre = kPreReads>
__device__ __forceinline__ void k_preread(const lds_char* __restrict__ kt, bf16x8 (&kp)[kPre],
                                          int lane) {
  constexpr int kKB = Geo<D>::kBN / 32;  // 32-key blocks per tile
#pragma unroll
  for (int i = 0; i < kPre; ++i)
    kp[i] = *(const lds_bf16x8*)k_frag<D>(kt, i / kKB, i % kKB, lane);
}

template <int D, int kPre = kPreReads>
__device__ __forceinline__ void qk_tile(const lds_char* __restrict__ kt, const bf16x8 (&qf)[D / 16],
                                        const bf16x8 (&kp)[kPre],
                                        f32x16 (&s)[Geo<D>::kBN / 32], int lane) {
  constexpr int kKB = Geo<D>::kBN / 32;
#pragma unroll
  for (int kb = 0; kb < kKB; ++kb) s[kb] = f32x16{};
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
    for (int kb = 0; kb < kKB; ++kb) {
      const int i = kKB * kk + kb;
      bf16x8 a = i < kPre ? kp[i] : *(const lds_bf16x8*)k_frag<D>(kt, kk, kb, lane);
      s[kb] = mfma32(a, qf[kk], s[kb]);
    }
}

// Lane offsets of the transposed V reads inside a V tile: for 8-row group r2 and 32-channel
// block db, the 8 bytes of row 8 r2 + vr (+16 t) that this lane addresses.  Within each
// 16-lane group, lane 4R + c addresses 4 channels of key row R, and after the transpose lane j
// holds channel j of those 4 rows.
template <int D>
struct VOffsets {
  int off[2][D / 32];
  __device__ __forceinline__ explicit VOffsets(int lane) {
    using G = Geo<D>;
    const int g = lane >> 4, i16 = lane & 15;
    const int vr = 4 * (g >> 1) + (i16 >> 2);        // key row inside an 8-key group
    const int vch = 2 * (g & 1) + ((i16 & 3) >> 1);  // 16-byte chunk inside a 64-byte block
    const int vhalf = 8 * (i16 & 1);                 // 8-byte half of that chunk
#pragma unroll
    for (int r2 = 0; r2 < 2; ++r2)
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        const int row = 8 * r2 + vr;  // the swizzle depends on the row mod 16 only
        off[r2][db] = row * G::kVRow + (((4 * db + vch) ^ G::vswz(row)) << 4) + vhalf;
      }
  }
};

// Row sums of the weights on the matrix core: one 16x16x32 MFMA per 16-key step.  The B operand
// is the step's weight fragment p[t] as it is (lane l: 8 keys of query l & 31), which this MFMA
// reads as column l & 15, k = 8 (l >> 4) + 0..7; the A operand is 1 on the k-groups {G, G ^ 2}
// of the rows 4G..4G+3 and 0 elsewhere.  Result row 4G + r, column n is then the sum of lanes
// 16G + n and 16(G ^ 2) + n -- the two lanes of one query, l and l ^ 32 -- and it lands in
// exactly those lanes, in all four accumulator registers.  The sum is formed from exactly the
// bf16 weights the PV product uses, so a row dominated by one key returns that key's value
// exactly.  Summing in the vector step instead costs two VALU instructions per weight (a pair of
// bf16 is widened by a shift and a mask and added; v_dot2_f32_bf16 issues to the matrix core and
// stalls behind the other wave's MFMAs), and that step is the longer of the two.

// A operand of the row-sum MFMA for this lane: bf16 1.0 where the lane's k-group is one of the
// two groups its row block sums, else 0.
__device__ __forceinline__ bf16x8 row_sum_selector(int lane) {
  const int g = lane >> 4, mg = (lane & 15) >> 2;
  const unsigned one = (g == mg || g == (mg ^ 2)) ? 0x3f803f80u : 0u;
  return __builtin_bit_cast(bf16x8, u32x4{one, one, one, one});
}

// The row sums of one tile's weights, on two accumulators in turn: switching the matrix core
// between the 32x32x16 and the 16x16x32 shape costs about 6 clocks each way (measured), so the
// four row-sum MFMAs are issued together, and two chains keep them from waiting on each other.
template <int NT>
__device__ __forceinline__ void row_sums(bf16x8 sel, const bf16x8 (&p)[NT], f32x4 (&l)[2]) {
#pragma unroll
  for (int t = 0; t < NT; ++t)
    l[t & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(sel, p[t], l[t & 1], 0, 0, 0);
}

// O^T += V^T P^T for one 64-key tile.  p[t] holds the bf16 weights
// of keys 16t + 8*(m/4) + 4*hb + m%4 (m = 0..7) -- the accumulator order of qk_tile -- and the
// V^T fragments are read in that same key order with the transpose read: elements 0-3 from rows
// 16t + 4hb + 0..3, elements 4-7 from rows 16t + 8 + 4hb + 0..3.
template <int D>
__device__ __forceinline__ void pv_tile(const lds_char* __restrict__ vt, const VOffsets<D>& vo,
                                        const bf16x8 (&p)[Geo<D>::kBN / 16], f32x16 (&o)[D / 32]) {
  using G = Geo<D>;
#pragma unroll
  for (int t = 0; t < G::kBN / 16; ++t)
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      const lds_char* base = vt + 16 * t * G::kVRow;
      bf16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(base + vo.off[0][db]));
      bf16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(base + vo.off[1][db]));
      bf16x8 a = {v0[0], v0[1], v0[2], v0[3], v1[0], v1[1], v1[2], v1[3]};
      o[db] = mfma32(a, p[t], o[db]);
    }
}

// Waits until at most N of this wave's vector-memory operations are outstanding.
template <int N>
__device__ __forceinline__ void wait_vmem() {
  static_assert(N >= 0 && N < 16, "vmcnt field");
  __builtin_amdgcn_s_waitcnt(0x0F70 | N);  // gfx9 encoding: expcnt and lgkmcnt left open
}

// Waits until this wave's LDS operations are done (gfx9 encoding: vmcnt and expcnt left open).
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(0xC07F); }

// Workgroup barrier without a memory fence (the waits before it are explicit); the empty asm
// statements keep the compiler from moving memory accesses across it.
__device__ __forceinline__ void block_sync() {
  __asm__ volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  __asm__ volatile("" ::: "memory");
}

// The matrix step of tile j: the row sums of P_{j-1}, S_j = K_j Q^T, then O += V_{j-1} P_{j-1},
// in one basic block.  None of the first MFMAs waits for the LDS: the row sums read registers
// only, and the K fragments of the first kPreReads S MFMAs were read in the vector step before
// the barrier.  After that the issue order is pinned so that each MFMA's LDS operand is
// requested kPreReads MFMAs earlier (one b128 read per S MFMA, two transpose reads per PV MFMA).
// kSums = false: without the row sums, for kernels that form them in the vector step.  kPre: in place of kPreReads.
template <int D, bool kPV, bool kSums = true, int kPre = kPreReads>
__device__ __forceinline__ constexpr int m_step_reads(int i) {
  constexpr int kBN = Geo<D>::kBN;
  constexpr int kRS = kPV && kSums ? kBN / 16 : 0;  // row-sum MFMAs
  constexpr int kQK = (kBN / 32) * (D / 16);
  if (i < kRS) return 0;
  i -= kRS;
  return i < kQK ? (i < kPre ? 0 : 1) : 2;
}

template <int D, bool kPV, bool kSums = true, int kPre = kPreReads>
__device__ __forceinline__ void m_step(const lds_char* __restrict__ kt, const lds_char* __restrict__ vt,
                                       const VOffsets<D>& vo, const bf16x8 (&qf)[D / 16],
                                       const bf16x8 (&kp)[kPre],
                                       f32x16 (&s)[Geo<D>::kBN / 32],
                                       const bf16x8 (&p)[Geo<D>::kBN / 16], f32x16 (&o)[D / 32],
                                       bf16x8 sel, f32x4 (&l)[2], int lane) {
  constexpr int kBN = Geo<D>::kBN;
  if (kPV && kSums) row_sums(sel, p, l);
  qk_tile<D, kPre>(kt, qf, kp, s, lane);
  if (kPV) pv_tile<D>(vt, vo, p, o);
  // MFMAs: row sums (4), S (16 at d = 128), PV (16 at d = 128)
  constexpr int kN = (kPV && kSums ? kBN / 16 : 0) + (kBN / 32) * (D / 16) + (kPV ? (kBN / 16) * (D / 32) : 0);
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    const int next = i + kPre;  // MFMA whose operands are requested now
    const int reads = next < kN ? m_step_reads<D, kPV, kSums, kPre>(next) : 0;
    if (reads == 1) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    else if (reads == 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
  }
}

// n / d for 0 <= n < 2^23 and 1 <= d < 2^23 (float division is off by one at most there)
__device__ __forceinline__ int small_div(int n, int d) {
  int q = (int)((float)n * __builtin_amdgcn_rcpf((float)d));
  const int r = n - q * d;
  if (r < 0) --q;
  if (r >= d) ++q;
  return q;
}

}  // namespace tsattn
