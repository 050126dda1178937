// attn_bwd.hip -- the gradients of packed attention (ts_attn_bwd): D and the scaled log-sum-exp of each row, then dq and
// dk, dv on the matrix cores.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "attn_tile.h"
#include "block_launch.h"

namespace tsblock {

using namespace tsattn;

// The rows of one side are held in registers (dq: queries and d_o; dk, dv: keys and values), 32 by a wave, and those of
// the other stream through LDS, `kBN` of them at a time.  With X1, X2 the streamed pair (dq: k, v; dk, dv: q, d_o)
// and Y1, Y2 the held one, a wave computes for 32 streamed rows
//   S = X1 Y1^T,  T = X2 Y2^T           (32 x 32: streamed rows in registers, held ones over the lanes)
//   P = exp(scale S - lse),  R = P (T - D)
//   acc1^T += X1^T R   (dq or dk),      acc2^T += X2^T P   (dv)
// where P and R, as they lie, are the B operands of the last two products, whose A operands are transposed reads of
// the same LDS rows.
//
// LDS layout of a streamed tile: rows in groups of four, so that both the row reads (b128: 16 rows, the same 16-byte
// chunk) and the transposed ones (b64: 4 rows x 64 bytes) fall on distinct banks, with offsets that are sums of a
// lane's own and an immediate.  At d = 128 the four rows are 320 bytes apart, at d = 64 at 0, 128, 320 and 448.
template <int D>
struct Bwd {
  static constexpr int kBN = bwd_step(D);
  static constexpr int kGroup = D == 128 ? 1232 : 592;  // bytes of a group of four rows, 16 mod 64
  static constexpr int kTile = (kBN / 4 * kGroup + 1023) / 1024 * 1024;
  static constexpr int kDma = kTile / 1024;  // DMA instructions of a tile
  static constexpr int kDmaMax = (kDma + kWaves - 1) / kWaves, kDmaMin = kDma / kWaves;  // of a wave
  static constexpr int kStat = 2 * kTile;  // [2][kBN] floats, after X1 and X2
  static constexpr int kStage = 2 * kTile + 2 * kBN * 4;
  static constexpr int kStages = 3;
  static constexpr int kLds = kStages * kStage;
  static constexpr int kStatDma = kBN / 64;  // 4-byte DMA instructions of each statistic
  static_assert(kLds <= 160 * 1024, "LDS of a CU");
  __host__ __device__ static constexpr int row_offset(int r) {
    return (r >> 2) * kGroup + (D == 128 ? 320 * (r & 3) : 128 * (r & 1) + 320 * ((r >> 1) & 1));
  }
};

// Item `item` of a call: which segment, head, tile and range.
struct Found {
  int seg, h, tile, split;
  bool keys;  // dk, dv (held rows are keys), else dq
  int q0, nq, k0, nk;  // the segment's rows
};

struct Offsets {
  const int32_t* cu_q;
  const int32_t* cu_k;
  int nseq, max_q, max_k, total_q, total_k;
};

// A segment's rows; none where its offsets break the rules.
__device__ __forceinline__ void segment(const Offsets& f, int s, int& q0, int& nq, int& k0, int& nk) {
  q0 = f.cu_q[s];
  k0 = f.cu_k[s];
  const int q1 = f.cu_q[s + 1], k1 = f.cu_k[s + 1];
  const bool ok = q0 >= 0 && q1 >= q0 && q1 <= f.total_q && q1 - q0 <= f.max_q && k0 >= 0 && k1 >= k0 &&
                  k1 <= f.total_k && k1 - k0 <= f.max_k;
  nq = ok ? q1 - q0 : 0;
  nk = ok ? k1 - k0 : 0;
}

__device__ __forceinline__ int wave_sum_to(int x, int lane) {  // inclusive prefix sum over the lanes
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  return x;
}

// Tiles of both sides over all segments.
__device__ __forceinline__ void count_tiles(const Offsets& f, int lane, int& tiles_q, int& tiles_k) {
  tiles_q = tiles_k = 0;
  for (int s0 = 0; s0 < f.nseq; s0 += 64) {
    int q0, nq = 0, k0, nk = 0;
    if (s0 + lane < f.nseq) segment(f, s0 + lane, q0, nq, k0, nk);
    const int a = wave_sum_to((nq + kBwdTile - 1) / kBwdTile, lane), b = wave_sum_to((nk + kBwdTile - 1) / kBwdTile, lane);
    tiles_q += __shfl(a, 63);
    tiles_k += __shfl(b, 63);
  }
}

// The segment that holds item `at` of one side, whose segments have H * n items a tile; `at` becomes the item's place in it.
__device__ __forceinline__ void find_segment(const Offsets& f, bool keys, int per_tile, int lane, int& at, Found& w) {
  int before = 0;
  for (int s0 = 0; s0 < f.nseq; s0 += 64) {
    int q0 = 0, nq = 0, k0 = 0, nk = 0;
    if (s0 + lane < f.nseq) segment(f, s0 + lane, q0, nq, k0, nk);
    const int items = ((keys ? nk : nq) + kBwdTile - 1) / kBwdTile * per_tile;
    const int upto = before + wave_sum_to(items, lane);
    const uint64_t beyond = __builtin_amdgcn_ballot_w64(upto > at);
    if (beyond != 0) {
      const int l = __builtin_ctzll(beyond);
      w.seg = s0 + l;
      w.q0 = __shfl(q0, l);
      w.nq = __shfl(nq, l);
      w.k0 = __shfl(k0, l);
      w.nk = __shfl(nk, l);
      at -= __shfl(upto - items, l);
      return;
    }
    before = __shfl(upto, 63);
  }
}

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
  Offsets f;
  int H, n_q, n_k;
  bool q_first;
  float scale, c;  // c: log2(e) times the scale, or log2(e) for a scale of 0
};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Item `item`, or false past the last one.  The side with the longer items comes first; a side's items go by segment, head,
// range and tile, so that neighbours stream the same rows.
__device__ __forceinline__ bool find_item(const BwdCall& a, int item, int tiles_q, int tiles_k, int lane, Found& w) {
  const int items_q = tiles_q * a.H * a.n_q, items_k = tiles_k * a.H * a.n_k;
  if (item >= items_q + items_k) return false;
  int at = item;
  w.keys = a.q_first ? at >= items_q : at < items_k;
  if (w.keys && a.q_first) at -= items_q;
  if (!w.keys && !a.q_first) at -= items_k;
  const int n = w.keys ? a.n_k : a.n_q;
  find_segment(a.f, w.keys, a.H * n, lane, at, w);
  const int tiles = ((w.keys ? w.nk : w.nq) + kBwdTile - 1) / kBwdTile;
  const int j = at / tiles;
  w.tile = uniform(at - j * tiles);
  w.h = uniform(j / n);
  w.split = uniform(j % n);
  w.q0 = uniform(w.q0);
  w.nq = uniform(w.nq);
  w.k0 = uniform(w.k0);
  w.nk = uniform(w.nk);
  return true;
}

// Workgroup `item` of the dq (kKeys = false) or the dk, dv side.
template <int D, bool kKeys>
__device__ __forceinline__ void run_item(const BwdCall& a, const Found& w, lds_char* lds) {
  using G = Bwd<D>;
  constexpr int kBN = G::kBN;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int col = lane & 31, hb = lane >> 5;
  const int row_bytes = a.H * D * 2;
  const int held_len = kKeys ? w.nk : w.nq, len = kKeys ? w.nq : w.nk;  // held and streamed rows of the segment
  const int64_t held0 = ((int64_t)(kKeys ? w.k0 : w.q0) * a.H + w.h) * D, str0 = ((int64_t)(kKeys ? w.q0 : w.k0) * a.H + w.h) * D;
  const int row0 = w.tile * kBwdTile + 32 * wave;  // this wave's first held row

  // the range of steps
  const int steps_all = (len + kBN - 1) / kBN, n = kKeys ? a.n_k : a.n_q;
  const int begin = (int)((int64_t)steps_all * w.split / n), end = (int)((int64_t)steps_all * (w.split + 1) / n);
  const int steps = end - begin;

  f32x16 acc1[D / 32], acc2[kKeys ? D / 32 : 1];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) acc1[i] = f32x16{};
#pragma unroll
  for (int i = 0; i < (kKeys ? D / 32 : 1); ++i) acc2[i] = f32x16{};

  if (steps > 0) {
    const uint32_t held_bytes = (uint32_t)(held_len - 1) * (uint32_t)row_bytes + D * 2;
    const uint32_t str_bytes = (uint32_t)(len - 1) * (uint32_t)row_bytes + D * 2;
    const __amdgpu_buffer_rsrc_t ry1 = make_rsrc((kKeys ? a.k : a.q) + held0, held_bytes);
    const __amdgpu_buffer_rsrc_t ry2 = make_rsrc((kKeys ? a.v : a.d_o) + held0, held_bytes);
    const __amdgpu_buffer_rsrc_t rx1 = make_rsrc((kKeys ? a.q : a.k) + str0, str_bytes);
    const __amdgpu_buffer_rsrc_t rx2 = make_rsrc((kKeys ? a.d_o : a.v) + str0, str_bytes);
    // the head's statistics of the segment's queries
    const float* const stat = a.stat + (int64_t)w.h * a.f.total_q + w.q0;
    const int64_t stat_d = (int64_t)a.H * a.f.total_q;
    const __amdgpu_buffer_rsrc_t ra = make_rsrc(stat, (uint32_t)w.nq * 4);
    const __amdgpu_buffer_rsrc_t rd = make_rsrc(stat + stat_d, (uint32_t)w.nq * 4);

    // DMA: instruction i = wave + 8 u of a tile fills LDS bytes [1024 i, 1024 i + 1024), lane l 16 of them; lanes of the
    // pads fetch a row's first chunk again
    int off[G::kDmaMax];
#pragma unroll
    for (int u = 0; u < G::kDmaMax; ++u) {
      const int b = 1024 * (wave + kWaves * u) + 16 * lane;
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
    // Rows past the segment's end read as zeros.  Fetches past the range's last step stop at the segment's end, so that
    // no offset exceeds (len + 2 kBN - 1) rows.
    auto fetch = [&](int j, lds_char* stage) {
      const int step = min(begin + j, steps_all), skip = step * kBN * row_bytes;
#pragma unroll
      for (int u = 0; u < G::kDmaMax; ++u) {
        const int i = wave + kWaves * u;
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
    fetch(0, lds);
    fetch(1, lds + G::kStage);

    // held rows as B operands: row col, channels 16 kk + 8 hb + 0..7
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

    int slot = 0;
    for (int j = 0; j < steps; ++j) {
      wait_lds();
      wait_vmem<2 * G::kDmaMin>();  // step j is here, step j + 1 may be on its way
      block_sync();
      {
        int to = slot + 2;
        to -= to >= 3 ? 3 : 0;
        fetch(j + 2, lds + to * G::kStage);
      }
      const lds_char* const stage = lds + slot * G::kStage;
      const lds_char* const xr = stage + row_lane;
      const lds_char* const xt = stage + tr_lane;
      const int left = len - (begin + j) * kBN;  // streamed rows from the step's first one on
      if (active) {
#pragma unroll 1
        for (int b = 0; b < kBN / 32; ++b) {
          f32x16 s = {}, t = {};
          if (kKeys) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
              const f32x4 x = *(const lds_f32x4*)(stage + G::kStat + (32 * b + 8 * g + 4 * hb) * 4);
              const f32x4 y = *(const lds_f32x4*)(stage + G::kStat + kBN * 4 + (32 * b + 8 * g + 4 * hb) * 4);
#pragma unroll
              for (int r = 0; r < 4; ++r) s[4 * g + r] = x[r], t[4 * g + r] = y[r];
            }
          }
#pragma unroll
          for (int kk = 0; kk < D / 16; ++kk) {
            s = mfma32(*(const lds_bf16x8*)(xr + 8 * b * G::kGroup + 32 * kk), y1[kk], s);
            t = mfma32(*(const lds_bf16x8*)(xr + G::kTile + 8 * b * G::kGroup + 32 * kk), y2[kk], t);
          }
          // the reads of two products ahead of them
          __builtin_amdgcn_sched_group_barrier(0x100, kKeys ? 12 : 4, 0);
#pragma unroll
          for (int i = 0; i < D / 8; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (i < D / 8 - 4) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
          }
          __builtin_amdgcn_sched_barrier(0);
          bf16x8 p[2], ds[2];
          const bool whole = left >= 32 * b + 32;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            float e = __builtin_amdgcn_exp2f(kKeys ? s[r] * c : __builtin_fmaf(s[r], c, la));
            float x = e * (kKeys ? t[r] : t[r] + ld);
            if (!whole && 32 * b + 8 * (r >> 2) + 4 * hb + (r & 3) >= left) e = x = 0.0f;
            p[r >> 3][r & 7] = (__bf16)e;
            ds[r >> 3][r & 7] = (__bf16)x;
          }
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int db = 0; db < D / 32; ++db) {
              const lds_char* at = xt + (8 * b + 4 * u) * G::kGroup + 64 * db;
              bf16x4 a0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)at);
              bf16x4 a1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(at + 2 * G::kGroup));
              acc1[db] = mfma32(bf16x8{a0[0], a0[1], a0[2], a0[3], a1[0], a1[1], a1[2], a1[3]}, ds[u], acc1[db]);
              if (kKeys) {
                a0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(at + G::kTile));
                a1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(at + G::kTile + 2 * G::kGroup));
                acc2[db] = mfma32(bf16x8{a0[0], a0[1], a0[2], a0[3], a1[0], a1[1], a1[2], a1[3]}, p[u], acc2[db]);
              }
            }
          __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
#pragma unroll
          for (int i = 0; i < D / 16 * (kKeys ? 2 : 1); ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (i < D / 16 * (kKeys ? 2 : 1) - 4) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      slot = slot == 2 ? 0 : slot + 1;
    }
    wait_lds();
    wait_vmem<0>();
    block_sync();  // the next item's fetches come into stages that nobody reads or fills any more
  }

  // accumulator register 4 g + r of block db: channel 32 db + 8 g + 4 hb + r of the lane's row
  const int row = row0 + col;
  if (row >= held_len) return;
  const float scale = a.scale;
  if (n > 1) {
    const int64_t rows = (int64_t)(kKeys ? a.f.total_k : a.f.total_q) * a.H * D;
    float* const to = (kKeys ? a.part_k : a.part_q) + w.split * rows + held0 + (int64_t)row * a.H * D + 4 * hb;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        *(f32x4*)(to + 32 * db + 8 * g) = f32x4{acc1[db][4 * g], acc1[db][4 * g + 1], acc1[db][4 * g + 2], acc1[db][4 * g + 3]};
        if (kKeys)
          *(f32x4*)(to + a.n_k * rows + 32 * db + 8 * g) =
              f32x4{acc2[db][4 * g], acc2[db][4 * g + 1], acc2[db][4 * g + 2], acc2[db][4 * g + 3]};
      }
    return;
  }
  const int64_t to = held0 + (int64_t)row * a.H * D + 4 * hb;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      bf16x4 x;
#pragma unroll
      for (int r = 0; r < 4; ++r) x[r] = (__bf16)(acc1[db][4 * g + r] * scale);
      *(bf16x4*)((kKeys ? a.dk : a.dq) + to + 32 * db + 8 * g) = x;
      if (kKeys) {
#pragma unroll
        for (int r = 0; r < 4; ++r) x[r] = (__bf16)acc2[db][4 * g + r];
        *(bf16x4*)(a.dv + to + 32 * db + 8 * g) = x;
      }
    }
}

template <int D>
__global__ __launch_bounds__(kThreads, 2) void attn_bwd_kernel(BwdCall a) {
  extern __shared__ char smem[];
  const int lane = threadIdx.x & 63;
  int tiles_q, tiles_k;
  count_tiles(a.f, lane, tiles_q, tiles_k);
  const int total = tiles_q * a.H * a.n_q + tiles_k * a.H * a.n_k;
  for (int b = blockIdx.x; b < total; b += gridDim.x) {
    Found w;
    if (!find_item(a, remap_block(b, total, 32), tiles_q, tiles_k, lane, w)) break;
    if (w.keys) run_item<D, true>(a, w, (lds_char*)smem);
    else run_item<D, false>(a, w, (lds_char*)smem);
  }
}

// -lse / scale and -D of every query and head, [2][H][total_q]: 64 tokens of one head to a workgroup, a row of d bf16 to
// d / 8 lanes.
template <int D>
__global__ __launch_bounds__(256) void bwd_stat_kernel(const __bf16* d_o, const __bf16* o, const float* lse, float* stat, int T,
                                                       int H, float inv) {
  constexpr int kLanes = D / 8, kRows = 256 / kLanes;
  const int h = blockIdx.x % H, t0 = blockIdx.x / H * 64;
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
      stat[(int64_t)h * T + t] = -lse[(int64_t)t * H + h] * inv;
      stat[((int64_t)H + h) * T + t] = -sum;
    }
  }
}

// Sums of the ranges' partial gradients, in order.  Workgroups take the tiles of the segments, as attn_bwd_kernel does.
template <int D>
__global__ __launch_bounds__(256) void bwd_join_kernel(BwdCall a) {
  const int lane = threadIdx.x & 63;
  int tiles_q, tiles_k;
  count_tiles(a.f, lane, tiles_q, tiles_k);
  BwdCall whole = a;
  whole.n_q = whole.n_k = 1;
  const int total = (tiles_q + tiles_k) * a.H;
  for (int b = blockIdx.x; b < total; b += gridDim.x) {
    Found w;
    if (!find_item(whole, b, tiles_q, tiles_k, lane, w)) break;
    const int n = w.keys ? a.n_k : a.n_q;
    if (n == 1) continue;
    const int64_t rows = (int64_t)(w.keys ? a.f.total_k : a.f.total_q) * a.H * D;
    const int64_t start = ((int64_t)(w.keys ? w.k0 : w.q0) * a.H + w.h) * D;
    const int end = min(w.keys ? w.nk : w.nq, (w.tile + 1) * kBwdTile);
    constexpr int kLanes = D / 4;
    for (int r = w.tile * kBwdTile + threadIdx.x / kLanes; r < end; r += 256 / kLanes) {
      const int64_t at = start + (int64_t)r * a.H * D + 4 * (threadIdx.x % kLanes);
      for (int which = 0; which < (w.keys ? 2 : 1); ++which) {
        const float* p = (w.keys ? a.part_k + which * n * rows : a.part_q) + at;
        f32x4 sum = *(const f32x4*)p;
        for (int i = 1; i < n; ++i) sum += *(const f32x4*)(p + i * rows);
        const float f = which == 1 ? 1.0f : a.scale;
        __bf16* const to = !w.keys ? a.dq : which == 1 ? a.dv : a.dk;
        *(bf16x4*)(to + at) = bf16x4{(__bf16)(sum[0] * f), (__bf16)(sum[1] * f), (__bf16)(sum[2] * f), (__bf16)(sum[3] * f)};
      }
    }
  }
}

template <int D>
hipError_t launch(const BwdArgs& x, hipStream_t st) {
  const float s = x.scale == 0.0f ? 1.0f : x.scale;
  const BwdCall a{(const __bf16*)x.d_o, (const __bf16*)x.q, (const __bf16*)x.k, (const __bf16*)x.v, x.stat,
                  (__bf16*)x.dq, (__bf16*)x.dk, (__bf16*)x.dv, x.part_q, x.part_k,
                  {x.cu_q, x.cu_k, x.nseq, x.max_q, x.max_k, x.total_q, x.total_k}, x.H, x.n_q, x.n_k,
                  3ll * x.max_k * x.n_k >= 4ll * x.max_q * x.n_q, x.scale, s * kLog2e};
  const int64_t stats = ((int64_t)x.total_q + 63) / 64 * x.H;
  if (stats > 0)
    bwd_stat_kernel<D><<<(unsigned)stats, 256, 0, st>>>(a.d_o, (const __bf16*)x.o, x.lse, x.stat, x.total_q, x.H, 1.0f / s);
  const int64_t tiles_q = bwd_tiles(x.nseq, x.max_q, x.total_q, x.H), tiles_k = bwd_tiles(x.nseq, x.max_k, x.total_k, x.H);
  const int64_t items = std::min<int64_t>(tiles_q * x.n_q + tiles_k * x.n_k, kBwdGrid);
  if (items > 0) attn_bwd_kernel<D><<<(unsigned)items, kThreads, Bwd<D>::kLds, st>>>(a);
  if (items > 0 && (x.n_q > 1 || x.n_k > 1)) bwd_join_kernel<D><<<(unsigned)(tiles_q + tiles_k), 256, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_attn_bwd(const BwdArgs& a, hipStream_t st) {
  return a.d == 64 ? launch<64>(a, st) : launch<128>(a, st);
}

hipError_t configure_kernels() {
  hipError_t e = hipFuncSetAttribute((const void*)attn_bwd_kernel<64>, hipFuncAttributeMaxDynamicSharedMemorySize, Bwd<64>::kLds);
  if (e == hipSuccess)
    e = hipFuncSetAttribute((const void*)attn_bwd_kernel<128>, hipFuncAttributeMaxDynamicSharedMemorySize, Bwd<128>::kLds);
  return e;
}

}  // namespace tsblock
