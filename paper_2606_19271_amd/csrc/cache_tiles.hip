// cache_tiles.hip -- attention of many query rows over the session cache: 256-row tiles on the matrix cores.
//
// The schedule is the one of the bf16 kernels (attn_kernels.hip): a workgroup of eight waves owns 256 query
// rows of one cached head; a wave has 32 of them and alternates between a matrix step (S = K Q^T of one key
// tile, O += V P of the one before, on 32x32x16 MFMAs) and a vector step (the online softmax), the two waves of
// a SIMD in opposite steps.  What differs is how the tiles arrive.  A page's bytes cannot go to LDS by DMA,
// because the MFMA operands are bf16: the vector step's waves load a tile's bytes into registers one step
// ahead (8 KiB per tile and operand, half of what bf16 takes), widen them (one instruction per two elements,
// with the page's power of two; exact) and write the bf16 image.  Each element is widened once per workgroup.
//
// The registers between memory and LDS are one more stage, so the rings are shorter.  Phases are numbered as in
// attn_kernels.hip (A's M(j) = 2j, A's V(j) = B's M(j) = 2j + 1, B's V(j) = 2j + 2).  Group A (waves 0-3) writes
// K_{j+2} in its V(j), phase 2j + 1, over K_{j-1}, whose last reader is B's M(j-1) in phase 2j - 1; its first
// reader is A itself at the end of V(j+1), phase 2j + 3.  Group B (waves 4-7) writes V_{j+1} in its V(j), phase
// 2j + 2, over V_{j-1}, last read by B's M(j) in phase 2j + 1, first read by A's M(j+2) in phase 2j + 4.  So K
// has three stages and V two.
//
// The sum of the weights is formed in the vector step before their rounding to bf16 (two chains of additions; the sum
// also tells whether a weight is too large for the running maximum), so that the log-sum-exp is good to fp32: the
// cached tokens' weights are formed against it.  On the matrix core, from the rounded weights as in attn_kernels.hip,
// it would take 1.4 % less time (4680 rows x 32760 keys x 40 heads, d = 128: 2548 against 2583 us).
//
// Registers bound the matrix step: with the bytes of the next tile held through it, operands read 8 MFMAs ahead leave
// the scheduler without room (it then reads each one right before its use); 4 ahead cost nothing (attn_kernels.hip
// reads 8 ahead).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "attn_tile.h"
#include "cache_device.h"
#include "cache_launch.h"
#include "cache_rows.h"

namespace tscache {

template <int D>
struct TileGeo {
  using G = Geo<D>;
  static constexpr int kBN = G::kBN;                     // keys of a tile
  static constexpr int kPages = kBN / kPage;             // pages of a tile (1 at d = 128, 2 at d = 64)
  static constexpr int kLoads = kBN * D / 4 / 1024;      // 16-byte loads per lane, tile and operand (4 waves)
  static constexpr int kVRing = 0, kVStages = 2;
  static constexpr int kKRing = kVStages * G::kVTile, kKStages = 3;
  static constexpr int kRings = kKRing + kKStages * G::kKTile;
  static constexpr int kQBase = kRings;                  // 32 rows of each wave, in the prologue
  static constexpr int kOBase = kRings;                  // and of O in the epilogue
  static constexpr int kPre = 4;                         // LDS reads ahead of their MFMAs
  static constexpr int kEntries = 512;                   // pages in a group's list (PageEntry)
  static constexpr int kList = kRings + kWaves * (G::kQWave > G::kOWave ? G::kQWave : G::kOWave);
  static constexpr int kLds = kList + 2 * kEntries * 8;
  static_assert(G::kVTile == 16384 && kVRing == 0 && kVStages == 2, "a V stage is one bit of an LDS address");
  static_assert(kLoads == 2, "two loads per lane: one page each at d = 64, both of one at d = 128");
  static_assert(kLds + 32 <= 160 * 1024, "LDS of a CU");
};

// One item: query rows [row0, row0 + 256) of (session, head h) against key tiles [tile_begin, + ntiles).
struct TileItem {
  Session se;
  const int32_t* table;  // the session's pages
  int h, row0, rows, tile_begin, ntiles, split;
  int slot;  // where a piece of the item goes that kEven's shares have cut, or -1
};

// A page of the session's as a group fetches it: its number, and its exponent as the bits of a float.  Pages past the
// session's end are page 0 (of which no byte is read), with a scale of 1; pages outside the pool are page 0 with the
// scale that makes them NaN.
struct PageEntry {
  int id;
  unsigned scale;
};

// exp2(S c - m_c) of the lane's scores, packed for the PV product; returns their sum, in fp32 before that rounding.
template <int NT, int kIssue, int kEvery, typename Issue>
__device__ __forceinline__ float exp_pack(const f32x16 (&s)[NT / 2], bf16x8 (&p)[NT], float m_c, float c,
                                          Issue&& issue) {
  float sum0 = 0.0f, sum1 = 0.0f;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
#pragma unroll
    for (int m = 0; m < 8; m += 2) {
      const int step = 4 * t + m / 2;
      if (kIssue > 0 && step % kEvery == 0 && step / kEvery < kIssue) {
        __builtin_amdgcn_sched_barrier(0);
        issue(step / kEvery);
        __builtin_amdgcn_sched_barrier(0);
      }
      const float x0 = s[t >> 1][8 * (t & 1) + m], x1 = s[t >> 1][8 * (t & 1) + m + 1];
      const f32x2 e = {__builtin_amdgcn_exp2f(__builtin_fmaf(x0, c, -m_c)),
                       __builtin_amdgcn_exp2f(__builtin_fmaf(x1, c, -m_c))};
      sum0 += e[0];
      sum1 += e[1];
      // the weights enter the product in 16 bits, its operands' type
      const bf16x2 pb = __builtin_convertvector(e, bf16x2);
      p[t][m] = pb[0];
      p[t][m + 1] = pb[1];
    }
  }
  float sum = sum0 + sum1;
  // keeps the additions here: sunk behind a test of the weights, they would hold all of them in registers
  __asm__ volatile("" : "+v"(sum));
  return sum;
}

struct NoHook {
  __device__ void operator()(int) const {}
};

// As kBias of attn_kernels.hip, the running maximum is raised by this, so that the largest weight so far is 2^-15 and a later one can
// be 2^16 times as large before the maximum moves.  Less than kBias: exponents of the largest weights are good to half a step
// at 15, 2^-21 (of numbers around 39 it is 2^-19), which the log-sum-exp shows, and products with the smallest values that
// a page holds, 2^-109, stay normal numbers.
constexpr float kTileBias = 15.0f;
constexpr int kTileDown = 4;  // value_exp: beside the bias, for rows of 2^19 keys
enum TilePlace { kFirst = 0, kInner = 1, kLast = 2 };

// x of the wave's two 32-lane halves (lane l and lane l ^ 32) added up.
__device__ __forceinline__ float half_sum(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// The online softmax of one tile, as softmax_tile of attn_kernels.hip: the running maximum stays while the weights of
// no lane add up to 2, nor to more than kDominant times what the row has.  So a key that dominates a row moves the maximum to
// itself, and its weight is a power of two, which the product's 16 bits hold: O is its value as it is, though l sums the
// weights before they are rounded.  The test takes 0.7 % (1560 rows x 32760 keys x 12 heads, d = 128, 290 -> 292 us; 293 with its
// limit formed behind the weights), each move another tile's time: the cost goes by how far scores spread.  1536 rows x 16384
// keys x 12 heads, scores of standard deviation 1, 2, 3 and 5, in us without it, with 16 times, with 2 times:
//   d = 128   159 161 162 165    161 162 166 179    160 165 178 196
//   d = 64    105 105 105 108    105 105 109 130    106 109 127 140
// Dividing by sums of the rounded weights instead, from the matrix core as in attn_kernels.hip beside these, takes 2.5 to 5 %
// more time for any scores.  l: the row sum over the lane's half of the keys.
constexpr float kDominant = 16.0f;

template <int D, int kPlace, int kHooks, int kEvery, typename Issue>
__device__ __forceinline__ void tile_softmax(f32x16 (&s)[Geo<D>::kBN / 32], bf16x8 (&p)[Geo<D>::kBN / 16],
                                             float& m_c, float& l, f32x16 (&o)[D / 32], float c, int keys,
                                             int lane, Issue&& issue) {
  constexpr int kBN = Geo<D>::kBN;
  const int hb = lane >> 5;
  if (kPlace == kInner) {
    float before = l;
    __asm__ volatile("" : "+v"(before));  // (l itself, when it is tested here, has the compiler spill 40 to 120 registers)
    // of the row: a lane's own is next to nothing where the other one's keys hold the row
    float limit = fminf(2.0f, kDominant * half_sum(before));
    __asm__ volatile("" : "+v"(limit));
    const float sum = exp_pack<kBN / 16, kHooks, kEvery>(s, p, m_c, c, issue);
    if (__builtin_amdgcn_ballot_w64(!(sum < limit)) == 0) {  // (NaN and infinities among them)
      l += sum;
      return;
    }
  }
  if (kPlace == kLast) {
#pragma unroll
    for (int kb = 0; kb < kBN / 32; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (32 * kb + 8 * (r >> 2) + 4 * hb + (r & 3) >= keys) s[kb][r] = -INFINITY;
  }
  float mt = s[0][0];
#pragma unroll
  for (int kb = 0; kb < kBN / 32; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) mt = fmaxf(mt, s[kb][r]);
  mt = half_max(mt);
  const float m_new = fmaxf(m_c, __builtin_fmaf(mt, c, kTileBias));
  if (kPlace != kFirst) {
    const float alpha = __builtin_amdgcn_exp2f(m_c - m_new);  // 0 where m_c = -inf
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[db][r] *= alpha;
    l *= alpha;
  }
  m_c = m_new;
  l += kPlace == kInner ? exp_pack<kBN / 16, 0, 1>(s, p, m_c, c, NoHook{})
                        : exp_pack<kBN / 16, kHooks, kEvery>(s, p, m_c, c, issue);
}

// O = O / l of a wave's 32 rows, through LDS so that whole lines are stored (as write_result of
// attn_kernels.hip), and the rows' log-sum-exp.
template <int D, Out kOut>
__device__ __forceinline__ void write_rows(const TileItem& it, const RowArgs& a, const f32x16 (&oacc)[D / 32],
                                           float l, float m_c, int q0, lds_char* stage, int lane) {
  using G = Geo<D>;
  const int col = lane & 31, hb = lane >> 5, H = a.pool.H;
  const float inv = l == 0.0f ? 0.0f : (float)(1 << kTileDown) / l;
  const int orow = lane >> 3, ochunk = lane & 7;
  lds_char* const put = stage + col * G::kORow;
  const lds_char* const get = stage + orow * G::kORow + ochunk * 16;
  auto in_order = [] { __asm__ volatile("" ::: "memory"); };
  constexpr bool kPartial = kOut != kResult;
  const int64_t slab = kOut == kSlab ? (int64_t)it.split * a.ss.total * (H * a.G) : 0;
  auto place = [&](int r) {
    return kOut == kSlot ? (int64_t)it.slot * kBM + (r - it.row0) : slab + row_of(it.se, r, it.h, H, a.G);
  };
  int64_t at[4];  // rows that this lane stores
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int r = q0 + orow + 8 * u;
    at[u] = r < it.rows ? place(r) : -1;
  }
  constexpr int kBlocks = kPartial ? 1 : 2;  // 32-channel blocks of a pass: 128 bytes of each row
#pragma unroll
  for (int d0 = 0; d0 < D / 32; d0 += kBlocks) {
#pragma unroll
    for (int db = d0; db < d0 + kBlocks; ++db)
#pragma unroll
      for (int g4 = 0; g4 < 4; ++g4) {
        const f32x4 x = {oacc[db][4 * g4] * inv, oacc[db][4 * g4 + 1] * inv, oacc[db][4 * g4 + 2] * inv,
                         oacc[db][4 * g4 + 3] * inv};
        const int ch = 32 * (db - d0) + 8 * g4 + 4 * hb;
        if (kPartial) *(lds_u32x4*)(put + ch * 4) = __builtin_bit_cast(u32x4, x);
        else *(lds_u32x2*)(put + ch * 2) = __builtin_bit_cast(u32x2, __builtin_convertvector(x, bf16x4));
      }
    in_order();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const u32x4 x = *(const lds_u32x4*)(get + 8 * u * G::kORow);
      if (at[u] >= 0) {
        if (kPartial) *(u32x4*)((char*)(a.part_o + at[u] * D + 32 * d0) + ochunk * 16) = x;
        else *(u32x4*)((char*)(a.o + at[u] * D + 32 * d0) + ochunk * 16) = x;
      }
    }
    in_order();
  }
  float* const lse = kPartial ? a.part_lse : a.lse;
  if (lse != nullptr && hb == 0 && q0 + col < it.rows)
    // the bias is taken out of both terms first: numbers of its size that cancel would leave their rounding
    lse[place(q0 + col)] =
        l == 0.0f ? -INFINITY : ((m_c - kTileBias) + __builtin_amdgcn_logf(l * (float)(1 << (int)kTileBias))) * kLn2;
}

// How the work is dealt to workgroups: an item each (find_item), whole or in n_split ranges of keys; or equal shares of it
// (Work below).
enum Mode { kWhole, kSplit, kEven };

// kActive = false: a wave whose rows all lie past the session's: it fetches its share and keeps the barriers.
template <int D, bool kGroupB, Mode kMode, bool kActive>
__device__ __forceinline__ void run_tile_group(const TileItem& it, const RowArgs& a, char* smem) {
  using G = Geo<D>;
  using T = TileGeo<D>;
  constexpr int kBN = G::kBN, kPre = T::kPre;
  const int tid = thread_anew(), lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int gw = wave & (G::kGroupWaves - 1);
  const int H = a.pool.H;
  lds_char* const lds = (lds_char*)smem;
  auto ktile = [&](int stage) { return lds + T::kKRing + stage * G::kKTile; };
  auto vtile = [&](int stage) { return lds + T::kVRing + stage * G::kVTile; };
  VOffsets<D> vo(lane);  // in the V stage that the next matrix step reads

  // ---- fetching
  const uint8_t* const bytes = (kGroupB ? a.pool.v : a.pool.k) + (int64_t)it.h * (kPage * D);
  const uint8_t* const exps = kGroupB ? a.pool.v_exp : a.pool.k_exp;
  const int len = it.se.len, pages = (len + kPage - 1) / kPage;
  const int first = it.tile_begin * T::kPages;  // page index of the item's first tile
  // The group's list of pages in LDS, entry i mod kEntries the item's i-th page: filled in the prologue, and its halves
  // renewed in turn as the item moves on, an entry a lane of the group.
  typedef __attribute__((address_space(3))) u32x2 lds_entry;
  lds_char* const list = lds + T::kList + (kGroupB ? T::kEntries * 8 : 0);
  constexpr int kHalf = T::kEntries / 2;
  static_assert(kHalf == 64 * G::kGroupWaves, "an entry a lane");
  auto page_id = [&](int i) { return first + i < pages ? it.table[first + i] : 0; };
  auto put_entry = [&](int i, int id) {
    const bool bad = (unsigned)id >= (unsigned)a.pool.pages;
    const unsigned e = exps[(int64_t)(bad ? 0 : id) * H + it.h];
    const unsigned exp = bad ? 255u : first + i < pages ? e : 127u, scale = (kGroupB ? value_exp(exp, kTileDown) : exp) << 23;
    *(lds_entry*)(list + (i & (T::kEntries - 1)) * 8) = u32x2{bad ? 0u : (unsigned)id, scale};
  };
  {
    const int i = 64 * gw + lane, id0 = page_id(i), id1 = page_id(i + kHalf);
    put_entry(i, id0);
    put_entry(i + kHalf, id1);
  }
  wait_lds();
  block_sync();  // the list is there
  // Tile j's bytes, into registers: load u of a lane covers bytes 1024 n + 16 lane of the tile, n = gw + 4 u;
  // at d = 128 both lie in the one page, at d = 64 load u in page u.  Its entries are read well before.
  u32x4 raw[T::kLoads];
  unsigned scale[T::kPages];
  u32x2 entry[T::kPages];
  auto read_entries = [&](int j) {
#pragma unroll
    for (int x = 0; x < T::kPages; ++x)
      entry[x] = *(const lds_entry*)(list + ((j * T::kPages + x) & (T::kEntries - 1)) * 8);
  };
  const int lane_byte = 1024 * gw + 16 * lane;
  auto load = [&](int j, int u) {
    const int x = T::kPages == 2 ? u : 0;
    const int id = __builtin_amdgcn_readfirstlane((int)entry[x][0]);
    // tokens of the page (rows past them read as zeros); a scalar, as the descriptor has to be
    const int n = __builtin_amdgcn_readfirstlane(max(0, min(kPage, len - (first + j * T::kPages + x) * kPage)));
    __amdgpu_buffer_rsrc_t r = make_rsrc(bytes + (int64_t)id * H * (kPage * D), (uint32_t)(n * D));
    raw[u] = __builtin_amdgcn_raw_buffer_load_b128(r, lane_byte + (T::kPages == 2 ? 0 : 4096 * u), 0, 0);
    if (T::kPages == 2 || u == 0) scale[x] = __builtin_amdgcn_readfirstlane(entry[x][1]);
  };
  // Half of load u's 16 elements, widened (times sc), to its place in the tile's LDS image.
  const int row0 = lane_byte / D, chunk0 = lane % (D / 16) * 2;
  auto put = [&](lds_char* tile, int u, int half, unsigned sc) {
    const int row = row0 + u * (4096 / D);
    const bf16x8 x = widen8(raw[u][2 * half], raw[u][2 * half + 1], __uint_as_float(sc));
    lds_char* const to = kGroupB ? tile + row * G::kVRow + (((chunk0 + half) ^ G::vswz(row)) << 4)
                                 : tile + row * G::kKRow + ((chunk0 + half) << 4);
    *(lds_bf16x8*)to = x;
  };
  // Renews half of the list when the tiles about to be fetched (tile j next) enter its other half: the page numbers
  // first, the entries, which need the numbers to find the exponents, half way through.
  int fresh = 0;
  auto renew = [&](int j) {
    const int i = j * T::kPages, in_half = i & (kHalf - 1);
    if (i >= kHalf && in_half == 0) fresh = page_id(i + kHalf + 64 * gw + lane);
    if (i >= kHalf && in_half == kHalf / 2) put_entry(i + kHalf / 2 + 64 * gw + lane, fresh);
  };
  constexpr int kAhead = kGroupB ? 1 : 2;  // tiles between a vector step and the tile it writes

  // ---- prologue: the first tiles' images, the next one's bytes, the wave's query rows
  {
    const int qrow0 = it.row0 + 32 * wave;
    if constexpr (kActive) {
      const int last = it.rows - 1, step = H * a.G * D * 2;
      const int t_last = a.G == 1 ? last : last / a.G;
      __amdgpu_buffer_rsrc_t rq =
          make_rsrc(a.q + ((int64_t)it.se.q0 * (H * a.G) + it.h * a.G) * D,
                    (uint32_t)t_last * (uint32_t)step + (uint32_t)(last - t_last * a.G + 1) * (D * 2));
#pragma unroll
      for (int n = 0; n < G::kQWave / 1024; ++n) {
        const int row = (64 * n + lane) / G::kChunks;
        const int chunk = (lane % G::kChunks) ^ (D == 128 ? row & 15 : (row >> 1) & 7);
        const int r = qrow0 + row, t = a.G == 1 ? r : r / a.G;
        dma16(rq, lds + T::kQBase + wave * G::kQWave + 1024 * n, t * step + (r - t * a.G) * (D * 2) + chunk * 16);
      }
    }
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      read_entries(j);
#pragma unroll
      for (int u = 0; u < T::kLoads; ++u) load(j, u);
#pragma unroll
      for (int u = 0; u < T::kLoads; ++u)
#pragma unroll
        for (int half = 0; half < 2; ++half)
          put(kGroupB ? vtile(j) : ktile(j), u, half, scale[T::kPages == 2 ? u : 0]);
    }
    read_entries(kAhead);
#pragma unroll
    for (int u = 0; u < T::kLoads; ++u) load(kAhead, u);
  }
  bf16x8 qf[D / 16] = {};
  if constexpr (kActive) {
    wait_vmem<0>();
    __asm__ volatile("" ::: "memory");
    const lds_char* const stage = lds + T::kQBase + wave * G::kQWave;
    const int row = lane & 31, hb = lane >> 5;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      const u32x4 x = *(const lds_u32x4*)(stage + row * D * 2 +
                                          (((2 * kk + hb) ^ (D == 128 ? row & 15 : (row >> 1) & 7)) << 4));
      qf[kk] = __builtin_bit_cast(bf16x8, x ^ u32x4{a.flip, a.flip, a.flip, a.flip});
    }
  }
  wait_lds();
  block_sync();

  f32x16 oacc[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db) oacc[db] = f32x16{};
  f32x16 s[kBN / 32];
  bf16x8 p[kBN / 16];
  bf16x8 kp[kPre];
  f32x4 unused[2] = {};  // row sums of m_step
  float m_c = -INFINITY, l = 0.0f;
  const int ntiles = it.ntiles;
  const int last_keys = min(kBN, len - (it.tile_begin + ntiles - 1) * kBN);
  if constexpr (kActive) k_preread<D, kPre>(ktile(0), kp, lane);
  if (kGroupB) block_sync();  // group B starts one step behind

  // Vector step j: the softmax of tile j, and in four places of it the image of the tile fetched a step ago (each
  // a quarter), a load of the next tile's bytes wherever its registers have come free.  `stage`: where the image goes.
  constexpr int kHooks = 4, kEvery = kBN / 16;
  auto vstep = [&](int j, int stage, auto place) {
    constexpr int kPlace = decltype(place)::value;
    lds_char* const to = kGroupB ? vtile(stage) : ktile(stage);
    renew(j + kAhead + 1);
    read_entries(j + kAhead + 1);
    const unsigned was = scale[0];  // of the bytes in the registers (at d = 64, where load 1 has its own, of load 0)
    auto hook = [&](int i) {
      put(to, i >> 1, i & 1, i >> 1 && T::kPages == 2 ? scale[T::kPages - 1] : was);
      if (i & 1) load(j + kAhead + 1, i >> 1);
    };
    if constexpr (kActive) {
      tile_softmax<D, kPlace, kHooks, kEvery>(s, p, m_c, l, oacc, a.c, last_keys, lane, hook);
    } else {
#pragma unroll
      for (int i = 0; i < kHooks; ++i) hook(i);
    }
    wait_lds();
    if (kActive && kPlace != kLast) k_preread<D, kPre>(ktile((j + 1) % T::kKStages), kp, lane);
  };
  using First = std::integral_constant<int, kFirst>;
  using Inner = std::integral_constant<int, kInner>;
  using Last = std::integral_constant<int, kLast>;
  // stages of K_j and of the tile that vector step j writes
  int ks = 0;
  auto write_stage = [&](int j) { return kGroupB ? (j + 1) & 1 : ks == 0 ? 2 : ks - 1; };  // (j + 2) % 3

  if constexpr (kActive) {
    __builtin_amdgcn_s_setprio(1);
    m_step<D, false, false, kPre>(ktile(0), lds, vo, qf, kp, s, p, oacc, bf16x8{}, unused, lane);
    __builtin_amdgcn_s_setprio(0);
  }
  block_sync();
  auto vector = [&](int j, auto place) { vstep(j, write_stage(j), place); };
  if (ntiles == 1) vector(0, Last{});
  else vector(0, First{});
  auto tile = [&](int j, auto place) {
    ks = ks == 2 ? 0 : ks + 1;
    block_sync();  // closes V(j - 1)
    if constexpr (kActive) {
      __builtin_amdgcn_s_setprio(1);
      m_step<D, true, false, kPre>(ktile(ks), lds, vo, qf, kp, s, p, oacc, bf16x8{}, unused, lane);
      __builtin_amdgcn_s_setprio(0);
#pragma unroll
      for (int r2 = 0; r2 < 2; ++r2)
#pragma unroll
        for (int db = 0; db < D / 32; ++db) vo.off[r2][db] ^= G::kVTile;
    }
    block_sync();
    vector(j, place);
  };
  int j = 1;
  for (; j < ntiles - 1; ++j) tile(j, Inner{});
  if (j == ntiles - 1) tile(j, Last{});
  block_sync();  // closes V(ntiles - 1)
  if constexpr (kActive) pv_tile<D>(lds, vo, p, oacc);
  if (!kGroupB) block_sync();  // matches group B's extra barrier at the start

  if constexpr (kActive) {
    l = half_sum(l);
    const int q0 = it.row0 + 32 * wave;
    lds_char* const stage = lds + T::kOBase + wave * G::kOWave;
    if constexpr (kMode != kEven) write_rows<D, kMode == kSplit ? kSlab : kResult>(it, a, oacc, l, m_c, q0, stage, lane);
    else if (it.slot < 0) write_rows<D, kResult>(it, a, oacc, l, m_c, q0, stage, lane);
    else write_rows<D, kSlot>(it, a, oacc, l, m_c, q0, stage, lane);
  }
}

// The item of a workgroup.  A session has H x n_split x ceil(rows / 256) items, head-major, then by page range, then
// by row tile, so that neighbours read the same keys.  The hardware deals workgroups to the eight XCDs in turn,
// workgroup b to XCD b % 8, and an XCD starts its own in order.  Every XCD gets a consecutive eighth of each
// session's items (what is left over goes to the XCDs in turn, from session to session), so an eighth of the
// keys passes through its L2, and the XCDs have equal work; within an XCD the longest sessions come first, so
// that it ends evenly.  Up to 64 sessions are put in order by every wave itself, one per lane; more keep their order.
// (Spans of 8 x 32 items dealt over the XCDs instead leave the first ones all the long items: six sessions of 2730 to
// 32760 keys x 1560 queries x 12 heads took 1.12 times as long.)
struct Share {  // of a session's `count` items, `before` items of earlier sessions: this XCD's
  int n, first;
  __device__ __forceinline__ Share(int count, int before, int xcd) {
    const int y = (xcd - before) & 7, q = count >> 3, r = count & 7;
    n = q + (y < r ? 1 : 0);
    first = y * q + min(y, r);
  }
};

//
// There are as many workgroups as disjoint sessions can have items (attn_items).  Where offsets run backwards, sessions can
// name rows that others have too, and their items be more: then (crossed, in some lane) every workgroup goes on to the item
// that comes a grid later.  A session's items are less than 2^23, so that those of 64 fit 32 bits.
__device__ __forceinline__ bool crossed(const Sessions& ss) {
  bool back = false;
  for (int s = threadIdx.x & 63; s < ss.nseq; s += 64) back |= ss.cu[s + 1] < ss.cu[s];
  return back;
}

// The at-th item of this workgroup's XCD.
template <int D>
__device__ __forceinline__ bool find_item(const RowArgs& a, int64_t at, TileItem* it) {
  const int lane = thread_anew() & 63, per_tile = a.pool.H * a.n_split;
  const int xcd = blockIdx.x & 7;
  auto items_of = [&](const Session& se) {
    return se.ok ? per_tile * (int)(((int64_t)se.rows * a.G + kBM - 1) / kBM) : 0;
  };
  int s = -1, local = 0;
  if (a.ss.nseq <= 64) {
    Session mine{};
    if (lane < a.ss.nseq) mine = session_of(a.ss, lane);
    const int count = lane < a.ss.nseq ? items_of(mine) : 0;
    auto earlier = [&](int i, int li) { return li > mine.len || (li == mine.len && i < lane); };
    int before = 0, start = 0;
    for (int i = 0; i < a.ss.nseq; ++i)
      before += earlier(i, __builtin_amdgcn_readlane(mine.len, i)) ? __builtin_amdgcn_readlane(count, i) : 0;
    const Share share(count, before, xcd);
    for (int i = 0; i < a.ss.nseq; ++i)
      start += earlier(i, __builtin_amdgcn_readlane(mine.len, i)) ? __builtin_amdgcn_readlane(share.n, i) : 0;
    const unsigned long long hit = __builtin_amdgcn_ballot_w64(start <= at && at - start < share.n);
    if (hit != 0) {
      s = __builtin_ctzll(hit);
      local = (int)at - __builtin_amdgcn_readlane(start, s) + __builtin_amdgcn_readlane(share.first, s);
    }
  } else {
    auto scan = [&](int x) {  // inclusive, over the lanes
#pragma unroll
      for (int m = 1; m < 64; m <<= 1) {
        const int y = __shfl_up(x, m);
        if (lane >= m) x += y;
      }
      return x;
    };
    unsigned items = 0;  // of the sessions so far, modulo 8
    int64_t base = 0;    // of them, this XCD's
    for (int s0 = 0; s0 < a.ss.nseq && s < 0; s0 += 64) {
      const int count = s0 + lane < a.ss.nseq ? items_of(session_of(a.ss, s0 + lane)) : 0;
      const int counts = scan(count);
      const Share share(count, (int)(items & 7) + counts - count, xcd);
      const int shares = scan(share.n);
      const int64_t start = base + (shares - share.n);
      const unsigned long long hit = __builtin_amdgcn_ballot_w64(start <= at && at - start < share.n);
      if (hit != 0) {
        const int i = __builtin_ctzll(hit);
        s = s0 + i;
        local = (int)(at - base) - __builtin_amdgcn_readlane(shares - share.n, i) + __builtin_amdgcn_readlane(share.first, i);
      }
      items += (unsigned)__builtin_amdgcn_readlane(counts, 63);
      base += __builtin_amdgcn_readlane(shares, 63);
    }
  }
  if (s < 0) return false;
  // everything about the item is the same in all lanes: in scalar registers
  s = __builtin_amdgcn_readfirstlane(s);
  local = __builtin_amdgcn_readfirstlane(local);
  it->se = session_of(a.ss, s);
  it->se.q0 = __builtin_amdgcn_readfirstlane(it->se.q0);
  it->se.rows = __builtin_amdgcn_readfirstlane(it->se.rows);
  it->se.len = __builtin_amdgcn_readfirstlane(it->se.len);
  it->table = a.ss.table + (int64_t)s * a.ss.width;
  it->rows = it->se.rows * a.G;
  const int nq = (it->rows + kBM - 1) / kBM, per_head = nq * a.n_split;
  it->h = __builtin_amdgcn_readfirstlane(small_div(local, per_head));
  local -= it->h * per_head;
  it->split = a.n_split == 1 ? 0 : __builtin_amdgcn_readfirstlane(small_div(local, nq));
  it->row0 = (local - it->split * nq) * kBM;
  const int tiles = (it->se.len + Geo<D>::kBN - 1) / Geo<D>::kBN;
  const int per = a.n_split == 1 ? tiles : __builtin_amdgcn_readfirstlane((tiles + a.n_split - 1) / a.n_split);
  it->tile_begin = it->split * per;
  it->ntiles = max(0, min(per, tiles - it->tile_begin));
  it->slot = -1;
  return true;
}

// A last tile of at most twice kThinRows rows is shared by the eight waves, each taking pages of its own (rows_item): in
// the schedule above one wave would work and seven keep its barriers, for three quarters of a full tile's time (32768
// keys, d = 128: 201 us for 24 rows this way, 566 for 100, 710 for 256); six sessions of 16384 keys x 300 rows x 12 heads take
// 258 us, and 318 with their 44 rows in the schedule above.  Calls of up to 64 rows that come here at all (call_tile) do so for that
// schedule, in a kernel of their own whose thin tiles (kThin) end at kThinRows: as an argument the limit costs the other
// calls up to 4 %.
constexpr int kThinRows = 32;

template <int D>
constexpr int tiles_lds() {
  return TileGeo<D>::kLds > RowGeo<D, kThinRows / 16, kWaves>::kLds ? TileGeo<D>::kLds
                                                                   : RowGeo<D, kThinRows / 16, kWaves>::kLds;
}

constexpr int kStateBytes = 32;  // where a share stands (kEven)

// Equal shares.  Items as they come, the sessions' in their order and of each head-major, cost kStartCost and their tiles,
// less where the last rows leave waves idle; share i of P has [i S, (i + 1) S) of their sum, S = sum / P but at least
// kShareMin: whole items, and the parts of those that a border cuts.  A cut is at a tile, and none within kCutMin tiles
// of an item's ends (it moves there).  What a share has of a cut item goes to
// one of its two slots: 2 i, if the item began in an earlier share, else 2 i + 1; cache_join_kernel joins them.
// Consecutive eighths of the shares go to the XCDs.  Against whole row tiles, or as many ranges of each as fill the device
// when all sessions have the stated length: 257 .. 640 odd rows x 777 .. 20011 keys x 12 heads x 2, d = 64, 152 -> 119 us; six
// sessions of 2730 to 32760 keys 961 -> 923.  But the workgroups of an XCD no longer read the same keys at one time: one session
// of 32760 keys x 1560 rows x 12 heads, whose row tiles in three ranges just fill the device, took 302 us instead of 294,
// so a call of one session takes shares only where ranges leave a sixth idle; and finding a share takes 10 us, so
// small calls take none (attn_parts).
struct Spot {
  int s, h, tile, t;  // session, head, row tile, key tile of it (0 unless the spot is inside an item)
  int64_t from;       // where its item begins
  __device__ __forceinline__ bool before(const Spot& o) const {
    if (s != o.s) return s < o.s;
    if (h != o.h) return h < o.h;
    return tile != o.tile ? tile < o.tile : t < o.t;
  }
};

__device__ __forceinline__ void next_item(Spot& p, int nq, int H) {
  p.t = 0;
  if (++p.tile < nq) return;
  p.tile = 0;
  if (++p.h < H) return;
  p.h = 0, ++p.s;
}

// The share of a workgroup: consecutive eighths to the XCDs (workgroup b runs on XCD b % 8).
__device__ __forceinline__ int share_of_block() {
  return (blockIdx.x & 7) * (gridDim.x >> 3) + (blockIdx.x >> 3);
}

// The kernel's arguments, read from memory at this point.
__device__ __forceinline__ RowArgs args_anew() {
  typedef __attribute__((address_space(4))) const uint64_t const_word;
  struct Words {
    uint64_t w[sizeof(RowArgs) / 8];
  } x;
  uintptr_t p = (uintptr_t)__builtin_amdgcn_kernarg_segment_ptr();
  __asm__ volatile("" : "+s"(p));
#pragma unroll
  for (unsigned i = 0; i < sizeof(x) / 8; ++i) x.w[i] = ((const_word*)p)[i];
  return __builtin_bit_cast(RowArgs, x);
}

template <int D>
struct Work {
  const RowArgs& a;
  int64_t sum, share;
  int64_t cost, to;  // of up to 64 sessions, one a lane: its cost, and where it ends

  struct Shape {  // of a session: key tiles, row tiles, costs of a row tile, of the last one, and of a head
    int tiles, nq;
    int part;  // 20ths of a full tile's time that the last one takes: 24, 100 and 256 rows measured
    int cost, last;
    int64_t head;
    __device__ __forceinline__ Shape(const Session& se, int G) {
      const int rows = se.rows * G;
      tiles = (se.len + Geo<D>::kBN - 1) / Geo<D>::kBN;
      nq = (rows + kBM - 1) / kBM;
      cost = tiles + kStartCost;
      const int active = (rows - (nq - 1) * kBM + 31) / 32;  // waves
      part = active <= 2 ? 8 * active : 12 + active;
      last = (int)((int64_t)tiles * part / 20) + kStartCost;
      head = (int64_t)(nq - 1) * cost + last;
    }
    // the tile at which a border `in` past the item's start cuts it: 0 and `tiles` are its ends
    __device__ __forceinline__ int cut(int tile, int in) const {
      const int t = tile == nq - 1 ? (int)((int64_t)(in - kStartCost) * 20 / part) : in - kStartCost;
      return t < kCutMin ? 0 : tiles - t < kCutMin ? tiles : t;
    }
  };
  __device__ __forceinline__ int64_t cost_of(int s) const {
    if (s >= a.ss.nseq) return 0;
    const Session se = session_of(a.ss, s);
    return se.rows > 0 ? Shape(se, a.G).head * a.pool.H : 0;
  }
  // of numbers that are not negative; most fit 32 bits, in which the division takes a fourth of the time
  static __device__ __forceinline__ int64_t quotient(int64_t x, int64_t y) {
    return (uint64_t)(x | y) >> 32 == 0 ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
  }
  static __device__ __forceinline__ int64_t scan(int64_t x, int lane) {  // inclusive, over the lanes
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
      const int64_t y = __shfl_up(x, m);
      if (lane >= m) x += y;
    }
    return x;
  }
  __device__ __forceinline__ Work(const RowArgs& args) : a(args) {
    const int lane = threadIdx.x & 63;
    sum = 0;
    for (int s0 = 0; s0 < a.ss.nseq; s0 += 64) {
      cost = cost_of(s0 + lane);
      to = sum + scan(cost, lane);
      sum = __shfl(to, 63);
    }
    const int64_t each = quotient(sum + a.shares - 1, a.shares);
    share = each > kShareMin ? each : kShareMin;
  }
  __device__ __forceinline__ Spot at(int64_t x) const {
    const int lane = threadIdx.x & 63;
    Spot p{a.ss.nseq, 0, 0, 0, sum};
    if (x >= sum) return p;
    auto find = [&](int s0, int64_t cost, int64_t to) {
      const unsigned long long hit = __builtin_amdgcn_ballot_w64(x < to);
      if (hit == 0) return false;
      const int i = __builtin_ctzll(hit);  // the first that ends past x
      p.s = s0 + i, p.from = __shfl(to - cost, i);
      return true;
    };
    if (a.ss.nseq <= 64) {
      find(0, cost, to);
    } else {
      int64_t base = 0;
      for (int s0 = 0; s0 < a.ss.nseq; s0 += 64) {
        const int64_t c = cost_of(s0 + lane), t = base + scan(c, lane);
        if (find(s0, c, t)) break;
        base = __shfl(t, 63);
      }
    }
    const Shape sh(session_of(a.ss, p.s), a.G);
    p.h = (int)quotient(x - p.from, sh.head);
    p.from += p.h * sh.head;
    const int64_t tile = quotient(x - p.from, sh.cost);
    p.tile = tile < sh.nq ? (int)tile : sh.nq - 1;
    p.from += (int64_t)p.tile * sh.cost;
    p.t = sh.cut(p.tile, (int)(x - p.from));
    if (p.t > 0 && p.t == sh.tiles) next_item(p, sh.nq, a.pool.H);
    return p;
  }
};

template <int D, Mode kMode>
constexpr Out out_of() { return kMode == kEven ? kSlot : kMode == kSplit ? kSlab : kResult; }

// An item without keys: zeros, or nothing but the log-sum-exp of an empty range.
template <int D, Mode kMode>
__device__ __forceinline__ void run_empty(const TileItem& it, const RowArgs& a) {
  constexpr Out kOut = out_of<D, kMode>();
  const int n = min(it.rows - it.row0, kBM), H = a.pool.H;
  float* const lse = kOut == kSlab ? a.part_lse + (int64_t)it.split * a.ss.total * (H * a.G) : a.lse;
  for (int i = thread_anew(); i < n * (D / 8); i += kThreads) {
    const int64_t at = row_of(it.se, it.row0 + i / (D / 8), it.h, H, a.G);
    if (kOut != kSlab) *(u32x4*)(a.o + at * D + i % (D / 8) * 8) = u32x4{};
    if (lse != nullptr && i % (D / 8) == 0) lse[at] = -INFINITY;
  }
}

// An item's rows, kThinRows at a time, by waves that take pages of their own.
template <int D, Mode kMode>
__device__ __forceinline__ void run_thin(const TileItem& it, const RowArgs& a, char* smem) {
  const int begin = it.tile_begin * TileGeo<D>::kPages, row_end = min(it.rows, it.row0 + kBM);
  const int end = min((it.se.len + kPage - 1) / kPage, begin + it.ntiles * TileGeo<D>::kPages);
  const int id = first_ids<kWaves>(it.table, a.ss.width, begin, 1);
  for (int row0 = it.row0; row0 < row_end; row0 += kThinRows) {
    const int slot = it.slot < 0 ? -1 : it.slot * kBM + row0 - it.row0;
    if (row0 > it.row0) __syncthreads();  // every wave is done with the rows before
    rows_item<D, kThinRows / 16, kWaves, out_of<D, kMode>()>(a, it.se, it.table, it.h, row0, it.rows, {begin, 1, end}, id,
                                                             kMode == kEven ? slot : it.split, smem);
  }
}

template <int D, Mode kMode, int kThin>
__device__ __forceinline__ void run_item(const TileItem& it, const RowArgs& a, char* smem) {
  const int wave = __builtin_amdgcn_readfirstlane(thread_anew() >> 6);
  if (it.ntiles <= 0) return run_empty<D, kMode>(it, a);
  if (it.rows - it.row0 <= kThin) return run_thin<D, kMode>(it, a, smem);
  const bool active = it.row0 + 32 * wave < it.rows;
  if (wave >= kWaves / 2) {
    if (active) run_tile_group<D, true, kMode, true>(it, a, smem);
    else run_tile_group<D, true, kMode, false>(it, a, smem);
  } else {
    if (active) run_tile_group<D, false, kMode, true>(it, a, smem);
    else run_tile_group<D, false, kMode, false>(it, a, smem);
  }
}

template <int D, Mode kMode, int kThin = 2 * kThinRows>
__global__ void __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
cache_tiles_kernel(RowArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  if constexpr (kMode != kEven) {
    TileItem it;
    const bool back = crossed(a.ss);  // (asked for with the sessions, looked at behind them)
    if (!find_item<D>(a, blockIdx.x >> 3, &it)) return;
    const bool more = __builtin_amdgcn_ballot_w64(back) != 0;
    run_item<D, kMode, kThin>(it, a, smem);
    if (!more) return;
    // The items that are left where sessions share rows, by the thin path whatever their rows: run_item in a loop would have
    // the registers of every call's items hold what the next one needs (4680 rows x 32760 keys x 40 heads, d = 128: 3030
    // instead of 2706 us).
    for (int64_t at = (blockIdx.x >> 3) + (gridDim.x >> 3);; at += gridDim.x >> 3) {
      __syncthreads();  // every wave is done with the last item's LDS
      const RowArgs b = args_anew();
      if (!find_item<D>(b, at, &it)) return;
      if (it.ntiles <= 0) run_empty<D, kMode>(it, b);
      else run_thin<D, kMode>(it, b, smem);
    }
  }
  // Between items the share's place is in LDS and the arguments are read again: held in scalar registers through the
  // items, they leave the scheduler without room (the matrix step's reads then wait for each other).
  typedef __attribute__((address_space(3))) int lds_int;
  lds_int* const state = (lds_int*)((lds_char*)smem + tiles_lds<D>());  // Spot p, Spot end
  {
    const Work<D> work(a);
    const int64_t x = share_of_block() * work.share;
    if (x >= work.sum) return;
    const Spot p = work.at(x), end = work.at(x + work.share);
    if (threadIdx.x == 0) {
      state[0] = p.s, state[1] = p.h, state[2] = p.tile, state[3] = p.t;
      state[4] = end.s, state[5] = end.h, state[6] = end.tile, state[7] = end.t;
    }
  }
  for (;;) {
    __syncthreads();  // the state is there, and every wave is done with the last item's LDS
    int base = (int)(uintptr_t)state;
    __asm__ volatile("" : "+v"(base));
    auto word = [&](int n) { return __builtin_amdgcn_readfirstlane(*(lds_int*)(uintptr_t)(unsigned)(base + 4 * n)); };
    Spot p{word(0), word(1), word(2), word(3), 0};
    const Spot end{word(4), word(5), word(6), word(7), 0};
    if (!p.before(end)) return;
    const RowArgs b = args_anew();
    TileItem it;
    it.se = session_of(b.ss, p.s);
    it.se.q0 = __builtin_amdgcn_readfirstlane(it.se.q0);
    it.se.rows = __builtin_amdgcn_readfirstlane(it.se.rows);
    it.se.len = __builtin_amdgcn_readfirstlane(it.se.len);
    it.rows = it.se.rows * b.G;
    const int tiles = (it.se.len + Geo<D>::kBN - 1) / Geo<D>::kBN;
    const bool last = p.s == end.s && p.h == end.h && p.tile == end.tile;
    it.table = b.ss.table + (int64_t)p.s * b.ss.width;
    it.h = p.h, it.row0 = p.tile * kBM, it.split = 0;
    it.tile_begin = p.t, it.ntiles = (last ? end.t : tiles) - p.t;
    it.slot = it.ntiles == tiles ? -1 : 2 * share_of_block() + (p.t > 0 ? 0 : 1);
    const int nq = (it.rows + kBM - 1) / kBM;
    const bool none = it.se.rows == 0;
    if (none) p = {p.s + 1, 0, 0, 0, 0};
    else if (last) p = end;
    else next_item(p, nq, b.pool.H);
    __syncthreads();  // every wave has read the state
    if (threadIdx.x == 0) state[0] = p.s, state[1] = p.h, state[2] = p.tile, state[3] = p.t;
    if (!none) run_item<D, kEven, kThin>(it, b, smem);
  }
}

// Joins the parts of the items that the shares have cut: kJoinBlocks workgroups to a border between shares, the first of
// those inside its item.
constexpr int kJoinBlocks = 8;

template <int D>
__global__ void __launch_bounds__(kMergeThreads) cache_join_kernel(RowArgs a) {
  const Work<D> work(a);
  const int b = blockIdx.x / kJoinBlocks + 1;
  if (b * work.share >= work.sum) return;
  const Spot p = work.at(b * work.share);
  if (p.t == 0) return;
  const Session se = session_of(a.ss, p.s);
  const typename Work<D>::Shape sh(se, a.G);
  const int rows = se.rows * a.G, row0 = p.tile * kBM;
  const int64_t cost = p.tile == sh.nq - 1 ? sh.last : sh.cost;
  auto inside = [&](int j) {  // whether border j cuts this item
    const int64_t in = j * work.share - p.from;
    if (in < 0 || in >= cost) return false;
    const int t = sh.cut(p.tile, (int)in);
    return t > 0 && t < sh.tiles;
  };
  if (inside(b - 1)) return;
  int n = 2;
  while (inside(b + n - 1)) ++n;
  constexpr int kChunks = D / 8;
  for (int e = blockIdx.x % kJoinBlocks * kMergeThreads + threadIdx.x; e < kBM * kChunks; e += kJoinBlocks * kMergeThreads) {
    const int r = e / kChunks, ch = e % kChunks * 8;
    if (row0 + r >= rows) return;
    auto part = [&](int k) { return (int64_t)(2 * (b + k) - (k == 0 ? 1 : 2)) * kBM + r; };
    join_parts<D, 4>(a, n, part, row_of(se, row0 + r, p.h, a.pool.H, a.G), ch);
  }
}

template <int D>
static hipError_t configure_d() {
  const void* const all[] = {(const void*)cache_tiles_kernel<D, kWhole>, (const void*)cache_tiles_kernel<D, kSplit>,
                             (const void*)cache_tiles_kernel<D, kEven>, (const void*)cache_tiles_kernel<D, kSplit, kThinRows>};
  for (const void* kern : all) {
    const hipError_t e = hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, tiles_lds<D>() + kStateBytes);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t configure_tiles() {
  const hipError_t e = configure_d<64>();
  return e != hipSuccess ? e : configure_d<128>();
}

template <int D>
static void launch_tiles_d(const RowArgs& r, int64_t items, hipStream_t st) {
  if (r.shares > 0) {
    hipLaunchKernelGGL((cache_tiles_kernel<D, kEven>), dim3((r.shares + 7) / 8 * 8), dim3(kThreads), tiles_lds<D>() + kStateBytes, st, r);
    hipLaunchKernelGGL(cache_join_kernel<D>, dim3((r.shares - 1) * kJoinBlocks), dim3(kMergeThreads), 0, st, r);
    return;
  }
  const unsigned grid = (unsigned)((items + 7) / 8 * 8);  // every XCD has up to ceil(items / 8)
  auto kern = r.n_split == 1 ? cache_tiles_kernel<D, kWhole> : r.few ? cache_tiles_kernel<D, kSplit, kThinRows> : cache_tiles_kernel<D, kSplit>;
  hipLaunchKernelGGL(kern, dim3(grid), dim3(kThreads), tiles_lds<D>(), st, r);
}

// RowArgs' workgroups are 256-row tiles of a session and head here, `items` of them at most.
void launch_tiles(const RowArgs& r, int d, int64_t items, hipStream_t st) {
  if (d == 64) launch_tiles_d<64>(r, items, st);
  else launch_tiles_d<128>(r, items, st);
}

}  // namespace tscache
