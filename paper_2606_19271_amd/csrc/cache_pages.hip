// cache_pages.hip -- gfx950 kernels that write the session cache's pages: append and evict.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_launch.h"
#include "cache_device.h"

namespace tscache {

constexpr int kPageThreads = 256;
constexpr int kPageWaves = kPageThreads / 64;

// Largest of the workgroup's two values of every thread (buf: 2 * kPageWaves words of LDS).
__device__ __forceinline__ void block_max2(unsigned& a, unsigned& b, unsigned* buf) {
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) {
    a = max(a, (unsigned)__shfl_xor((int)a, m));
    b = max(b, (unsigned)__shfl_xor((int)b, m));
  }
  if ((threadIdx.x & 63) == 0) {
    buf[threadIdx.x >> 6] = a;
    buf[kPageWaves + (threadIdx.x >> 6)] = b;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kPageWaves; ++w) {
    a = max(a, buf[w]);
    b = max(b, buf[kPageWaves + w]);
  }
}

// ---- append: one workgroup per (session, touched page, head).  A thread holds pieces of 16 channels of a
// token (32 bytes in, 16 out), so K and V are each read once, the page's amax formed and the pieces
// converted from registers.  Bound by HBM: 5 x 4680 tokens x 40 heads, d = 128, 143 us, 0.72 GB at 5.0 TB/s; eight single
// tokens take 4.5 us, of which their pages' rewriting is the least part.
template <int D>
__global__ void __launch_bounds__(kPageThreads)
cache_append_kernel(Pool pool, Sessions ss, const __bf16* __restrict__ k, const __bf16* __restrict__ v,
                    int32_t* __restrict__ new_lens, int page_slots) {
  constexpr int kPieces = D / 16;                           // of a token
  constexpr int kPer = kPage * kPieces / kPageThreads;      // of a thread
  __shared__ unsigned buf[2 * kPageWaves];
  const int b = blockIdx.x;
  const int h = b % pool.H, sj = b / pool.H, j = sj % page_slots, s = sj / page_slots;
  const Session se = session_of(ss, s);
  const bool fits = se.ok && se.rows <= ss.max_len - se.len;
  if (j == 0 && h == 0 && threadIdx.x == 0) new_lens[s] = se.len + (fits ? se.rows : 0);
  if (!fits) return;
  const int p = se.len / kPage + j;                  // page of the session
  const int old = max(0, se.len - p * kPage);        // its slots that hold older tokens
  const int end = min(kPage, se.len + se.rows - p * kPage);
  if (se.rows == 0 || old >= end) return;
  const int page = ss.table[(int64_t)s * ss.width + p];
  if ((unsigned)page >= (unsigned)pool.pages) return;
  const int64_t ph = (int64_t)page * pool.H + h;
  const int64_t row0 = (int64_t)se.q0 - se.len + (int64_t)p * kPage;  // packed row of slot 0
  u32x4 kx[kPer][2] = {}, vx[kPer][2] = {};
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int n = threadIdx.x + kPageThreads * i, slot = n / kPieces, c = n % kPieces;
    if (slot >= old && slot < end) {
      const int64_t at = ((row0 + slot) * pool.H + h) * D + 16 * c;
      kx[i][0] = *(const u32x4*)(k + at), kx[i][1] = *(const u32x4*)(k + at + 8);
      vx[i][0] = *(const u32x4*)(v + at), vx[i][1] = *(const u32x4*)(v + at + 8);
    }
  }
  const int k_was = old > 0 ? pool.k_exp[ph] : 0, v_was = old > 0 ? pool.v_exp[ph] : 0;
  unsigned ka = 0, va = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i)
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        ka = amax_bits(ka, kx[i][u][x]);
        va = amax_bits(va, vx[i][u][x]);
      }
  block_max2(ka, va, buf);
  const int ke = max(exponent_of(ka), k_was), ve = max(exponent_of(va), v_was);
  auto put = [&](uint8_t* base, const u32x4 (&x)[kPer][2], int exp, int was) {
    const float up = scale_of(254 - exp, false);  // 2^-n; exp is at most 247 unless the page's was more
    uint8_t* const at = base + ph * (kPage * D);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int n = threadIdx.x + kPageThreads * i, slot = n / kPieces;
      u32x4 r;
      if (slot >= old && slot < end) {
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const u32x4 w = x[i][y / 2];
          const unsigned a = w[2 * (y & 1)], c = w[2 * (y & 1) + 1];
          r[y] = narrow4(__uint_as_float(a << 16) * up, __uint_as_float(a & 0xffff0000u) * up,
                         __uint_as_float(c << 16) * up, __uint_as_float(c & 0xffff0000u) * up);
        }
      } else if (slot < old && exp != was) {
        const u32x4 w = *(const u32x4*)(at + n * 16);
        const float s0 = scale_of(was, false);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const bf16x4 f = widen4(w[y], s0);
          r[y] = narrow4((float)f[0] * up, (float)f[1] * up, (float)f[2] * up, (float)f[3] * up);
        }
      } else {
        continue;
      }
      *(u32x4*)(at + n * 16) = r;
    }
    if (exp != kTopExp) return;  // (apart, and over again: in line it takes a single token's call from 4.6 to 5.0 us)
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int n = threadIdx.x + kPageThreads * i, slot = n / kPieces;
      if (slot < old || slot >= end) continue;
      u32x4 r = *(const u32x4*)(at + n * 16);
#pragma unroll
      for (int y = 0; y < 4; ++y) r[y] = in_bf16(r[y]);
      *(u32x4*)(at + n * 16) = r;
    }
  };
  put(pool.k, kx, ke, k_was);
  put(pool.v, vx, ve, v_was);
  if (threadIdx.x == 0) {
    pool.k_exp[ph] = (uint8_t)ke;
    pool.v_exp[ph] = (uint8_t)ve;
  }
  if (pool.weight != nullptr && (int)threadIdx.x >= old && (int)threadIdx.x < end)
    pool.weight[ph * kPage + threadIdx.x] = 0.0f;
}

// ---- evict, first kernel: which tokens stay.  One workgroup per (session, head).
//
// The tokens of the middle (neither the first nor the last protected ones) are ranked by their weight as an
// ordered integer, read once into LDS (as many as fit: kCachedMax; further ones are read again in every pass).  Four
// passes over 8 bits find the m-th largest, threshold, each narrowing the prefix by a histogram in LDS; then a pass
// counts what every wave keeps and one writes the positions.  A histogram has 16 copies, one to a bank or two: weights
// share their exponents, and lanes that count in one bin of one copy do so one after the other.  200 workgroups of 32760
// tokens take 42 us (85 us with one histogram of 2048 bins and the weights read again in each of five passes).
constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / 64;
constexpr int kBins = 256, kCopies = 16;
constexpr int kHistBytes = kBins * kCopies * 4;
constexpr int kCachedMax = 575 * kPage;  // with the histogram and the scans' words within the 160 KiB of a CU
constexpr int kAhead = 8;                // pages of weights that a wave has in flight

// Monotone in the weight: -infinity (and NaN) lowest, -0 equal to 0.
__device__ __forceinline__ unsigned rank_bits(float w) {
  unsigned u = __float_as_uint(w);
  if (w != w) u = 0xff800000u;
  if (w == 0.0f) u = 0u;
  return u >> 31 ? ~u : u | 0x80000000u;
}

__global__ void __launch_bounds__(kSelectThreads)
cache_select_kernel(Pool pool, Sessions ss, int32_t* __restrict__ new_lens, int32_t* __restrict__ kept,
                    int keep, int first, int last, int cached) {
  extern __shared__ __attribute__((aligned(16))) unsigned select_lds[];
  __shared__ unsigned wave_a[kSelectWaves], wave_b[kSelectWaves];
  __shared__ unsigned found[2];
  unsigned* const hist = select_lds;                    // [kBins][kCopies]
  unsigned* const ranks = select_lds + kBins * kCopies; // of the first `cached` tokens
  const int h = blockIdx.x % pool.H, s = blockIdx.x / pool.H;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const Session se = session_of(ss, s);
  int32_t* const out = kept + (int64_t)blockIdx.x * keep;
  if (h == 0 && tid == 0) new_lens[s] = se.ok ? min(se.len, keep) : se.len;
  if (!se.ok || se.len <= keep) {
    for (int i = tid; i < keep; i += kSelectThreads) out[i] = se.ok && i < se.len ? i : -1;
    return;
  }
  const int begin = first, end = se.len - last;  // the middle; begin < end since len > keep >= first + last
  const int32_t* const table = ss.table + (int64_t)s * ss.width;
  auto weight_of = [&](int page, int slot) {  // tokens of pages outside the pool rank lowest
    const bool bad = (unsigned)page >= (unsigned)pool.pages;
    const float w = pool.weight[page_offset(page, bad, pool.H, h, kPage) + slot];
    return bad ? -INFINITY : w;
  };
  auto rank_at = [&](int i) -> unsigned {
    return i < cached ? ranks[i] : rank_bits(weight_of(table[i / kPage], i % kPage));
  };
  unsigned want = (unsigned)(keep - first - last);  // tokens of the middle that stay
  unsigned prefix = 0, mask = 0;
  const bool none = want == 0;
  if (!none) {
    // wave w reads the pages w, w + kSelectWaves, ...; lane i has the number of the i-th of 64 of them
    const int pages = min((se.len + kPage - 1) / kPage, cached / kPage);
    for (int p0 = wave; p0 < pages; p0 += kSelectWaves * 64) {
      const int mine = min(64, (pages - p0 + kSelectWaves - 1) / kSelectWaves);
      const int id = lane < mine ? table[p0 + kSelectWaves * lane] : 0;
      for (int k = 0; k < mine; k += kAhead) {
        float w[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) w[u] = weight_of(__builtin_amdgcn_readlane(id, min(k + u, mine - 1)), lane);
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
          if (k + u < mine) ranks[(p0 + kSelectWaves * (k + u)) * kPage + lane] = rank_bits(w[u]);
      }
    }
  }
  for (int shift = 24; shift >= 0 && !none; shift -= 8) {
    *(u32x4*)(hist + 4 * tid) = u32x4{};
    __syncthreads();
    for (int i = begin + tid; i < end; i += kSelectThreads) {
      const unsigned u = rank_at(i);
      if ((u & mask) == prefix) atomicAdd(&hist[(u >> shift & (kBins - 1)) * kCopies + (lane & (kCopies - 1))], 1u);
    }
    __syncthreads();
    // the bin that holds the want-th largest: suffix sums, four lanes to a bin, from the top
    const int bin = kBins - 1 - tid / 4;
    const u32x4 part = *(const u32x4*)(hist + bin * kCopies + tid % 4 * 4);
    unsigned here = (part[0] + part[1]) + (part[2] + part[3]);
    here += (unsigned)__shfl_xor((int)here, 1);
    here += (unsigned)__shfl_xor((int)here, 2);
    unsigned sum = here;
#pragma unroll
    for (int m = 4; m < 64; m <<= 1) {
      const unsigned y = (unsigned)__shfl_up((int)sum, m);
      if (lane >= m) sum += y;
    }
    if (lane == 63) wave_a[wave] = sum;
    __syncthreads();
    unsigned before = sum - here;
    for (int w = 0; w < wave; ++w) before += wave_a[w];
    if (before < want && before + here >= want && tid % 4 == 0) found[0] = (unsigned)bin, found[1] = before;
    __syncthreads();
    prefix |= found[0] << shift;
    mask |= (unsigned)(kBins - 1) << shift;
    want -= found[1];
  }
  // kept of the middle: every rank above prefix, and of those equal to it the first `want`
  const int per = ((end - begin + kSelectWaves - 1) / kSelectWaves + 63) / 64 * 64;
  const int wb = begin + wave * per, we = min(end, wb + per);
  unsigned above = 0, equal = 0;
  if (!none)
    for (int i = wb; i < we; i += 64) {
      const bool in = i + lane < we;
      const unsigned u = in ? rank_at(i + lane) : 0u;
      above += (unsigned)__builtin_popcountll(__builtin_amdgcn_ballot_w64(in && u > prefix));
      equal += (unsigned)__builtin_popcountll(__builtin_amdgcn_ballot_w64(in && u == prefix));
    }
  if (lane == 0) wave_a[wave] = above, wave_b[wave] = equal;
  __syncthreads();
  unsigned at = (unsigned)first, eq = 0;
  for (int w = 0; w < wave; ++w) {
    at += wave_a[w] + (eq < want ? min(want - eq, wave_b[w]) : 0u);
    eq += wave_b[w];
  }
  const unsigned long long below = ((unsigned long long)1 << lane) - 1;
  if (!none)
    for (int i = wb; i < we; i += 64) {
      const bool in = i + lane < we;
      const unsigned u = in ? rank_at(i + lane) : 0u;
      const unsigned long long be = __builtin_amdgcn_ballot_w64(in && u == prefix);
      const bool stay = in && (u > prefix || (u == prefix && eq + (unsigned)__builtin_popcountll(be & below) < want));
      const unsigned long long bs = __builtin_amdgcn_ballot_w64(stay);
      if (stay) out[at + (unsigned)__builtin_popcountll(bs & below)] = i + lane;
      at += (unsigned)__builtin_popcountll(bs);
      eq += (unsigned)__builtin_popcountll(be);
    }
  for (int i = tid; i < first; i += kSelectThreads) out[i] = i;
  for (int i = tid; i < last; i += kSelectThreads) out[keep - last + i] = end + i;
}

// ---- evict, second kernel: the kept tokens into their new pages.  One workgroup per (session, new page,
// head); a thread holds pieces of 16 channels of a token: whole 64- or 128-byte rows of wherever the tokens lie, so
// nothing is read beside them.  Bound by HBM: 200 heads x 16380 tokens, d = 128, 362 us, 0.89 GB read + 0.85 written at 4.8 TB/s.
template <int D>
__global__ void __launch_bounds__(kPageThreads)
cache_gather_kernel(Pool pool, Sessions ss, const int32_t* __restrict__ new_table,
                    const int32_t* __restrict__ kept, int new_width, int keep, int page_slots) {
  constexpr int kPieces = D / 16;
  constexpr int kPer = kPage * kPieces / kPageThreads;
  __shared__ unsigned buf[2 * kPageWaves];
  const int b = blockIdx.x;
  const int h = b % pool.H, sj = b / pool.H, j = sj % page_slots, s = sj / page_slots;
  const Session se = session_of(ss, s);
  if (!se.ok) return;
  const int live = min(kPage, min(se.len, keep) - j * kPage);
  if (live <= 0) return;
  const int page = new_table[(int64_t)s * new_width + j];
  if ((unsigned)page >= (unsigned)pool.pages) return;
  const int64_t ph = (int64_t)page * pool.H + h;
  const int32_t* const table = ss.table + (int64_t)s * ss.width;
  const int32_t* const ids = kept + ((int64_t)s * pool.H + h) * keep + j * kPage;
  u32x4 kx[kPer] = {}, vx[kPer] = {};
  float ks[kPer] = {}, vs[kPer] = {};
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int n = threadIdx.x + kPageThreads * i, slot = n / kPieces, c = n % kPieces;
    if (slot < live) {
      const int id = ids[slot], from = table[id / kPage];
      const bool bad = (unsigned)from >= (unsigned)pool.pages;
      const int64_t fh = page_offset(from, bad, pool.H, h, 1);
      const int64_t at = fh * (kPage * D) + (id % kPage) * D + 16 * c;
      kx[i] = *(const u32x4*)(pool.k + at);
      vx[i] = *(const u32x4*)(pool.v + at);
      ks[i] = scale_of(pool.k_exp[fh], bad);
      vs[i] = scale_of(pool.v_exp[fh], bad);
      if (c == 0) pool.weight[ph * kPage + slot] = bad ? -INFINITY : pool.weight[fh * kPage + id % kPage];
    }
  }
  unsigned ka = 0, va = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i)
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const u32x2 a = __builtin_bit_cast(u32x2, widen4(kx[i][x], ks[i]));
      const u32x2 c = __builtin_bit_cast(u32x2, widen4(vx[i][x], vs[i]));
      ka = amax_bits(amax_bits(ka, a[0]), a[1]);
      va = amax_bits(amax_bits(va, c[0]), c[1]);
    }
  block_max2(ka, va, buf);
  const int ke = exponent_of(ka), ve = exponent_of(va);
  auto put = [&](uint8_t* base, const u32x4 (&x)[kPer], const float (&from)[kPer], int exp) {
    const float up = scale_of(254 - exp, false);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int n = threadIdx.x + kPageThreads * i;
      if (n / kPieces >= live) continue;
      u32x4 r;
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const bf16x4 f = widen4(x[i][y], from[i]);
        r[y] = narrow4((float)f[0] * up, (float)f[1] * up, (float)f[2] * up, (float)f[3] * up);
      }
      *(u32x4*)(base + ph * (kPage * D) + n * 16) = r;
    }
  };
  put(pool.k, kx, ks, ke);
  put(pool.v, vx, vs, ve);
  if (threadIdx.x == 0) {
    pool.k_exp[ph] = (uint8_t)ke;
    pool.v_exp[ph] = (uint8_t)ve;
  }
}

// ---------------------------------------------------------------------------------------------
// host-side launchers

hipError_t launch_append(const AppendArgs& a, hipStream_t st) {
  const int64_t items = append_items(a.ss.nseq, a.ss.max_rows, a.pool.H);
  const int page_slots = (int)(items / ((int64_t)a.ss.nseq * a.pool.H));
  auto kern = a.d == 64 ? cache_append_kernel<64> : cache_append_kernel<128>;
  hipLaunchKernelGGL(kern, dim3((unsigned)items), dim3(kPageThreads), 0, st, a.pool, a.ss,
                     (const __bf16*)a.k, (const __bf16*)a.v, a.new_lens, page_slots);
  return hipGetLastError();
}

hipError_t configure_pages() {
  return hipFuncSetAttribute((const void*)cache_select_kernel, hipFuncAttributeMaxDynamicSharedMemorySize,
                             kHistBytes + kCachedMax * 4);
}

hipError_t launch_evict(const EvictArgs& a, hipStream_t st) {
  const int cached = min((a.ss.max_len + kPage - 1) / kPage * kPage, kCachedMax);
  hipLaunchKernelGGL(cache_select_kernel, dim3((unsigned)(a.ss.nseq * a.pool.H)), dim3(kSelectThreads),
                     kHistBytes + cached * 4, st, a.pool, a.ss, a.new_lens, a.kept, a.keep, a.first, a.last, cached);
  const hipError_t e = hipGetLastError();
  const int64_t items = gather_items(a.ss.nseq, a.keep, a.pool.H);
  if (e != hipSuccess || items == 0) return e;
  auto kern = a.d == 64 ? cache_gather_kernel<64> : cache_gather_kernel<128>;
  hipLaunchKernelGGL(kern, dim3((unsigned)items), dim3(kPageThreads), 0, st, a.pool, a.ss, a.new_table,
                     a.kept, a.new_width, a.keep, (a.keep + kPage - 1) / kPage);
  return hipGetLastError();
}

}  // namespace tscache
