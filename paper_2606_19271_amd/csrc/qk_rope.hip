// qk_rope.hip -- norm and rotation of queries and keys in one pass (ts_qk_rope), and its gradients.
//
// Both are bound by memory, each row read and written once: 23400 tokens x 80 heads (d = 128) 181 us, 5.3 TB/s read and
// written, the gradients of 32760 x 80 heads 400 us, 5.0 TB/s with two thirds of it reads (a copy of 1 GB by torch: 5.0).
// Small calls are bound by the latency of launch, positions and rows: 4 tokens 3.7 us, 1560 x 24 heads 8.0 us.
// A wave has one step's loads under way while it works on the one before; every 8 to 16 heads share a token's angles,
// which cost each lane one sine and cosine.  (With the eight of its pairs formed by each lane, and the loads one
// after the other, 1560 x 24 heads took 17.8 us.)
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "block_launch.h"

namespace tsblock {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kWaves = kRopeThreads / 64;

// A head's d channels lie over d / 16 lanes: lane j has channels 8j..8j+7 and d/2 + 8j..8j+7, two 16-byte loads, so that
// the pairs of both orders lie within a lane: neighbours (2i, 2i + 1), or (i, i + d / 2).  A wave's step is
// 64 / (d / 16) heads of one token.
template <int D>
struct Geo {
  static constexpr int kLanes = D / 16;
  static constexpr int kHeads = 64 / kLanes;
};

struct Head {
  bf16x8 lo, hi;
};

// kFar: past the caches (see `far`).
template <int D, bool kFar>
__device__ __forceinline__ Head load_head(const __bf16* p, bool live) {
  if (!live) return Head{};
  const bf16x8 *const lo = (const bf16x8*)p, *const hi = (const bf16x8*)(p + D / 2);
  return kFar ? Head{__builtin_nontemporal_load(lo), __builtin_nontemporal_load(hi)} : Head{*lo, *hi};
}

template <int D, bool kFar>
__device__ __forceinline__ void store_head(__bf16* p, const float (&x)[16], bool live) {
  if (!live) return;
  bf16x8 lo, hi;
#pragma unroll
  for (int i = 0; i < 8; ++i) lo[i] = (__bf16)x[i], hi[i] = (__bf16)x[8 + i];
  if (kFar) {
    __builtin_nontemporal_store(lo, (bf16x8*)p);
    __builtin_nontemporal_store(hi, (bf16x8*)(p + D / 2));
  } else {
    *(bf16x8*)p = lo;
    *(bf16x8*)(p + D / 2) = hi;
  }
}

__device__ __forceinline__ void widen(const Head& h, float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)h.lo[i], x[8 + i] = (float)h.hi[i];
}

// The lane's slots of its eight pairs, in x[16]: pair i's members.
template <bool kPairs>
__device__ __forceinline__ constexpr int member(int i, int which) {
  return kPairs ? 2 * i + which : i + 8 * which;
}

// cos and sin of a token's angles.  Each lane forms those of one of the wave's d / 2 pairs and leaves them in the wave's LDS,
// where it finds the eight of its own pairs.  A turn's fraction is exact to 2^-53 of the angle in 64 bits, and what is left
// of it, half a turn at most, fits 32.
constexpr int kAngleRow = 64 + 4;  // floats

// A token's place on the axis of the lane's pair, and the lane's frequency.  (All three places are read, by scalar loads.)
struct Place {
  int32_t p0, p1, p2;
};
__device__ __forceinline__ Place place(const Rope& rope, int t) {
  if (!rope.freq) return Place{0, 0, 0};
  const int32_t* const pos = rope.pos + 3 * (int64_t)t;
  return Place{pos[0], pos[1], pos[2]};
}

template <int D, bool kPairs>
__device__ __forceinline__ void angles(const Rope& rope, const Place& at, int lane, double freq, float* lds, float (&c)[8],
                                       float (&s)[8]) {
  const int pair = lane % (D / 2);
  const int32_t p = pair < rope.n0 ? at.p0 : pair < rope.n01 ? at.p1 : at.p2;
  double turns = (double)p * (freq * 0.15915494309189535);
  turns -= __builtin_rint(turns);
  float sine, cosine;
  sincospif(2.0f * (float)turns, &sine, &cosine);
  __builtin_amdgcn_wave_barrier();  // (the token before has read its angles)
  lds[pair] = cosine;  // (at d = 64 by two lanes alike)
  lds[kAngleRow + pair] = sine;
  __builtin_amdgcn_wave_barrier();
  const int j = lane % Geo<D>::kLanes, lo = kPairs ? 4 * j : 8 * j, hi = kPairs ? D / 4 + 4 * j : 8 * j + 4;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    c[i] = lds[lo + i];
    c[4 + i] = lds[hi + i];
    s[i] = lds[kAngleRow + lo + i];
    s[4 + i] = lds[kAngleRow + hi + i];
  }
}

// x of the lane l ^ kXor (1, 2 or 4) of its eight.
template <int kXor>
__device__ __forceinline__ int from_lane(int x) {
  constexpr int kCtrl = kXor == 1 ? 0xB1 : kXor == 2 ? 0x4E : 0x141;  // quad_perm, quad_perm, row_half_mirror
  return __builtin_amdgcn_update_dpp(0, x, kCtrl, 0xF, 0xF, true);
}
template <int kXor>
__device__ __forceinline__ float from_lane(float x) { return __int_as_float(from_lane<kXor>(__float_as_int(x))); }
template <int kXor>
__device__ __forceinline__ double from_lane(double x) {
  return __hiloint2double(from_lane<kXor>(__double2hiint(x)), from_lane<kXor>(__double2loint(x)));
}

// The sum over a head's lanes, in each of them (the half mirror takes a quad's sum from the other quad).
template <int D, typename T>
__device__ __forceinline__ T head_sum(T x) {
  x += from_lane<1>(x);
  x += from_lane<2>(x);
  if (D == 128) x += from_lane<4>(x);
  return x;
}

// 1 / sqrt(mean of squares + eps).  In 64 bits, where no bfloat16 square overflows or vanishes.
template <int D>
__device__ __forceinline__ float inverse_rms(const float (&x)[16], float eps) {
  double sum = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) sum = __builtin_fma((double)x[i], (double)x[i], sum);
  const double m = __builtin_fma(head_sum<D>(sum), 1.0 / D, (double)eps);
  const double y = __builtin_amdgcn_rsq(m);
  const double z = y * __builtin_fma(-0.5 * m * y, y, 1.5);  // (NaN at infinity, where y is 0)
  return (float)(y == 0 ? y : z);
}

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

template <int D>
__device__ __forceinline__ void load_weights(const float* w, int j, float (&x)[16]) {
  if (!w) return;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const f32x4_any y = *(const f32x4_any*)(w + 8 * j + 4 * (u & 1) + (u >> 1) * (D / 2));
#pragma unroll
    for (int i = 0; i < 4; ++i) x[4 * u + i] = y[i];
  }
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// A wave's steps: `count` from `first` on, step s being heads kHeads (s % groups) .. of token s / groups, those of q before
// those of k.
struct Steps {
  int t, g, left;
  __device__ Steps(int wave, int per, int all, int groups) {
    const int first = (int)min((int64_t)wave * per, (int64_t)all);
    t = first / groups;
    g = first - t * groups;
    left = min(per, all - first);
  }
  __device__ bool next(int groups) {  // whether the token is another one
    --left;
    if (++g < groups) return false;
    g = 0;
    ++t;
    return true;
  }
};

template <int D, bool kPairs, bool kFar>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeArgs a, int groups_q, int groups, int steps, int per) {
  using G = Geo<D>;
  const int lane = threadIdx.x & 63, wave = uniform(blockIdx.x * kWaves + (threadIdx.x >> 6));
  const int j = lane % G::kLanes, r = lane / G::kLanes;
  Steps at(wave, per, steps, groups);
  if (at.left <= 0) return;
  __shared__ float lds[kWaves][2 * kAngleRow];
  float wq[16], wk[16], c[8], s[8];
  auto rows = [&](const Rows& q, const Rows& k, const Steps& at, bool& live) {
    const bool is_k = at.g >= groups_q;
    const Rows& x = is_k ? k : q;
    const int h = (at.g - (is_k ? groups_q : 0)) * G::kHeads + r;
    live = h < x.heads;
    return (__bf16*)x.p + at.t * x.stride + h * D + 8 * j;
  };
  bool live;
  const __bf16* from = rows(a.q, a.k, at, live);
  Head in = load_head<D, kFar>(from, live);
  const double freq = a.rope.freq ? a.rope.freq[lane % (D / 2)] : 0.0;
  load_weights<D>(a.q_weight, j, wq);
  load_weights<D>(a.k_weight, j, wk);
  bool fresh = true;
  while (true) {
    if (fresh && a.rope.freq) angles<D, kPairs>(a.rope, place(a.rope, at.t), lane, freq, lds[threadIdx.x >> 6], c, s);
    const Steps here = at;
    Head after = in;
    fresh = at.next(groups);
    if (at.left > 0) {
      bool next_live;
      from = rows(a.q, a.k, at, next_live);
      after = load_head<D, kFar>(from, next_live);
    }
    float x[16];
    widen(in, x);
    const bool is_k = here.g >= groups_q;
    if (is_k ? a.k_weight : a.q_weight) {
      const float f = inverse_rms<D>(x, a.eps);
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = x[i] * f * (is_k ? wk[i] : wq[i]);
    }
    if (a.rope.freq) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float u = x[member<kPairs>(i, 0)], v = x[member<kPairs>(i, 1)];
        x[member<kPairs>(i, 0)] = u * c[i] - v * s[i];
        x[member<kPairs>(i, 1)] = u * s[i] + v * c[i];
      }
    }
    __bf16* const to = rows(a.q_out, a.k_out, here, live);
    store_head<D, kFar>(to, x, live);
    if (at.left <= 0) return;
    in = after;
  }
}

// Gradients.  As many workgroups as the device holds at once take equal parts of the steps, whatever their number, so that the sums'
// order is the call's own.  With g the result's gradient turned back, n = x r the normalised row:
//   dw = sum g n,   dx = r (g w - n mean(g w n))
// Each lane sums dw over kChain steps at most, in 32 bits; what the wave's lanes have then goes into the wave's sums in LDS, in 64, as a
// chain of all steps would lose as many bits as it is long (8192 equal terms 11, 128 of them 5).  The workgroup adds its
// waves' sums, and rope_bwd_join_kernel those of the workgroups.
constexpr int kChain = 128;

template <int D, bool kPairs, bool kFar>
__global__ __launch_bounds__(kRopeThreads) void rope_bwd_kernel(RopeBwdArgs a, int groups_q, int groups, int steps, int per) {
  using G = Geo<D>;
  const int lane = threadIdx.x & 63, wave = uniform(blockIdx.x * kWaves + (threadIdx.x >> 6));
  const int j = lane % G::kLanes, r = lane / G::kLanes;
  Steps at(wave, per, steps, groups);
  __shared__ float lds[kWaves][2 * kAngleRow];
  __shared__ double sums[kWaves][2 * D];
  double* const sum = sums[threadIdx.x >> 6];
  if (at.left <= 0)
    for (int ch = lane; ch < 2 * D; ch += 64) sum[ch] = 0;
  float wq[16], wk[16], c[8], s[8], sum_q[16] = {}, sum_k[16] = {};
  auto rows = [&](const Rows& q, const Rows& k, const Steps& at, bool& live) {
    const bool is_k = at.g >= groups_q;
    const Rows& x = is_k ? k : q;
    const int h = (at.g - (is_k ? groups_q : 0)) * G::kHeads + r;
    live = h < x.heads && x.p;
    return (__bf16*)x.p + at.t * x.stride + h * D + 8 * j;
  };
  bool fresh = true;
  auto load = [&](Head& dy, Head& x) {
    bool live;
    const __bf16* p = rows(a.dq_out, a.dk_out, at, live);
    dy = load_head<D, kFar>(p, live);
    p = rows(a.q, a.k, at, live);
    x = load_head<D, kFar>(p, live && (at.g >= groups_q ? a.k_weight : a.q_weight));
  };
  Head dy_in{}, x_in{};
  if (at.left > 0) load(dy_in, x_in);
  const double freq = a.rope.freq ? a.rope.freq[lane % (D / 2)] : 0.0;
  load_weights<D>(a.q_weight, j, wq);
  load_weights<D>(a.k_weight, j, wk);
  int chain = 0;
  bool begun = false;  // whether the wave's sums hold anything
  while (at.left > 0) {
    if (fresh && a.rope.freq) angles<D, kPairs>(a.rope, place(a.rope, at.t), lane, freq, lds[threadIdx.x >> 6], c, s);
    const Steps here = at;
    Head dy_next = dy_in, x_next = x_in;
    fresh = at.next(groups);
    if (at.left > 0) load(dy_next, x_next);
    float g[16];
    widen(dy_in, g);
    if (a.rope.freq) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float u = g[member<kPairs>(i, 0)], v = g[member<kPairs>(i, 1)];
        g[member<kPairs>(i, 0)] = u * c[i] + v * s[i];
        g[member<kPairs>(i, 1)] = v * c[i] - u * s[i];
      }
    }
    const bool is_k = here.g >= groups_q;
    if (is_k ? a.k_weight : a.q_weight) {
      float n[16], dot = 0;
      widen(x_in, n);
      const float f = inverse_rms<D>(n, a.eps);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        n[i] *= f;
        const float dw = g[i] * n[i];
        if (is_k) sum_k[i] += dw;
        else sum_q[i] += dw;
        g[i] *= is_k ? wk[i] : wq[i];
        dot = __builtin_fmaf(g[i], n[i], dot);
      }
      dot = head_sum<D>(dot) * (1.0f / D);
#pragma unroll
      for (int i = 0; i < 16; ++i) g[i] = (g[i] - n[i] * dot) * f;
    }
    bool live;
    __bf16* const to = rows(a.dq, a.dk, here, live);
    store_head<D, kFar>(to, g, live);
    dy_in = dy_next;
    x_in = x_next;
    if (!a.part || (++chain < kChain && at.left > 0)) continue;
    chain = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
#pragma unroll
      for (int o = G::kLanes; o < 64; o <<= 1) {
        sum_q[i] += __shfl_xor(sum_q[i], o);
        sum_k[i] += __shfl_xor(sum_k[i], o);
      }
    }
    auto channel = [&](int i) { return (i < 8 ? 0 : D / 2 - 8) + 8 * j + i; };
    if (r == 0 && !begun) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[channel(i)] = sum_q[i], sum[D + channel(i)] = sum_k[i];
    } else if (r == 0) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[channel(i)] += sum_q[i], sum[D + channel(i)] += sum_k[i];
    }
    begun = true;
#pragma unroll
    for (int i = 0; i < 16; ++i) sum_q[i] = sum_k[i] = 0;
  }
  if (!a.part) return;
  __syncthreads();
  for (int ch = threadIdx.x; ch < 2 * D; ch += kRopeThreads) {
    double x = sums[0][ch];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) x += sums[w][ch];
    a.part[(int64_t)blockIdx.x * 2 * D + ch] = (float)x;
  }
}

// The weights' gradients: 16 channels to a workgroup, the workgroups' sums dealt to 64 threads of each, in 64 bits.
template <int D>
__global__ __launch_bounds__(1024) void rope_bwd_join_kernel(const float* part, int blocks, float* dq_weight, float* dk_weight) {
  __shared__ double sums[64][17];
  const int i = threadIdx.x & 15, ch = blockIdx.x * 16 + i, u = threadIdx.x >> 4;
  double x = 0;
  for (int b = u; b < blocks; b += 64 * 8) {
    float y[8];  // eight reads under way
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] = b + 64 * k < blocks ? part[(int64_t)(b + 64 * k) * 2 * D + ch] : 0.0f;
#pragma unroll
    for (int k = 0; k < 8; ++k) x += y[k];
  }
  sums[u][i] = x;
  __syncthreads();
  for (int n = 32; n > 0; n >>= 1) {
    if (u < n) sums[u][i] += sums[u + n][i];
    __syncthreads();
  }
  float* const to = ch < D ? dq_weight : dk_weight;
  if (u == 0 && to) to[ch < D ? ch : ch - D] = (float)sums[0][i];
}

int64_t ceil_div(int64_t a, int64_t b) { return a / b + (a % b != 0); }

// Whether a call of so many bytes reads and writes past the caches, which do not hold them for another reader then: 40 + 40 heads (d = 128),
// plain and past the caches, us: 6000 tokens (246 MB) 40 and 48, 8000 (328 MB) 63 and 60, 24000 (983 MB) 182 and 172,
// their gradients of 24000 (1.5 GB) 308 and 300.
bool far(int64_t bytes) { return bytes > (int64_t)256 << 20; }

template <int D>
hipError_t rope(const RopeArgs& a, hipStream_t st) {
  const int gq = (int)ceil_div(a.q.heads, Geo<D>::kHeads), groups = gq + (int)ceil_div(a.k.heads, Geo<D>::kHeads);
  const int steps = a.T * groups;
  const int per = (int)std::max({(int64_t)1, std::min<int64_t>(groups, ceil_div(steps, 4096)), ceil_div(steps, (int64_t)1 << 24)});
  const unsigned blocks = (unsigned)ceil_div(ceil_div(steps, per), kWaves);
  const bool pairs = a.rope.interleaved, past = far((int64_t)a.T * (a.q.heads + a.k.heads) * D * 4);
  auto kernel = pairs ? past ? rope_kernel<D, true, true> : rope_kernel<D, true, false>
                      : past ? rope_kernel<D, false, true> : rope_kernel<D, false, false>;
  kernel<<<blocks, kRopeThreads, 0, st>>>(a, gq, groups, steps, per);
  return hipGetLastError();
}

template <int D>
hipError_t rope_bwd(const RopeBwdArgs& a, hipStream_t st) {
  const int gq = (int)ceil_div(a.dq.heads, Geo<D>::kHeads), groups = gq + (int)ceil_div(a.dk.heads, Geo<D>::kHeads);
  const int steps = a.T * groups;
  const int blocks = rope_bwd_blocks(a.T, a.dq.heads, a.dk.heads, D);
  const int per = blocks ? (int)ceil_div(steps, (int64_t)blocks * kWaves) : 1;
  if (blocks > 0) {
    const bool pairs = a.rope.interleaved, past = far((int64_t)a.T * (a.dq.heads + a.dk.heads) * D * 6);
    auto kernel = pairs ? past ? rope_bwd_kernel<D, true, true> : rope_bwd_kernel<D, true, false>
                        : past ? rope_bwd_kernel<D, false, true> : rope_bwd_kernel<D, false, false>;
    kernel<<<blocks, kRopeThreads, 0, st>>>(a, gq, groups, steps, per);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;  // (the sums' kernel reads what this one writes)
  }
  if (a.dq_weight || a.dk_weight) rope_bwd_join_kernel<D><<<2 * D / 16, 1024, 0, st>>>(a.part, blocks, a.dq_weight, a.dk_weight);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopeArgs& a, hipStream_t st) { return a.d == 64 ? rope<64>(a, st) : rope<128>(a, st); }
hipError_t launch_rope_bwd(const RopeBwdArgs& a, hipStream_t st) { return a.d == 64 ? rope_bwd<64>(a, st) : rope_bwd<128>(a, st); }

}  // namespace tsblock
