// block_plan.cpp -- host-side sizes of the transformer block's launches, shared by the argument checks of ts_block.cpp
// and the launch code; no device code.
#include <stdint.h>

#include <algorithm>

#include "block_launch.h"

namespace tsblock {

namespace {
int64_t ceil_div(int64_t a, int64_t b) { return a / b + (a % b != 0); }
int64_t align256(int64_t x) { return (x + 255) / 256 * 256; }
}  // namespace

int32_t rope_bwd_blocks(int32_t T, int32_t q_heads, int32_t k_heads, int32_t d) {
  const int per = 64 / (d / 16);  // heads of a wave's step
  const int64_t steps = (int64_t)T * (ceil_div(q_heads, per) + ceil_div(k_heads, per));
  return (int32_t)std::min<int64_t>(1024, ceil_div(steps, kRopeThreads / 64));
}

int64_t bwd_tiles(int32_t nseq, int32_t most, int32_t total) {
  // each segment fills all its tiles but the last, and has one more at most
  return std::min<int64_t>(nseq * ceil_div(most, kBwdTile), (int64_t)total / kBwdTile + std::min(nseq, total));
}

namespace {
BwdParts layout(int32_t n_q, int32_t n_k, int64_t tiles, int64_t rows_q, int64_t rows_k, int32_t d) {
  BwdParts p{n_q, n_k, 0, 0, 0, 0};
  p.stat_offset = align256((int64_t)sizeof(BwdPlan) + tiles * (int64_t)sizeof(BwdTile));
  p.q_offset = p.stat_offset + align256(2 * rows_q * 4);
  p.k_offset = p.q_offset + (n_q > 1 ? align256(n_q * rows_q * d * 4) : 0);
  p.bytes = p.k_offset + (n_k > 1 ? align256(2 * n_k * rows_k * d * 4) : 0);
  return p;
}
}  // namespace

BwdParts bwd_parts(int32_t nseq, int32_t max_q, int32_t max_k, int32_t total_q, int32_t total_k, int32_t H, int32_t d,
                   int32_t num_splits, int64_t workspace, int32_t cus) {
  const int64_t rows_q = (int64_t)total_q * H, rows_k = (int64_t)total_k * H;
  const int64_t tiles_q = bwd_tiles(nseq, max_q, total_q), tiles_k = bwd_tiles(nseq, max_k, total_k), tiles = tiles_q + tiles_k;
  if (num_splits > 0) return layout(num_splits, num_splits, tiles, rows_q, rows_k, d);
  // costs in products of a tile and a step: three for dq, four for dk and dv
  const int64_t steps_k = ceil_div(max_k, bwd_step(d)), steps_q = ceil_div(max_q, bwd_step(d));
  const int64_t share = H * (3 * tiles_q * steps_k + 4 * tiles_k * steps_q) / std::max(1, cus);  // of a CU
  auto ranges = [&](int64_t cost, int64_t steps) {  // so that an item is at most half of a CU's share
    return (int32_t)std::max<int64_t>(1, std::min({(int64_t)16, ceil_div(2 * cost, std::max<int64_t>(share, 1)), steps}));
  };
  int32_t n_q = ranges(3 * steps_k, steps_k), n_k = ranges(4 * steps_q, steps_q);
  if (tiles * H >= 4 * (int64_t)cus) n_q = n_k = 1;
  BwdParts p = layout(n_q, n_k, tiles, rows_q, rows_k, d);
  while (p.bytes > workspace && (n_q > 1 || n_k > 1)) {
    n_q = std::max(1, n_q / 2);
    n_k = std::max(1, n_k / 2);
    p = layout(n_q, n_k, tiles, rows_q, rows_k, d);
  }
  return p;
}

}  // namespace tsblock
