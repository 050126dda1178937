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
  return (int32_t)std::min<int64_t>(kRopeBwdBlocks, ceil_div(steps, kRopeThreads / 64));
}

int64_t bwd_tiles(int32_t nseq, int32_t most, int32_t total, int32_t tile) {
  // each segment fills all its tiles but the last, and has one more at most
  return std::min<int64_t>(nseq * ceil_div(most, tile), (int64_t)total / tile + std::min(nseq, total));
}

namespace {
struct Call {
  int64_t tiles_q, tiles_k, rows_q, rows_k;
  int32_t d, tile;
};

// d = 64 has tiles of 128 rows, three workgroups of four waves to a CU (in tiles of 256, two waves to a SIMD, 16380 x 16380 x 24 heads
// took 5 % longer).  At d = 128 tiles of 256 rows read the other side half as often: 32768 x 32768 x 12 heads 20.8 ms instead of
// 21.3, 2048 x 2048 x 12 heads 103 us instead of 105, 8190 x 8190 x 4 (256 such tiles) 453 instead of 459; where these are
// fewer than the CUs of an MI355X, those of 128 end sooner: 1024 x 1024 x 12 heads 42 us instead of 47, 256 x 256 x 12 heads 19
// instead of 22.
Call call(int32_t nseq, int32_t max_q, int32_t max_k, int32_t total_q, int32_t total_k, int32_t H, int32_t d) {
  const bool large = d == 128 && H * (bwd_tiles(nseq, max_q, total_q, 256) + bwd_tiles(nseq, max_k, total_k, 256)) >= 256;
  const int32_t tile = large ? 256 : 128;
  return {bwd_tiles(nseq, max_q, total_q, tile), bwd_tiles(nseq, max_k, total_k, tile), (int64_t)total_q * H, (int64_t)total_k * H, d, tile};
}

BwdParts layout(const Call& c, int32_t n_q, int32_t n_k) {
  BwdParts p{n_q, n_k, c.tile, 0, 0, 0, 0};
  p.stat_offset = align256((int64_t)sizeof(BwdPlan) + (c.tiles_q * n_q + c.tiles_k * n_k) * (int64_t)sizeof(BwdTile));
  p.q_offset = p.stat_offset + align256(2 * c.rows_q * 4);
  p.k_offset = p.q_offset + (n_q > 1 ? align256(n_q * c.rows_q * c.d * 4) : 0);
  p.bytes = p.k_offset + (n_k > 1 ? align256(2 * n_k * c.rows_k * c.d * 4) : 0);
  return p;
}
}  // namespace

namespace {
// When the last of `cus` workgroups ends that take a_items of a us, then b_items of b us (a >= b), the next one when one is
// done.  In closed form: it is asked for up to 64 times in a call of 20 us.
double ends(int64_t cus, int64_t a_items, double a, int64_t b_items, double b) {
  const int64_t rounds = a_items / cus, more = a_items % cus, rest = cus - more;  // `more` have one of a's more
  const double ratio = a / b, upto = (double)(rounds + (more > 0)) * a;
  if (b_items == 0) return upto;
  // the end is that of a b after b's from `rounds` a's on, i of them, or from one a more, j of them
  auto by_i = [&](int64_t i) { return rest * i + more * (int64_t)std::max(0.0, (double)i - ratio); };
  auto by_j = [&](int64_t j) { return more * j + rest * (int64_t)((double)j + ratio); };
  int64_t i = (int64_t)((double)(b_items + more * ratio) / (double)cus);
  while (by_i(i) < b_items) ++i;
  while (i > 0 && by_i(i - 1) >= b_items) --i;
  double t = (double)rounds * a + (double)i * b;
  if (more > 0) {
    int64_t j = (int64_t)std::max(0.0, (double)(b_items - rest * ratio) / (double)cus);
    while (by_j(j) < b_items) ++j;
    while (j > 0 && by_j(j - 1) >= b_items) --j;
    t = std::min(t, (double)(rounds + 1) * a + (double)j * b);
  }
  return std::max(t, upto);
}
}  // namespace

// The ranges that the library takes: those whose call ends first by an estimate, in us as measured.  A CU takes `product` of them for
// the product of a tile and 64 rows (four on either side: of dq the last one is two), and at least `alone` of them pass in a
// workgroup, or as many as those that share its CU take; beside its products an item takes kItem; joining ranges kJoin and, to write
// and read them, kMegabyte each.  1560 x 32760 x 12 heads (d = 128) take 1335 us with one range a side and 1076 as chosen, 2730 x
// 2730 x 12 heads 248 and 192, 1560 x 1560 x 2 heads (d = 64) 33 and 25; none of eleven calls took over 10 % more than the best of eight
// forced numbers of ranges.
BwdParts bwd_parts(int32_t nseq, int32_t max_q, int32_t max_k, int32_t total_q, int32_t total_k, int32_t H, int32_t d,
                   int32_t num_splits, int64_t workspace, int32_t cus) {
  const Call c = call(nseq, max_q, max_k, total_q, total_k, H, d);
  if (num_splits > 0) return layout(c, num_splits, num_splits);
  const double product = d == 64 ? 0.23 : c.tile == 256 ? 0.81 : 0.43, alone = d == 64 ? 0.27 : c.tile == 256 ? 0.81 : 0.64;
  const double kItem = 3.0, kJoin = 8.0, kMegabyte = 0.43;
  const int64_t items_q = c.tiles_q * H, items_k = c.tiles_k * H;
  if (items_q == 0 || items_k == 0 || items_q + items_k >= 16 * (int64_t)cus) return layout(c, 1, 1);  // (the last ones matter little)
  // steps of 64 rows that stream past a tile: of uneven segments, between the longest's and the mean
  auto steps = [&](int32_t most, int32_t total) { return (int32_t)ceil_div(((int64_t)most + std::min(most, total / nseq)) / 2, 64); };
  const int32_t steps_k = std::max(1, steps(max_k, total_k)), steps_q = std::max(1, steps(max_q, total_q));
  const double part = kMegabyte * 4e-6 * d;
  double least = 0;
  int32_t best_q = 1, best_k = 1;
  for (int32_t n_q : {1, 2, 3, 4, 6, 8, 12, 16}) {
    if (n_q > steps_k) break;
    for (int32_t n_k : {1, 2, 3, 4, 6, 8, 12, 16}) {
      if (n_k > steps_q) break;
      const int32_t in_q = 4 * ((steps_k + n_q - 1) / n_q), in_k = 4 * ((steps_q + n_k - 1) / n_k);  // products of an item
      const double q = product * in_q + kItem, k = product * in_k + kItem;
      double t = in_q > in_k ? ends(cus, items_q * n_q, q, items_k * n_k, k) : ends(cus, items_k * n_k, k, items_q * n_q, q);
      const int64_t beside = std::min<int64_t>(bwd_groups(d, c.tile), (items_q * n_q + items_k * n_k) / cus + 1);
      t = std::max(t, std::max(alone, product * (double)beside) * std::max(in_q, in_k) + kItem);
      if (n_q * n_k > 1) t += 0.03 * t + kJoin + part * (double)((n_q > 1 ? n_q * c.rows_q : 0) + (n_k > 1 ? 2 * n_k * c.rows_k : 0));
      if (least != 0 && t >= least) continue;
      if (n_q * n_k > 1 && layout(c, n_q, n_k).bytes > workspace) continue;
      least = t;
      best_q = n_q;
      best_k = n_k;
    }
  }
  return layout(c, best_q, best_k);
}

int64_t bwd_items(int32_t nseq, int32_t max_q, int32_t max_k, int32_t total_q, int32_t total_k, int32_t H, int32_t n_q, int32_t n_k,
                  int32_t tile) {
  return H * (bwd_tiles(nseq, max_q, total_q, tile) * n_q + bwd_tiles(nseq, max_k, total_k, tile) * n_k);
}

int64_t bwd_forced_items(int32_t nseq, int32_t max_q, int32_t max_k, int32_t total_q, int32_t total_k, int32_t H, int32_t d, int32_t n) {
  return bwd_items(nseq, max_q, max_k, total_q, total_k, H, n, n, call(nseq, max_q, max_k, total_q, total_k, H, d).tile);
}

int64_t bwd_least_workspace(int32_t nseq, int32_t max_q, int32_t max_k, int32_t total_q, int32_t total_k, int32_t H, int32_t d,
                            int32_t num_splits) {
  return layout(call(nseq, max_q, max_k, total_q, total_k, H, d), std::max(1, num_splits), std::max(1, num_splits)).bytes;
}

}  // namespace tsblock
