// cache_plan.cpp -- host-side sizes of the session cache's launches, shared by the argument checks of
// ts_cache.cpp and the launch code; no device code.
#include <stdint.h>

#include <algorithm>

#include "cache_launch.h"

namespace tscache {

namespace {
int64_t ceil_div(int64_t a, int64_t b) { return a / b + (a % b != 0); }
}  // namespace

// Up to 64 rows two tiles of 32, which read the pages twice, cost less than one of 256 with a quarter of its waves at work:
// 32 sessions of 16384 keys x 8 heads x 64 rows, d = 128, 307 against 419 us, 8 of 8192 keys x 40 heads 208 against 282, at d = 64 122
// against 143 (but see call_tile).  With 96 rows and three tiles the large one is ahead.
// Scale 0 is left to the row kernel: with a factor of 0 the tile kernel's masked scores would not vanish.
int row_tile(int64_t rows, float scale) {
  return rows <= 16 ? 16 : rows <= 64 || scale == 0.0f ? 32 : kTileRows;
}

// 33 to 64 rows that the library divides as it likes: where a few heads' keys are enough for a key range to each CU and no more,
// the ranges of 256-row tiles are fewer and longer than the row kernel's, and the pages are read once.  Both sides, us, row kernel
// against large tiles, 64 rows, d = 128 (d = 64): 12 heads x 4096 keys 23 / 20 (19 / 19), 12 x 16384 44 / 32 (31 / 25), 12 x 32768 56 / 50 (39 / 36),
// 40 x 4096 39 / 26 (26 / 21), 80 x 2048 39 / 27 (25 / 21), 96 x 4096 53 / 50 (34 / 36).  Less work than that ends together (12 x 2048 19 / 19,
// 40 x 512 14 / 16); more is bound by reading, where row tiles of every session go better together (48 x 16384 76 / 83,
// 24 x 32768 76 / 84, 128 x 2048 44 / 46); and few heads of long sessions have too few ranges (8 x 32768 47 / 59).
int call_tile(int32_t nseq, int64_t rows, int32_t max_len, int32_t H, int32_t d, float scale, int32_t num_splits) {
  const int tile = row_tile(rows, scale);
  const int64_t heads = (int64_t)nseq * H;
  if (num_splits != 0 || tile == kTileRows || scale == 0.0f || rows <= 32) return tile;
  if (heads < 8 || heads > (d == 64 ? 48 : 96) || max_len <= 768 || max_len > 2800 * heads) return tile;
  const int64_t keys = heads * max_len;
  return keys >= (d == 64 ? 90000 : 45000) && keys <= 400000 ? kTileRows : tile;
}

int64_t attn_items(int32_t nseq, int32_t max_rows, int32_t total, int32_t H, int32_t G, int tile) {
  const int64_t heads = (int64_t)nseq * H;
  if (tile == kTileRows)  // sum_s ceil(rows_s / tile) <= (all rows + nseq (tile - 1)) / tile
    return std::min<int64_t>(4 * kGridLimit / H, ((int64_t)total * G + (int64_t)nseq * (tile - 1)) / tile) * H;
  const int64_t tiles = ceil_div((int64_t)max_rows * G, tile);
  // nseq * H * tiles, saturating well above the limit
  return tiles > 0 && heads > 4 * kGridLimit / tiles ? 4 * kGridLimit : heads * tiles;
}

int64_t merge_blocks(int32_t nseq, int32_t max_rows, int32_t Hq, int32_t d) {
  const int64_t per = ceil_div((int64_t)max_rows * Hq * (d / 8), kMergeThreads);
  return per > 0 && nseq > 4 * kGridLimit / per ? 4 * kGridLimit : nseq * per;
}

namespace {
Parts parts(int32_t n_split, int32_t shares, int64_t rows, int32_t d) {
  const int64_t o_offset = (rows * 4 + 255) / 256 * 256;
  return {n_split, shares, o_offset, rows > 0 ? o_offset + rows * d * 4 : 0};
}
Parts ranges(int32_t n, int32_t total, int32_t Hq, int32_t d) {
  return parts(n, 0, n > 1 ? (int64_t)n * total * Hq : 0, d);
}
}  // namespace

Parts attn_parts(const Sessions& ss, int32_t H, int32_t G, int32_t d, int tile, int32_t num_splits, int64_t workspace,
                 int32_t cus) {
  int32_t n = std::max(1, num_splits);
  if (num_splits == 0) {
    const int64_t items = std::max<int64_t>(1, attn_items(ss.nseq, ss.max_rows, ss.total, H, G, tile));
    if (tile < kTileRows) {
      // Four workgroups a CU, and a page at least to each of their four waves.  Up to 768 tokens one workgroup is done
      // as soon as ranges and their merge are, and takes one launch (9.0 against 10.0 us at 512 tokens, 10.8 and 10.9 at
      // 768, 12.8 and 11.3 at 1024).
      const int64_t want = 4 * (int64_t)cus / items;
      if (ss.max_len > 768) n = (int32_t)std::max<int64_t>(1, std::min<int64_t>({want, ceil_div(ss.max_len, kPage) / 4, 64}));
      while (n > 1 && ranges(n, ss.total, H * G, d).bytes > workspace) --n;
    } else if (items < kEvenItems * (int64_t)cus) {
      const int64_t tiles = ceil_div(ss.max_len, d == 64 ? 2 * kPage : kPage), cost = items * (tiles + kStartCost);  // at most
      // Ranges that fill the device when all sessions have the stated length, as one has; costs in key tiles.  They are
      // also what small calls take, where the shares' longer start counts for more: two sessions of 512 and 1536 keys x 256
      // rows x 4 heads 23 us, in shares 38.
      const bool known = ss.nseq == 1 || ceil_div(cost, cus) < kEvenCost;
      int64_t best = INT64_MAX;
      for (int32_t i = 1; known && i <= 16 && (i == 1 || tiles / i >= kCutMin); ++i) {
        const int64_t c = ceil_div(items * i, cus) * (ceil_div(tiles, i) + kStartCost) + (i > 1 ? kMergeCost : 0);
        if (c < best && ranges(i, ss.total, H * G, d).bytes <= workspace) best = c, n = i;
      }
      const int64_t shares = std::min<int64_t>(cus, ceil_div(cost, kShareMin));
      const Parts p = parts(1, (int32_t)shares, 2 * shares * kTileRows, d);
      // (of one session, whose row tiles in ranges read the same keys at one time and in shares do not, only where ranges
      // leave a sixth of the device idle: see Work in cache_tiles.hip)
      const bool even = ss.nseq == 1 ? ceil_div(cost, shares) * 7 / 6 + kJoinCost < best : !known;
      if (even && shares > 1 && p.bytes <= workspace) return p;
    }
  }
  return ranges(n, ss.total, H * G, d);
}

int32_t weigh_rows(int32_t nseq, int32_t max_rows, int32_t max_len, int32_t H, int32_t G, int32_t cus) {
  if ((int64_t)max_rows * G > 64) return 0;
  const int64_t items = (int64_t)nseq * H;  // below the launch limit, as weigh_items is
  return (int32_t)std::max<int64_t>(1, std::min(8 * (int64_t)cus / items, ceil_div(max_len, 4 * kPage)));
}

bool weigh_few(int32_t nseq, int32_t max_len, int32_t H, int32_t cus) {
  return (int64_t)nseq * H * ceil_div(max_len, 4 * kPage) <= 2 * (int64_t)cus;
}

int64_t weigh_share(int32_t max_len, int32_t H) { return ceil_div((int64_t)H * ceil_div(max_len, 4 * kPage), 8); }

int64_t weigh_items(int32_t nseq, int32_t max_len, int32_t H) {
  const int64_t share = weigh_share(max_len, H);
  return share > 0 && nseq > kGridLimit / share ? 4 * kGridLimit : 8 * (int64_t)nseq * share;
}

int64_t append_items(int32_t nseq, int32_t max_rows, int32_t H) {
  // max_rows new tokens lie in at most that many pages, one more than the full ones on each side
  const int64_t pages = ((int64_t)max_rows + 2 * kPage - 2) / kPage, heads = (int64_t)nseq * H;
  return pages > 0 && heads > 4 * kGridLimit / pages ? 4 * kGridLimit : heads * pages;
}

int64_t gather_items(int32_t nseq, int32_t keep, int32_t H) {
  const int64_t pages = ceil_div(keep, kPage), heads = (int64_t)nseq * H;
  return pages > 0 && heads > 4 * kGridLimit / pages ? 4 * kGridLimit : heads * pages;
}

}  // namespace tscache
