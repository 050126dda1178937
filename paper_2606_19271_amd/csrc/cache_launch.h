// cache_launch.h -- internal interface between the C ABI of the session cache (ts_cache.cpp) and its
// kernels (cache_attn.hip, cache_tiles.hip, cache_weigh.hip, cache_pages.hip).  Not installed; the public interface is include/ts_cache.h.
#pragma once
#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace tscache {

constexpr int kPage = 64;               // tokens of a page
constexpr int kMergeThreads = 256;      // threads per workgroup of the merge kernel
constexpr int64_t kGridLimit = (int64_t)1 << 23;  // workgroups per launch

// The pool of pages (ts_cache).
struct Pool {
  uint8_t* k;
  uint8_t* v;
  uint8_t* k_exp;
  uint8_t* v_exp;
  float* weight;  // null where the call has none
  int32_t pages, H;
};

// The sessions of a call: packed rows cu[s] .. cu[s + 1] (null where the call has no rows), lens[s] cached
// tokens in the pages table[s][..].
struct Sessions {
  const int32_t* cu;
  const int32_t* table;
  const int32_t* lens;
  int32_t nseq, width, max_rows, max_len, total;
};

struct AttnArgs {
  Pool pool;
  Sessions ss;
  const void* q;
  void* o;
  float* lse;       // or null
  float* part_o;    // [n_split][total][Hq][d] (n_split > 1), [2 shares][256][d] (shares > 0)
  float* part_lse;  // the same without d
  int32_t d, G, tile, n_split, shares;
  float scale;
};

struct WeighArgs {
  Pool pool;
  Sessions ss;
  const void* q;
  const float* lse;
  float* out;
  int32_t d, G;
  float scale;
  int32_t cus;
};

struct AppendArgs {
  Pool pool;
  Sessions ss;  // max_len: 64 * width
  const void* k;
  const void* v;
  int32_t* new_lens;
  int32_t d;
};

struct EvictArgs {
  Pool pool;
  Sessions ss;
  const int32_t* new_table;
  int32_t* new_lens;
  int32_t* kept;
  int32_t d, new_width, keep, first, last;
};

// Host-side sizes (cache_plan.cpp).
// Query rows (tokens x G) of an attention workgroup's tile: 256 (cache_tiles_kernel), or 32 or 16
// (cache_rows_kernel); by the rows of a cached head at most, and by the call (call_tile).
constexpr int kTileRows = 256;
int row_tile(int64_t rows, float scale);
int call_tile(int32_t nseq, int64_t rows, int32_t max_len, int32_t H, int32_t d, float scale, int32_t num_splits);
// Workgroups of an unsplit attention call, and of its merge kernel.
int64_t attn_items(int32_t nseq, int32_t max_rows, int32_t total, int32_t H, int32_t G, int tile);
int64_t merge_blocks(int32_t nseq, int32_t max_rows, int32_t Hq, int32_t d);
// How the keys of an attention call are dealt out, and its workspace of partial results: every row tile's in n_split ranges of
// pages, as calls of few rows are, and 256-row tiles of one session or of little work; or those of several sessions in
// `shares` equal shares of the work.  A workspace that is too small makes them fewer or none.
struct Parts {
  int32_t n_split, shares;
  int64_t o_offset, bytes;  // the partial log-sum-exps lie first, then O
};
Parts attn_parts(const Sessions& ss, int32_t H, int32_t G, int32_t d, int tile, int32_t num_splits, int64_t workspace,
                 int32_t cus);
// Equal shares (Work in cache_tiles.hip), costs in key tiles: what an item costs beside its tiles, the least share, the
// least part of an item.  With kEvenItems row tiles a CU and more, whole ones end evenly enough;
// less than kEvenCost tiles a CU are not worth the shares.
constexpr int kStartCost = 4, kShareMin = 12, kCutMin = 4;
constexpr int kEvenItems = 2, kEvenCost = 40;
// In key tiles too, of 1.7 us at 1560 rows x 32760 keys x 12 heads, d = 128: what ranges cost beside their tiles (writing the parts, and the
// merge kernel's 8 us and its launch), and shares (finding them, 10 us, and the join kernel, 10 to 20).
constexpr int kMergeCost = 6, kJoinCost = 14;
// Workgroups of the other kernels.
// weigh: with up to 64 rows of a cached head, the parts that the pages of a session and head are dealt to (else 0: not this
// kernel); a page to a workgroup where there are few, else four pages of a head, in 8 XCDs x nseq sessions x weigh_share
// workgroups, at most weigh_items.
int32_t weigh_rows(int32_t nseq, int32_t max_rows, int32_t max_len, int32_t H, int32_t G, int32_t cus);
bool weigh_few(int32_t nseq, int32_t max_len, int32_t H, int32_t cus);
int64_t weigh_share(int32_t max_len, int32_t H);
int64_t weigh_items(int32_t nseq, int32_t max_len, int32_t H);
int64_t append_items(int32_t nseq, int32_t max_rows, int32_t H);
int64_t gather_items(int32_t nseq, int32_t keep, int32_t H);

hipError_t configure_kernels();
hipError_t launch_attn(const AttnArgs& a, hipStream_t st);
hipError_t launch_weigh(const WeighArgs& a, hipStream_t st);
hipError_t launch_append(const AppendArgs& a, hipStream_t st);
hipError_t launch_evict(const EvictArgs& a, hipStream_t st);

}  // namespace tscache
