// block_launch.h -- internal interface between the C ABI of the transformer block's calls (ts_block.cpp) and its
// kernels (qk_rope.hip, attn_bwd.hip).  Not installed; the public interface is include/ts_block.h.
#pragma once
#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace tsblock {

// Rows of heads (ts_rows), or p = null.
struct Rows {
  void* p;
  int64_t stride;
  int32_t heads;
};

// Rotation (ts_rope); freq null: none.
struct Rope {
  const int32_t* pos;
  const double* freq;
  int32_t n0, n01;  // pairs of the first axis, of the first two
  int32_t interleaved;
};

struct RopeArgs {
  Rows q, k, q_out, k_out;
  const float* q_weight;
  const float* k_weight;
  Rope rope;
  int32_t T, d;
  float eps;
};

struct RopeBwdArgs {
  Rows dq_out, dk_out, q, k, dq, dk;
  const float* q_weight;
  const float* k_weight;
  float* dq_weight;
  float* dk_weight;
  float* part;  // [rope_bwd_blocks][2][d]: sums of each workgroup
  Rope rope;
  int32_t T, d;
  float eps;
};

constexpr int kRopeThreads = 256;
constexpr int kRopeBwdBlocks = 512;  // at most: as many as 256 CUs hold at once
// The workgroups of a gradient call with weights, whatever the device: its sums' order goes by them.
int32_t rope_bwd_blocks(int32_t T, int32_t q_heads, int32_t k_heads, int32_t d);

// What a call's workgroups do, in the order of the plan: a list of tiles for each segment and side, a tile being the
// held rows of a workgroup (keys for dk and dv, queries for dq) and one range of the rows that stream past them.  Each entry of a list
// says the same; the list's items are its tiles and ranges for every head, from first * H on: head, range, tile.
struct BwdTile {
  int32_t held0, held_len, str0, str_len;  // the segment's rows of either side
  int32_t first, tiles;                    // the list's first entry; tiles of one range
  int32_t keys, unused;
};
struct BwdPlan {  // ahead of its entries
  int32_t tiles;
  int32_t unused[7];
};
struct BwdOffsets {
  const int32_t* cu_q;
  const int32_t* cu_k;
  int32_t nseq, max_q, max_k, total_q, total_k;
};

struct BwdArgs {
  const void* d_o;
  const void* q;
  const void* k;
  const void* v;
  const void* o;
  const float* lse;
  void* dq;
  void* dk;
  void* dv;
  const int32_t* cu_q;
  const int32_t* cu_k;
  BwdPlan* plan;
  float* stat;     // [2][H][total_q]: -lse / scale, -D
  float* part_q;   // [n_q][total_q][H][d], where n_q > 1
  float* part_k;   // [n_k][total_k][H][d] of dk, then of dv, where n_k > 1
  int32_t nseq, max_q, max_k, total_q, total_k, H, d;
  int32_t n_q, n_k, tile;
  float scale;
};

// A workgroup of ts_attn_bwd holds `tile` queries (dq) or keys (dk, dv), 32 a wave; the rows of the other side come into LDS
// bwd_step at a time; a CU runs bwd_groups of them at once.
constexpr int bwd_step(int d, int tile) { return d == 128 && tile == 128 ? 32 : 64; }
constexpr int bwd_groups(int d, int tile) { return d == 64 ? 3 : tile == 128 ? 2 : 1; }

// How a call is divided: its tiles, the keys of a query tile in n_q ranges, the queries of a key tile in n_k; the workspace's layout.
struct BwdParts {
  int32_t n_q, n_k, tile;
  int64_t stat_offset, q_offset, k_offset, bytes;  // the plan comes first
};
BwdParts bwd_parts(int32_t nseq, int32_t max_q, int32_t max_k, int32_t total_q, int32_t total_k, int32_t H, int32_t d,
                   int32_t num_splits, int64_t workspace, int32_t cus);
// What the call needs at least: of forced ranges, or of the undivided call that the library falls back to.
int64_t bwd_least_workspace(int32_t nseq, int32_t max_q, int32_t max_k, int32_t total_q, int32_t total_k, int32_t H, int32_t d,
                            int32_t num_splits);
// An upper bound of the tiles of one side over all segments: sum of ceil(len / tile).
int64_t bwd_tiles(int32_t nseq, int32_t most, int32_t total, int32_t tile);
// Workgroups of the gradients' main kernel, 2 * tile threads each; and of ranges that the caller forces, as the call divides it.
int64_t bwd_items(int32_t nseq, int32_t max_q, int32_t max_k, int32_t total_q, int32_t total_k, int32_t H, int32_t n_q, int32_t n_k,
                  int32_t tile);
int64_t bwd_forced_items(int32_t nseq, int32_t max_q, int32_t max_k, int32_t total_q, int32_t total_k, int32_t H, int32_t d, int32_t n);

hipError_t configure_kernels();
hipError_t launch_rope(const RopeArgs& a, hipStream_t st);
hipError_t launch_rope_bwd(const RopeBwdArgs& a, hipStream_t st);
hipError_t launch_attn_bwd(const BwdArgs& a, hipStream_t st);

}  // namespace tsblock
