/*
 * ts_block.h -- C ABI of libts_block.so: what a transformer block does around attention on MI355X (gfx950),
 * norms and rotation of queries and keys, and the gradients of a training step.
 *
 * A streaming model's block normalises the queries and keys of every head, rotates them by their tokens'
 * places in the latent video (frame, row, column), and attends (ts_attn.h; or, in serving, appends the keys
 * to the session's cache and attends to that, ts_cache.h).  A training step goes back the same way:
 *
 *   ts_qk_rope -> ts_attn_fwd_kvcache (with its log-sum-exp) -> ... -> ts_attn_bwd -> ts_qk_rope_bwd
 *
 * Conventions of ts_attn.h hold here too: host checks first, ts_status results (named by
 * ts_attn_status_str of libts_attn.so), asynchronous on the caller's stream, no state kept between calls,
 * thread safe, bitwise reproducible results (no atomics, fixed orders of sums), nothing but kernels enqueued
 * (every call can be captured into a HIP graph once its device has been used outside capture,
 * TS_ERR_CAPTURE before that), tensors of zero rows may be NULL.  No call allocates device memory; those that
 * need scratch take it from the caller, who may use it for another call once this one is done.
 * All pointers are DEVICE memory unless it says HOST.
 */
#ifndef TS_BLOCK_H
#define TS_BLOCK_H

#include <stdint.h>

#include "ts_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TS_BLOCK_ABI_VERSION 1

/* Rows of heads: bfloat16, head h of token t at p + t * stride + h * d.  A projection's fused rows of queries,
 * keys and values are three of these with one stride.  p is 16-byte aligned; stride, in elements, is a
 * multiple of 8, heads * d at least, and below 2^30. */
typedef struct ts_rows {
  void* p;
  int64_t stride;
  int32_t heads;
} ts_rows;

/* Rotation by positions on three axes (time, height, width).  The d / 2 pairs of a head's channels go by one axis
 * each: the first axes[0] by pos[t][0], the next axes[1] by pos[t][1], the last axes[2] by pos[t][2]; pair i
 * turns by the angle pos * freq[i] (radians).  A frequency of 0 leaves its pair alone.  The angle is formed
 * and reduced in 64 bits, so positions may be anywhere in int32. */
typedef struct ts_rope {
  const int32_t* pos;   /* [T][3] */
  const double* freq;   /* [d / 2] */
  int32_t axes[3];      /* not negative, d / 2 in all */
  int32_t interleaved;  /* pair i is channels (2i, 2i + 1); if 0, channels (i, i + d / 2) */
} ts_rope;

/*
 * Norm and rotation of queries and keys, in one pass over them:
 *   x' = x * w / sqrt(mean over the head of x^2 + eps)      where there are weights, else x' = x
 *   (a, b) of x' becomes (a cos - b sin, a sin + b cos)     where there is a rope
 * for every token and head, in 32 bits (squares summed in 64), rounded to bfloat16 once.
 *  q, k          T tokens; k may be NULL (queries alone), and then k_out is NULL too
 *  q_out, k_out  as many heads as q and k; each is q's or k's own memory (the same p and stride) or overlaps
 *                no input and no other output (TS_ERR_ALIAS)
 *  q_weight, k_weight  float32 [d], or NULL: no norm
 *  rope          HOST struct, or NULL: no rotation
 *  d             64 or 128
 *  eps           a positive normal float (TS_ERR_SCALE)
 * T tokens times all heads must stay below 2^31 - 2^16 (TS_ERR_SHAPE).
 */
int ts_qk_rope(const ts_rows* q, const ts_rows* k, const ts_rows* q_out, const ts_rows* k_out, const float* q_weight,
               const float* k_weight, const ts_rope* rope, int32_t T, int32_t d, float eps, void* stream);

/*
 * Its gradients.  dq_out and dk_out are those of ts_qk_rope's results, q, k, weights and rope what it was given.
 *  dq, dk        gradients of q and k; each is dq_out's or dk_out's own memory, or q's or k's, or overlaps no
 *                input and no other output
 *  dq_weight, dk_weight  float32 [d]: the sums over tokens and heads, 128 terms at most in 32 bits and those sums in 64; NULL
 *                where the weight is
 *  q, k          may be NULL where their weight is (the rotation's gradient needs no input)
 *  workspace     (256-byte aligned) ts_qk_rope_bwd_workspace bytes; less gives TS_ERR_SCRATCH.  0 bytes are
 *                needed, and it may be NULL, where there are no weights.
 * With T = 0 the gradients of the weights are 0.
 */
int ts_qk_rope_bwd(const ts_rows* dq_out, const ts_rows* dk_out, const ts_rows* q, const ts_rows* k, const ts_rows* dq,
                   const ts_rows* dk, const float* q_weight, const float* k_weight, float* dq_weight, float* dk_weight,
                   const ts_rope* rope, int32_t T, int32_t d, float eps, void* workspace, int64_t workspace_bytes,
                   void* stream);

/* Bytes of workspace that ts_qk_rope_bwd needs where there are weights (0 for sizes that it refuses). */
int64_t ts_qk_rope_bwd_workspace(int32_t T, int32_t q_heads, int32_t k_heads, int32_t d);

/*
 * Gradients of the packed attention of ts_attn_fwd_kvcache (and so of ts_attn_fwd_varlen, with the same offsets for
 * queries and keys, and of ts_attn_fwd, with offsets L apart): segment s's queries
 * [cu_seqlens_q[s], cu_seqlens_q[s+1]) over its keys [cu_seqlens_k[s], cu_seqlens_k[s+1]).  From the result
 * o, its log-sum-exp lse and the gradient d_o of o:
 *   P[t,j] = exp(scale * <q[t], k[j]> - lse[t])       (computed again, never stored; 0 where lse[t] is -infinity)
 *   D[t]   = <d_o[t], o[t]>
 *   dv[j]  = sum_t P[t,j] * d_o[t]
 *   S[t,j] = P[t,j] * (<d_o[t], v[j]> - D[t])
 *   dq[t]  = scale * sum_j S[t,j] * k[j]
 *   dk[j]  = scale * sum_t S[t,j] * q[t]
 * per head.  P and S are formed in 32 bits and rounded to bfloat16 for the products they enter, S of dq in two parts (its
 * rounded value and the rounded rest); sums are 32 bits.
 *  q, o, d_o, dq   bfloat16 [total_q][H][d];  k, v, dk, dv  bfloat16 [total_k][H][d];  lse  float32 [total_q][H]
 *  cu_seqlens_q/k  int32, nseq + 1 entries each, read on the device only, under the rules of ts_attn_fwd_kvcache: they
 *                  start at 0, do not descend, end at total_q / total_k, and no segment is longer than its
 *                  max_seqlen.  Offsets that break them make the call a device-side no-op (the gradients are left
 *                  unwritten); with TS_ATTN_VALIDATE=1 the call instead synchronizes and returns
 *                  TS_ERR_SEGMENTS (not on a capturing stream).  Without segments (nseq = 0) nothing is done either, and
 *                  validation mode names rows that belong to none.  Segments may be empty on either side: queries
 *                  without keys get dq = 0, keys without queries dk = dv = 0.
 *  scale           0, or a float of magnitude 2^-100 to 2^100 (TS_ERR_SCALE)
 *  num_splits      0: the library divides the work.  n in 1..16: the keys of each query tile and the queries of each key tile
 *                  are taken in n ranges, whose 32-bit sums another kernel adds up in order.
 *  workspace       (256-byte aligned) ts_attn_bwd_workspace bytes for these sizes; with less, a forced n, or the
 *                  undivided call, gives TS_ERR_SCRATCH, and the library divides less.
 * The bits of a segment's gradients depend on its own rows and on the division; with n >= 1 on nothing else.
 * No output may overlap another one, an input or the workspace (TS_ERR_ALIAS).  Sizes, TS_ERR_SHAPE:
 * (max_seqlen + 256) * H * d * 2 below 2^31 for each side, and for the work items nseq * H * (max_seqlen_q / 128 +
 * max_seqlen_k / 128 + 2) below 2^26 and H * (total / 128 + nseq) below 2^19 for each side; of n >= 2 ranges
 * n * H * (tiles of queries + tiles of keys) below 2^23, tiles being of 128 or 256 rows, with a last one for each segment (never
 * reached where n * H * (total_q / 128 + total_k / 128 + 2 nseq) is below that).
 */
#define TS_ATTN_BWD_MAX_SPLITS 16
int ts_attn_bwd(const void* d_o, const void* q, const void* k, const void* v, const void* o, const float* lse, void* dq,
                void* dk, void* dv, const int32_t* cu_seqlens_q, const int32_t* cu_seqlens_k, int32_t nseq,
                int32_t max_seqlen_q, int32_t max_seqlen_k, int32_t total_q, int32_t total_k, int32_t H, int32_t d,
                float scale, int32_t num_splits, void* workspace, int64_t workspace_bytes, void* stream);

/* Bytes of workspace that ts_attn_bwd makes use of for these sizes on the current device (0 for sizes that it refuses). */
int64_t ts_attn_bwd_workspace(int32_t nseq, int32_t max_seqlen_q, int32_t max_seqlen_k, int32_t total_q,
                              int32_t total_k, int32_t H, int32_t d, int32_t num_splits);

/* TS_BLOCK_ABI_VERSION of the built library. */
int ts_block_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* TS_BLOCK_H */
