/*
 * ts_cache.h -- C ABI of libts_cache.so, the 8-bit paged session cache for MI355X (gfx950).
 *
 * A streaming session keeps the keys and values of its earlier chunks as isolated state (paper Sec. 2
 * and 6.1).  Here that state lives in a pool of pages of 64 tokens, in 8 bits, and a session is a row of
 * page numbers: it grows page by page without moving, pages of many sessions share one pool, a suspend
 * copies whole pages (ts_state_copy), and a session that outgrows its budget keeps the tokens that
 * attention used most.
 *
 * The pool (struct ts_cache), all DEVICE memory owned by the caller:
 *   k, v          e4m3 (OCP, no infinities) [pages][H][64][d], 16-byte aligned; d is 64 or 128
 *   k_exp, v_exp  uint8 [pages][H]: a stored element stands for e4m3 * 2^(exp - 127); 255 makes the
 *                 page's elements NaN.  ts_cache_append and ts_cache_evict write exponents in 27..247,
 *                 and every element of such a page is exact in bfloat16; tokens of a page with any other
 *                 exponent, and elements of 2^128 and more, have unspecified values.
 *   weight        float32 [pages][H][64] (16-byte aligned): the attention weight each token has
 *                 collected.  May be NULL where a call does not use it (ts_cache_attn; append, which
 *                 then clears nothing).
 * Sessions of a call (nseq of them):
 *   table  int32 [nseq][width]: session s's token j lies in page table[s][j / 64], slot j % 64.  Entries
 *          past the session's last page are not used.  A page may appear in one session once; sessions
 *          may share pages that a call only reads.
 *   lens   int32 [nseq]: tokens of every session.
 *   cu     int32 [nseq + 1]: session s's rows of the packed q, o, k, v are [cu[s], cu[s+1]).
 * These three are DEVICE memory, read on the device only.  What they hold is checked there: a session
 * whose length is outside [0, max_len] or beyond 64 * width, or whose rows are not inside [0, total] or
 * outnumber max_rows, is skipped (nothing of it is written; other sessions are not affected; sessions
 * whose rows overlap leave those rows unspecified).  A page number outside [0, pages) is never
 * followed: such a page reads as NaN (and its weights as -infinity), and nothing is written to it.
 * With the environment variable TS_ATTN_VALIDATE=1 a call synchronizes and returns
 * TS_ERR_SEGMENTS for any of these instead (not on a capturing stream).
 *
 * Conventions of ts_attn.h hold here too: host checks first, ts_status results (named by
 * ts_attn_status_str of libts_attn.so), asynchronous on the caller's stream, no state kept between calls,
 * bitwise reproducible results, thread safe, nothing but kernels enqueued (every call can be captured into
 * a HIP graph once its device has been used outside capture, TS_ERR_CAPTURE before that), tensors of zero
 * rows may be NULL.  No call allocates device memory; the one that needs scratch takes it from the caller.
 * H counts the cached heads and Hq = G * H the query heads: query head hq reads cached head hq / G.
 * Size limits: (max_rows + 256) * Hq * d * 2 and (64 * width + 256) * d must stay below 2^31, and the
 * workgroups of a launch below 2^23 (TS_ERR_SHAPE).
 */
#ifndef TS_CACHE_H
#define TS_CACHE_H

#include <stdint.h>

#include "ts_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TS_CACHE_ABI_VERSION 1
#define TS_CACHE_PAGE 64 /* tokens of a page */

typedef struct ts_cache {
  void* k;
  void* v;
  uint8_t* k_exp;
  uint8_t* v_exp;
  float* weight;
  int32_t pages;
  int32_t H;
  int32_t d;
} ts_cache;

/*
 * Appends each session's new tokens: k, v bfloat16 [total][H][d] (16-byte aligned), session s's rows
 * [cu[s], cu[s+1]) becoming its tokens lens[s], lens[s] + 1, ...  new_lens (DEVICE int32 [nseq], no
 * overlap with lens) receives lens[s] + the session's rows; for a skipped session, lens[s].  A session
 * is also skipped when its new length passes 64 * width.
 * Per page and head, n is the least integer >= -100 with |x| <= 448 * 2^n for every finite new element x
 * (-100 where there is none); a page that already holds tokens of the session keeps at least its exponent.
 * exp = n + 127, elements are stored as x * 2^-n rounded to nearest even (infinities and NaN as NaN; where
 * exp is 247, as 240 at most, since 256 * 2^120 is no bfloat16), and older tokens of a page whose exponent
 * rises are rounded again.  The new tokens' weights become 0; other
 * slots stay as they are.  The sessions' written pages must be distinct.
 */
int ts_cache_append(const ts_cache* cache, const void* k, const void* v, const int32_t* cu,
                    const int32_t* table, const int32_t* lens, int32_t* new_lens, int32_t nseq,
                    int32_t width, int32_t max_rows, int32_t total, void* stream);

/*
 * Attention of each session's query rows over its lens[s] cached tokens, keys of the queries' own chunk
 * among them if they have been appended:
 *   o[t,hq,:] = sum_j softmax_j(scale * <q[t,hq,:], k[j,hq/G,:]>) * v[j,hq/G,:]
 *   lse[t,hq] = ln sum_j exp(scale * <q[t,hq,:], k[j,hq/G,:]>)
 * q, o bfloat16 [total][Hq][d] (16-byte aligned); lse float32 [total][Hq] or NULL.  A session without
 * tokens gets o = 0 and lse = -infinity.  scale: any finite float.
 *  num_splits  0: the library divides the work, by the sessions' lengths where there are many rows; n in
 *              1..TS_CACHE_MAX_SPLITS: the keys of every query tile are split into n ranges of pages.  What
 *              is divided is joined by a second kernel, through float32 partial results in
 *  workspace   (DEVICE, 256-byte aligned, of this call alone until it is done): ts_cache_attn_workspace
 *              bytes.  With num_splits = 0 a smaller one, or NULL, divides less or not at all; a forced n
 *              that does not fit returns TS_ERR_SCRATCH.
 * The bits of a session's result depend on how its keys are divided, with num_splits = 0 on the call's
 * sizes and the other sessions' too; with n >= 1 on the session's own rows and length, on max_rows * G
 * (up to 16, up to 64, or more: another kernel each), and on whether scale is 0.
 * o, lse and workspace must not overlap each other or any input (TS_ERR_ALIAS).
 */
#define TS_CACHE_MAX_SPLITS 64
int ts_cache_attn(const ts_cache* cache, const void* q, void* o, float* lse, const int32_t* cu,
                  const int32_t* table, const int32_t* lens, int32_t nseq, int32_t width,
                  int32_t max_rows, int32_t max_len, int32_t total, int32_t Hq, float scale,
                  int32_t num_splits, void* workspace, int64_t workspace_bytes, void* stream);

/*
 * Bytes of workspace that ts_cache_attn makes use of for these sizes on the current device (0 for an
 * unsplit call, and for sizes that it refuses).
 */
int64_t ts_cache_attn_workspace(int32_t nseq, int32_t max_rows, int32_t max_len, int32_t total,
                                int32_t H, int32_t Hq, int32_t d, int32_t num_splits);

/*
 * Adds to each cached token the attention weight it gets from the queries:
 *   weight_out[j,h] = cache->weight[j,h] + sum over rows t of the session and heads hq of h's group of
 *                     exp(scale * <q[t,hq,:], k[j,h,:]> - lse[t,hq])
 * for the tokens j < lens[s] of each session (pages and slots as in cache->weight).  lse float32
 * [total][Hq] is ts_cache_attn's of the same queries: each row then hands out a weight of 1.  weight_out
 * is cache->weight itself or a buffer of its size that overlaps nothing; other slots of it stay as they
 * are.  The sessions' pages must be distinct.  Sums are float32 in a fixed order.
 */
int ts_cache_weigh(const ts_cache* cache, const void* q, const float* lse, const int32_t* cu,
                   const int32_t* table, const int32_t* lens, float* weight_out, int32_t nseq,
                   int32_t width, int32_t max_rows, int32_t max_len, int32_t total, int32_t Hq,
                   float scale, void* stream);

/*
 * Cuts every session down to `keep` tokens per head, into new pages.  Session s has len = lens[s] tokens;
 * if len <= keep all of them stay.  Otherwise each head keeps its first `first` tokens, its last `last`
 * tokens, and of the others the keep - first - last with the largest weight (of equal weights the earlier
 * token; NaN counts as -infinity): heads may keep different tokens.  The kept tokens move, in order, to
 * slots 0, 1, ... of the pages new_table[s][0], [1], ... (int32 [nseq][new_width], 64 * new_width >=
 * keep), with their weights, stored with the exponent that ts_cache_append would give these elements.
 * Slots past the last kept token, and pages past its page, stay as they are; so do the old pages.
 *  new_lens  DEVICE int32 [nseq]: min(len, keep); for a skipped session, its lens[s]
 *  kept      DEVICE int32 [nseq][H][keep]: the kept tokens' positions, ascending; -1 past new_lens.  Rows of
 *            skipped sessions are all -1.
 * first + last <= keep.  The new pages must be distinct and none of the sessions' old ones.
 */
int ts_cache_evict(const ts_cache* cache, const int32_t* table, const int32_t* lens,
                   const int32_t* new_table, int32_t* new_lens, int32_t* kept, int32_t nseq,
                   int32_t width, int32_t new_width, int32_t max_len, int32_t keep, int32_t first,
                   int32_t last, void* stream);

/* TS_CACHE_ABI_VERSION of the built library. */
int ts_cache_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* TS_CACHE_H */
