/*
 * attn_fp8_parts.h -- attention over parts of the KV cache of attn_fp8_cache.h: pages that
 * are chosen for the queries by bounds on their keys, and pages that the sequences of a batch
 * begin with.  Cache, batch, heads, statuses, alignment and streams are those of
 * attn_fp8_cache.h; a call validates its arguments before any HIP call, enqueues its kernels
 * on `stream`, allocates nothing and keeps nothing between calls.  Outputs and workspaces overlap
 * none of a call's other arrays.
 *
 * What the definition of attn_fp8_cache_fwd makes of a key does not depend on the other keys
 * but for groups of 32 in a page, so attention over parts of the cache is that of the whole
 * cache with the other keys left out.
 *
 * Lists.  The new tokens of a sequence are taken in runs of `run`, the last one of what is
 * left; a run and a KV head have one list of `take` pages:
 *   blocks   int32 [B][ceil(max_q / run)][Hkv][take], contiguous: block j of a sequence is the
 *            page pages[b][j], tokens j * page and on; below 0: none.
 */
#ifndef ATTN_FP8_PARTS_H
#define ATTN_FP8_PARTS_H

#include "attn_fp8_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Bounds of the pages that hold new tokens of the batch (as attn_fp8_cache_append touches
 * them): of each channel the least and the largest code of K over the page's tokens up to the
 * last new one, rounded outwards to a multiple of 1/2.  NaN codes count as 0.  Other pages'
 * bounds are left as they were.  A page's codes change when its scale grows, so its bounds are
 * taken again after each append to it.
 *   bounds   E4M3 [n_pages][Hkv][2][d] (least, largest), 16-byte aligned; on the K scale of
 *            the page.
 * T is looked at for the bound on the entries of cu, or with cu = NULL for the T / B new tokens
 * of each sequence.  B * Hkv is below 2^24 here (else ATTN_ERR_UNSUPPORTED), W as wide as a
 * table may be.  Pages that two sequences hold have to be full in both.
 */
int attn_fp8_cache_bounds(const attn_fp8_cache *cache, const attn_fp8_batch *batch, void *bounds, void *stream);

/*
 * The pages whose bounds allow the largest scores, for every run of new tokens and KV head.
 * The score of a block is the largest, over the run's tokens that see its first key and the
 * query heads of the group, of
 *   2^x sum_c max(Q_c least_c, Q_c largest_c),   Q = q 2^-e rounded to whole numbers (ties to even),
 * e the least whole number with |q| <= 127 2^e in all channels, x = e + k byte - 127 held to
 * -96 .. 96.  (All sums are exact in FP32.)  A query row with a channel that is not finite takes
 * no part; a block whose first key no other row sees scores -inf.  The list holds, in ascending
 * order, `take` of the blocks that the run's last token sees a key of and that have a page: the
 * first n_first, the last n_last, and those of the highest scores, equal ones from the lowest block
 * on.  What is left of the list is -1, and so are the lists of runs without tokens.
 *   q          as for attn_fp8_cache_fwd.
 *   bounds     of attn_fp8_cache_bounds, for all blocks that are seen.
 *   blocks     out.
 *   take       1 .. 16384; n_first, n_last >= 0, together at most take.  With causal = 1 the pages
 *              that a run's own tokens lie in are among the last 1 + ceil((run - 1) / page): with a
 *              smaller n_last a list may lack the own page of the run's earlier tokens, and such a
 *              token may see no key.
 *   run        >= 1.
 *   max_len    no lens[b] is larger (keys from max_len on are not seen); 0: W * page.  More than
 *              16384 blocks are ATTN_ERR_UNSUPPORTED.  The plan goes by it.
 *   workspace  256-byte aligned device memory of workspace_bytes, scratch of this call alone; at
 *              least what attn_fp8_cache_select_workspace_bytes gives, else ATTN_ERR_INVALID_ARG.
 *              NULL where that is 0.
 * Of the cache only k_scale is read.
 */
int attn_fp8_cache_select(const attn_fp8_cache *cache, const attn_fp8_batch *batch, const attn_fp8_heads *q, int Hq,
                          const void *bounds, int32_t *blocks, int take, int run, int n_first, int n_last, int causal,
                          int max_len, void *workspace, size_t workspace_bytes, void *stream);
int attn_fp8_cache_select_workspace_bytes(const attn_fp8_cache *cache, const attn_fp8_batch *batch, int Hq, int take,
                                          int run, int max_len, size_t *bytes);

/*
 * attn_fp8_cache_fwd with the keys of a run's list in the place of all (of them those that a
 * query sees).  A block that is listed twice counts twice; one that has no page, or none of the
 * sequence's keys, not at all.
 *   blocks, take, run   as above (of any origin and order); take at most 2^19.
 *   the others          as for attn_fp8_cache_fwd; the sequences' lengths are not bounded here.
 *   workspace           as there, of attn_fp8_cache_blocks_workspace_bytes.
 */
int attn_fp8_cache_fwd_blocks(const attn_fp8_cache *cache, const attn_fp8_batch *batch, const attn_fp8_heads *q, int Hq,
                              const int32_t *blocks, int take, int run, void *out, int out_type, float *lse, int causal,
                              float sm_scale, float q_descale, void *workspace, size_t workspace_bytes, void *stream);
int attn_fp8_cache_blocks_workspace_bytes(const attn_fp8_cache *cache, const attn_fp8_batch *batch, int Hq, int take,
                                          int run, size_t *bytes);

/*
 * attn_fp8_cache_fwd for a batch whose sequences begin with the same `shared` pages: the result
 * of that call (in another order of FP32 sums), with the shared pages read once for the queries
 * of all sequences.  Entries 0 .. shared - 1 of the page table are read from sequence 0's row,
 * those of the other sequences are not looked at.
 *   shared     0 .. W.
 *   the others as for attn_fp8_cache_fwd; Hq / Hkv times T is at most 2^24 here, else
 *              ATTN_ERR_UNSUPPORTED.
 *   workspace  as there, of attn_fp8_cache_shared_workspace_bytes.
 */
int attn_fp8_cache_fwd_shared(const attn_fp8_cache *cache, const attn_fp8_batch *batch, int shared,
                              const attn_fp8_heads *q, int Hq, void *out, int out_type, float *lse, int causal,
                              float sm_scale, float q_descale, int max_len, void *workspace, size_t workspace_bytes,
                              void *stream);
int attn_fp8_cache_shared_workspace_bytes(const attn_fp8_cache *cache, const attn_fp8_batch *batch, int shared, int Hq,
                                          int max_len, size_t *bytes);

#ifdef __cplusplus
}
#endif

#endif /* ATTN_FP8_PARTS_H */
