/*
 * attn_fp8_cache.h -- the KV cache of libattn_fp8.so: an E4M3 cache in pages with
 * one power-of-two scale per page and KV head, the calls that write, read and
 * shrink it, and rotary positions.  Statuses, alignment, streams and errors are
 * those of attn_fp8.h: every pointer is device memory of the caller, a call
 * validates its arguments before any HIP call, enqueues its kernels on `stream`,
 * allocates nothing and keeps nothing between calls; no C++ exception crosses
 * this interface.
 *
 * The cache.  A page holds `page` = 64 or 128 tokens of all KV heads:
 *   k, v             [n_pages][Hkv][page][d]  E4M3 bytes, d = 64 or 128
 *   k_scale, v_scale [n_pages][Hkv]           E8M0 bytes: a code stands for
 *                                             code * 2^(byte - 127), byte <= 254
 * The byte of a block (one page of one head) is the least for which no value of
 * the block exceeds 448 * 2^(byte - 127), and at least 0; powers of two keep
 * every rescaling exact and are what the matrix cores' block scales take.
 *
 * The batch.  Sequence b holds lens[b] tokens, the call's new ones included, in
 * the pages pages[b][0 .. ceil(lens[b] / page)); token t is at slot t % page of
 * page pages[b][t / page].  The call's tokens are packed, [T][heads][d], those
 * of sequence b from cu[b] to cu[b + 1]: they are its last ones, token i of n is
 * position lens[b] - n + i.  cu = NULL: T / B tokens of each sequence.
 * lens, pages and cu are read on the device, so a captured call follows them:
 *   - lens[b] below 0 counts as 0; a page number outside 0 .. n_pages - 1 is no
 *     page, and what lies past the W pages of a sequence has none (W * page is at
 *     most 2^26, else ATTN_ERR_UNSUPPORTED).  Tokens without a page are not written,
 *     and no query sees them; nor are tokens before position 0, whose queries see
 *     no key;
 *   - T is at most 2^30 and a launch (by B, max_q, the heads and bounds, not by lens and
 *     cu) has less than 2^32 threads, else ATTN_ERR_UNSUPPORTED;
 *   - a sequence has at most max_q new tokens; those beyond are left out (not
 *     written, their rows of an output left as they were), as are cu entries
 *     outside 0 .. T.
 * Rows of q, out and lse behind cu[B] are not touched.
 */
#ifndef ATTN_FP8_CACHE_H
#define ATTN_FP8_CACHE_H

#include "attn_fp8.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element types of the calls' inputs and outputs */
enum { ATTN_TYPE_F32 = 0, ATTN_TYPE_BF16 = 1, ATTN_TYPE_F16 = 2, ATTN_TYPE_E4M3 = 3 };

/* which channels a rotation pairs: i with i + rot / 2, or 2 i with 2 i + 1 */
enum { ATTN_ROPE_HALF = 0, ATTN_ROPE_INTERLEAVED = 1 };

typedef struct attn_fp8_cache {
    void *k, *v;                     /* E4M3 [n_pages][Hkv][page][d], 16-byte aligned */
    uint8_t *k_scale, *v_scale;      /* E8M0 [n_pages][Hkv] */
    int n_pages, Hkv, page, d;
} attn_fp8_cache;

typedef struct attn_fp8_batch {
    const int32_t *pages;            /* [B][W] */
    const int32_t *lens;             /* [B] */
    const int32_t *cu;               /* [B + 1], or NULL: T / B tokens each (T % B == 0) */
    int B, W, T, max_q;              /* max_q >= 1; with cu = NULL at least T / B */
} attn_fp8_batch;

/* packed tokens [T][H][d] of an element type; strides in elements, channels
 * contiguous.  Addresses and strides are multiples of 16 bytes. */
typedef struct attn_fp8_heads {
    void *data;
    int64_t stride_t, stride_h;
    int type;
} attn_fp8_heads;

/* cos and sin of the rotations: FP32 [n_pos][rot / 2][2], 16-byte aligned; rot a
 * positive multiple of 16.  positions: int32 [T], the row of each packed token;
 * NULL: its position in the sequence (attn_fp8_cache_append only).  A position
 * outside 0 .. n_pos - 1 makes NaN of the channels it would rotate. */
typedef struct attn_fp8_rotation {
    const float *table;
    const int32_t *positions;
    int n_pos, rot, layout;
} attn_fp8_rotation;

/*
 * Rotary positions of packed heads: channels a, b of a pair i at position p
 * become a cos - b sin and b cos + a sin with (cos, sin) = table[p][i]; channels
 * from rot on are copied.  FP32, rounded once to the type of x.
 *   x, out     [T][H][d] of one type, F32, BF16 or F16; out may be x.
 *   d          a multiple of 16, at most 1024; rot <= d.
 * T or H = 0 is a no-op; T H d / 16 is below 2^32 (else ATTN_ERR_UNSUPPORTED).
 */
int attn_fp8_rope(const attn_fp8_heads *x, const attn_fp8_heads *out, int T, int H, int d,
                  const attn_fp8_rotation *rotation, void *stream);

/*
 * Writes the new tokens of a batch into its pages: k rotated (in 64 bits,
 * rounded once to E4M3), v as it is.  A block that gets its first tokens takes
 * the scale they need; in a block that holds older ones the scale only grows,
 * and the older codes are rounded to the grown scale.  Values that are not
 * finite become NaN codes and do not count towards the scale; a rotated value past
 * FP32's largest is one of them, one below 2^-126 is rounded to FP32's subnormals
 * first.  Pages that are written belong to one sequence alone.
 *   k, v       [T][Hkv][d] of one type, F32, BF16 or F16.
 *   rotation   NULL: none.
 *   q, q_out   optional (both or neither): [T][Hq][d] of k's type, rotated like
 *              attn_fp8_rope does; needs a rotation.
 */
int attn_fp8_cache_append(const attn_fp8_cache *cache, const attn_fp8_batch *batch,
                          const attn_fp8_heads *k, const attn_fp8_heads *v,
                          const attn_fp8_rotation *rotation, const attn_fp8_heads *q,
                          const attn_fp8_heads *q_out, int Hq, void *stream);

/*
 * Attention of the batch's new tokens over its cached ones.  Query head h reads
 * KV head h / (Hq / Hkv).  With D the dot product of q and the codes of key t,
 *   x_t = D 2^(k byte - 127) log2(e) sm_scale q_descale     (FP32)
 * over the keys the query sees: t <= its position with causal = 1, all lens[b]
 * with causal = 0 (none in either case for a token before position 0).  P is rounded to E4M3 in groups of 32 keys [32 g, 32 g + 32),
 * each relative to its own power of two:
 *   M_g = ceil(largest x_t of the group),  code_t = E4M3(2^8 2^(x_t - M_g)),
 * so no group underflows for another's maximum and neither the codes nor their
 * scales depend on the order in which the groups are visited:
 *   out = sum_g 2^(M_g - 8) sum_t code_t v_t / l,  l = sum_t 2^(x_t) before the cast,
 * sums in FP32 relative to a power of two per row (which may lie 2^16 below its
 * largest: sums of values beyond 2^111 / lens[b] may pass FP32's range); lse = ln l.
 * A query that sees no key gets out = 0 and lse = -inf.  The matrix cores add the
 * products of P V in eights and drop what lies 13 bits below the largest of them: 5e-5
 * to 1e-4 of the result (relative norm), below a BF16 out's rounding, visible in an F32 one.
 * The rounding of P itself is 1.7e-2 (777 keys) to 3.7e-2 (131001) of the softmax
 * over the same codes.
 *   q          [T][Hq][d], BF16 or E4M3 (F32 and F16 queries are the caller's to
 *              round); Hq / Hkv at most 256, times max_q at most 2^24
 *              (beyond: ATTN_ERR_UNSUPPORTED).
 *   out        contiguous [T][Hq][d], BF16 or F32 by out_type, 16-byte aligned.
 *   lse        FP32 [T][Hq], or NULL.
 *   sm_scale, q_descale   finite and > 0, and so log2(e) times their product: a normal
 *              FP32 number.
 *   max_len    no lens[b] is larger (keys from max_len on are not seen); 0: W * page.
 *              The plan goes by it, so a close bound is a faster call.
 *   workspace  256-byte aligned device memory of workspace_bytes, scratch of this
 *              call alone; at least what attn_fp8_cache_workspace_bytes gives,
 *              else ATTN_ERR_INVALID_ARG.  NULL where that is 0.
 */
int attn_fp8_cache_fwd(const attn_fp8_cache *cache, const attn_fp8_batch *batch,
                       const attn_fp8_heads *q, int Hq, void *out, int out_type, float *lse,
                       int causal, float sm_scale, float q_descale, int max_len,
                       void *workspace, size_t workspace_bytes, void *stream);

/* Workspace of attn_fp8_cache_fwd for these sizes on the current device (0: the
 * call takes none).  Only the sizes of cache and batch are looked at. */
int attn_fp8_cache_workspace_bytes(const attn_fp8_cache *cache, const attn_fp8_batch *batch,
                                   int Hq, int max_len, size_t *bytes);

/*
 * Attention weight that the cached tokens receive: adds to weights[b][hk][t] the
 * softmax weights exp(z - lse) of key t over the new tokens and query heads of
 * the group that see it (z = x_t ln 2 as above).  lse is what attn_fp8_cache_fwd
 * gave for the same call (its FP32 rounding is in z - lse: weights are good while |lse|
 * is far below 2^23); a row of lse = -inf adds nothing.
 *   weights    FP32 [B][Hkv][..], stride_b and stride_h elements apart; entries
 *              t < min(lens[b], max_len) are updated, the others left as they
 *              were.  max_len 0: W * page.  max_len <= stride_h, and rows do not
 *              overlap: those of a sequence side by side, or those of a head.
 */
int attn_fp8_cache_weights(const attn_fp8_cache *cache, const attn_fp8_batch *batch,
                           const attn_fp8_heads *q, int Hq, const float *lse, int causal,
                           float sm_scale, float q_descale, int max_len, float *weights,
                           int64_t stride_b, int64_t stride_h, void *stream);

/*
 * Eviction: of every sequence and KV head the `budget` tokens that matter most
 * move, in their order, into new pages: the first n_sink, the last n_recent (of
 * what is left of the budget) and those of the largest weight; equal weights go
 * to the lower token, NaN counts as the lowest.  Sequences of at most budget
 * tokens move whole.  The moved block's scale is that of its own values.
 *   from, batch    the cache, of at least one page; of batch pages, lens, B and W
 *                  are used (T, max_q and cu are not, but have to be valid: T >= 0,
 *                  max_q >= 1).
 *   to, new_pages  the cache that takes them (it may be the same arrays) and
 *                  int32 [B][ceil(budget / page)]: pages that hold none of the
 *                  batch's tokens.  Its slots that get no token are left alone.
 *   weights        as above, entries t < lens[b] are read (<= stride_h).
 *   budget         1 .. 2^20.
 *   kept           int32 [B][Hkv][budget]: where each moved token was, then -1.
 *   new_lens       int32 [B]: min(lens[b], budget).
 *   new_weights    FP32 [B][Hkv][budget]: the moved tokens' weights, then 0; or NULL.
 * kept, new_lens and new_weights overlap neither each other nor lens, pages,
 * new_pages or weights (from its first row to the end of its last), else
 * ATTN_ERR_INVALID_ARG.
 */
int attn_fp8_cache_evict(const attn_fp8_cache *from, const attn_fp8_batch *batch,
                         const attn_fp8_cache *to, const int32_t *new_pages,
                         const float *weights, int64_t stride_b, int64_t stride_h, int budget,
                         int n_sink, int n_recent, int32_t *kept, int32_t *new_lens,
                         float *new_weights, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* ATTN_FP8_CACHE_H */
