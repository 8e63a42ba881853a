/*
 * Attention of a batch that shares a long prefix, for AMD MI355X (gfx950).  Keys and values lie
 * in the pages of a cache (kvcache.h), those of the prefix once; they are read once for all
 * queries of the batch, and each sequence's own suffix for its own queries.
 *
 * Sequence b has q_len queries, tokens b * q_len ... b * q_len + q_len - 1 of q, the last q_len
 * positions of the sequence.  With n = suffix_lens[b], query i sees
 *     all prefix_len keys of the prefix, and of the suffix the keys j with j <= n - q_len + i
 * and query head h uses the key and value head h / (q_heads / kv_heads):
 *     z_j = scale * (q . k_j);  out = sum_j softmax(z)_j v_j;  lse = log sum_j exp(z_j)
 * A query that sees no key gets zeros and lse = -infinity.  What lies in masked places (the rest
 * of a page, a later token) is not looked at, NaN and infinities neither.
 *
 * Scores, sums and their maxima are fp32; softmax weights are rounded to the activations' type
 * for the product with the values (half a unit in its last place, relative, each), partial
 * results of splits are fp32, and the output is rounded once.  out and lse are what
 * mergestates.h merges, should a caller have keys elsewhere, too.
 *
 * Status codes, pointer kinds and error text as in addrms.h.
 */
#ifndef PREFIXATTN_H
#define PREFIXATTN_H

#include "kvcache.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Sizes of a call: host. */
typedef struct prefixattn_shape {
    int32_t batch;          /* sequences                                                   */
    int32_t q_len;          /* queries of each; batch * q_len * q_heads up to 2^24         */
    int32_t q_heads;        /* a multiple of kv_heads, up to 65536                         */
    int32_t kv_heads;
    int32_t d;              /* a multiple of 16 up to KVCACHE_MAX_HEAD                     */
    int32_t page_size;      /* a power of two up to 65536                                  */
    int64_t pages;          /* of the cache, below 2^31                                    */
    int64_t prefix_len;     /* keys that all share, 0 for none; below 2^30                 */
    int64_t suffix_width;   /* pages that a sequence's row of suffix_pages holds; times page_size below 2^30 */
    int32_t dtype;          /* ADDRMS_BF16 or ADDRMS_FP16                                  */
    int32_t format;         /* KVCACHE_*                                                   */
} prefixattn_shape;

/* Bytes of device memory that a call of this shape keeps partial results in; depends on nothing else. */
int64_t prefixattn_workspace_bytes(const prefixattn_shape* shape);

/* Asynchronous, one launch or two.
 *   q             device, [batch * q_len, q_heads, d], last axis contiguous, q_strides: host, {token, head}, in elements
 *   k_pages ...   device, as in kvcache.h
 *   prefix_pages  device, int32, at least ceil(prefix_len / page_size); NULL if prefix_len is 0
 *   suffix_pages  device, int32 [batch][suffix_width]; NULL if suffix_width is 0
 *   suffix_lens   device, int32 [batch]: keys of each suffix, the queries' own among them; a number below 0
 *                 counts as 0, one beyond the row of pages as its end.  NULL if suffix_width is 0
 *                 A page number outside the cache is a page of masked keys.
 *   out           device, [batch * q_len, q_heads, d], contiguous, 16-byte aligned; must not overlap q
 *   lse           device, fp32 [batch * q_len, q_heads], or NULL
 *   scale         > 0, and finite times log2(e): up to 2.35e38
 *   workspace     device, 16-byte aligned, workspace_bytes >= prefixattn_workspace_bytes(shape); not for two
 *                 calls at a time, free again when the call's work is done
 * batch == 0 or q_len == 0 is a no-op.  Never synchronises, never allocates; can be captured into a HIP graph: page
 * tables and lengths are read when it is replayed. */
int prefixattn_run(const void* q, const int64_t* q_strides, const void* k_pages, const void* v_pages,
                   const uint8_t* k_scale, const uint8_t* v_scale, const int32_t* prefix_pages,
                   const int32_t* suffix_pages, const int32_t* suffix_lens, void* out, float* lse, float scale,
                   const prefixattn_shape* shape, void* workspace, int64_t workspace_bytes, void* stream);

/* Bytes that a call must move whose suffixes hold suffix_keys keys together: queries, prefix and suffixes read once, out and lse written. */
int64_t prefixattn_algorithmic_bytes(const prefixattn_shape* shape, int64_t suffix_keys);

#ifdef __cplusplus
}
#endif
#endif /* PREFIXATTN_H */
