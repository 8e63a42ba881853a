/*
 * Attention of trees of drafted tokens over a cache, for AMD MI355X (gfx950).  Keys and values lie in
 * the pages of a cache (kvcache.h): those of a prefix that all sequences share (prefix_len 0: none),
 * read once for all, and each sequence's own, with its tree's behind them.
 *
 * Sequence b has n = suffix_lens[b] keys of its own and q_len nodes, queries b * q_len ... of q, whose keys
 * are its keys n, n + 1, ...  Node i sees
 *     all prefix_len keys of the prefix, the sequence's keys below n,
 *     and key n + j where bit j of masks[b][i] is set (a node's own bit and those of the nodes that it comes from)
 * and query head h uses the key and value head h / (q_heads / kv_heads):
 *     z_j = scale * (q . k_j);  out = sum_j softmax(z)_j v_j;  lse = log sum_j exp(z_j)
 * A node that sees no key gets zeros and lse = -infinity.  Padding (nodes that a sequence has not) has masks
 * of 0: it sees the keys below n, and none sees it.  What lies in masked places is not looked at, NaN
 * and infinities neither.  A mask need not be a tree's; a lower triangle is prefixattn.h's order.
 *
 * Numerics, partial results and what out and lse are good for: as in prefixattn.h.
 * Status codes, pointer kinds and error text as in addrms.h.
 */
#ifndef TREEATTN_H
#define TREEATTN_H

#include "prefixattn.h"
#include "treeaccept.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of device memory that a call of this shape keeps partial results in; depends on nothing else.  q_len is the
 * number of nodes of each sequence, up to TREE_MAX_NODES; suffix_width holds contexts and nodes. */
int64_t treeattn_workspace_bytes(const prefixattn_shape* shape);

/* Asynchronous, one launch or two.  As prefixattn_run, but
 *   suffix_lens   device, int32 [batch]: keys of each sequence before its tree; a number below 0 counts as 0.
 *                 Keys beyond the row of pages are not there
 *   masks         device, int64 [batch][q_len]; bits from q_len on are not looked at
 * batch == 0 or q_len == 0 is a no-op.  Never synchronises, never allocates; can be captured into a HIP graph: page
 * tables, lengths and masks are read when it is replayed. */
int treeattn_run(const void* q, const int64_t* q_strides, const void* k_pages, const void* v_pages,
                 const uint8_t* k_scale, const uint8_t* v_scale, const int32_t* prefix_pages,
                 const int32_t* suffix_pages, const int32_t* suffix_lens, const int64_t* masks, void* out, float* lse,
                 float scale, const prefixattn_shape* shape, void* workspace, int64_t workspace_bytes, void* stream);

/* Bytes that a call must move whose sequences hold suffix_keys keys together, their trees' among them: queries, masks,
 * prefix and keys read once, out and lse written. */
int64_t treeattn_algorithmic_bytes(const prefixattn_shape* shape, int64_t suffix_keys);

#ifdef __cplusplus
}
#endif
#endif /* TREEATTN_H */
