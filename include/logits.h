/*
 * Penalties for repeated tokens, biases and a grammar's masks on logits, and the best token of each
 * row, for AMD MI355X (gfx950).
 *
 * Sequence b has `nodes` rows, b * nodes ... b * nodes + nodes - 1: one for decoding, or the nodes of a tree of drafted
 * tokens.  For row i of sequence b and token t, with x the logit, every step rounded to fp32:
 *     made   = how often t is among the sequence's tokens history[b][prompt_lens[b] ... history_lens[b] - 1], plus how
 *              many of the nodes that bits of tree_masks[b][i] name have the token t (node 0, the last token that
 *              is certain, is one of them: the history ends before it, or it counts twice)
 *     met    = made > 0, or t is among history[b][0 ... prompt_lens[b] - 1]
 *     z = x                                      with (r, f, p) = penalties[b]:
 *     z = z > 0 ? z / r : z * r                  if met
 *     z = z - f * made                           if made > 0
 *     z = z - p                                  if made > 0
 *     z = z + (sum of bias_values[b][j] over the j with bias_tokens[b][j] = t, in their order)       if there are any
 *     z = -infinity                              if bit t % 32 of allowed[row][t / 32] is clear
 * out[row][t] = z, rounded to the logits' type; best[row] = the lowest t with the largest z (before that rounding), NaN
 * counting as larger than all numbers; a row all of whose tokens are ruled out has the best token 0.
 * Numbers in lists that are no tokens (below 0, or from vocab on) are passed over.
 *
 * Status codes, pointer kinds and error text as in addrms.h.
 */
#ifndef LOGITS_H
#define LOGITS_H

#include "treeaccept.h"

#ifdef __cplusplus
extern "C" {
#endif

#define LOGITS_MAX_BIASES 1023
#define LOGITS_MAX_HISTORY 1048575

/* What a call goes by: host; pointers device.  Lists that are not used are NULL. */
typedef struct logits_lists {
    const int32_t* history;         /* [batch], rows of history_width tokens, history_stride apart        */
    const int32_t* history_lens;    /* [batch]; below 0 counts as 0, beyond history_width as history_width */
    const int32_t* prompt_lens;     /* [batch], as history_lens, and beyond these as these; NULL: no prompts */
    const float* penalties;         /* [batch][3]: r, f, p; NULL: 1, 0, 0, and history is not looked at   */
    const int32_t* bias_tokens;     /* [batch][biases]                                                    */
    const float* bias_values;       /* [batch][biases]                                                    */
    const uint32_t* allowed;        /* [batch * nodes] rows, allowed_stride words apart; at least ceil(vocab / 32) words each */
    const int32_t* tree_tokens;     /* [batch][nodes]; NULL: rows are no nodes                            */
    const int64_t* tree_masks;      /* [batch][nodes]; bits from `nodes` on are not looked at             */
    int64_t history_stride;         /* elements                                                           */
    int64_t allowed_stride;         /* elements                                                           */
    int32_t history_width;          /* up to LOGITS_MAX_HISTORY                                           */
    int32_t biases;                 /* up to LOGITS_MAX_BIASES                                            */
} logits_lists;

/* Bytes of device memory that a call that asks for best keeps partial results in; depends on nothing else. */
int64_t logits_workspace_bytes(int64_t batch, int32_t nodes, int64_t vocab, int dtype);

/* Asynchronous; a launch, and one more for best.
 *   logits      device, [batch * nodes][vocab], rows logits_stride elements apart
 *   out         device, as logits, rows out_stride elements apart; NULL: not written.  It may be logits itself (same pointer
 *               and stride) and overlaps it in no other way
 *   best        device, int32 [batch * nodes]; NULL: not looked for
 *   workspace   device, 8-byte aligned, workspace_bytes >= logits_workspace_bytes(...), NULL without best; not for two
 *               calls at a time, free again when the call's work is done
 * dtype: ADDRMS_BF16, ADDRMS_FP16 or ADDRMS_FP32.  batch * nodes below 2^24, nodes up to 65536 (TREE_MAX_NODES where rows
 * are nodes of a tree), vocab from 1 to 2^24; batch * nodes == 0 is a no-op.  Never synchronises, never allocates; can be
 * captured: lists and lengths are read when the graph is replayed. */
int logits_run(const void* logits, int64_t logits_stride, void* out, int64_t out_stride, int32_t* best, int64_t batch,
               int32_t nodes, int64_t vocab, int dtype, const logits_lists* lists, void* workspace,
               int64_t workspace_bytes, void* stream);

/* Bytes that a call must move whose histories hold `tokens` tokens together. */
int64_t logits_algorithmic_bytes(int64_t batch, int32_t nodes, int64_t vocab, int dtype, int64_t tokens, int32_t biases,
                                 int masked, int write);

#ifdef __cplusplus
}
#endif
#endif /* LOGITS_H */
