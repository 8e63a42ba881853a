/*
 * The path through a tree of drafted tokens that agrees with the model, for AMD MI355X (gfx950).
 *
 * A sequence has `nodes` drafted tokens, tokens[b][i], after its `suffix_lens[b]` keys in the cache; node 0 is
 * the last token that is certain.  Bit j of masks[b][i] says that node j is node i or one that it
 * comes from (the masks that treeattn.h attends with).  chosen[b][i] is the token that the model
 * gives after node i, the best one or one drawn.
 *
 * The path begins at node 0.  From node i it goes on to the child whose token is chosen[b][i], the
 * lowest where there are several; child c of node i is one whose mask is masks[b][i] with bit c
 * besides.  It ends where there is none, or after `depth` nodes.  A sequence whose masks[b][0] has
 * no bit 0 has no path.  Nodes that are padding have masks of 0.
 *
 *   path[b][k]       the path's nodes, -1 beyond its end
 *   count[b]         how many: so many keys are the sequence's from now on
 *   next_token[b]    chosen of the path's last node: the token that follows; -1 without a path
 *   from_slots[b][k], to_slots[b][k]   slots of the key of the path's k-th node, which lies at
 *                    position suffix_lens[b] + path[b][k] of its row of pages, and of position
 *                    suffix_lens[b] + k, where it belongs: what kvmove.h moves in groups of `depth`
 *                    tokens (of up to its KVMOVE_MAX_TOKENS; a path has TREE_MAX_NODES at most).
 *                    Both -1 where it is there already, beyond the path, and where either
 *                    position is beyond the row of pages or on a page outside the cache
 *
 * Status codes, pointer kinds and error text as in addrms.h.
 */
#ifndef TREEACCEPT_H
#define TREEACCEPT_H

#include "addrms.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TREE_MAX_NODES 64

/* One asynchronous launch.
 *   chosen, tokens         device, int32 [batch][nodes]
 *   masks                  device, int64 [batch][nodes]; bits from `nodes` on are not looked at
 *   suffix_pages           device, int32 [batch][suffix_width]
 *   suffix_lens            device, int32 [batch]; a number below 0 counts as 0
 *   path                   device, int32 [batch][depth]
 *   count, next_token      device, int32 [batch]
 *   from_slots, to_slots   device, int64 [batch][depth], or both NULL (then suffix_pages and suffix_lens may be, too)
 * 1 <= nodes <= TREE_MAX_NODES; depth from 1 to 65536; batch below 2^24; page_size a power of two up to 65536; pages
 * below 2^31; suffix_width * page_size below 2^30.  batch == 0 is a no-op.  Outputs must not overlap inputs.
 * Never synchronises, never allocates; can be captured. */
int treeaccept_run(const int32_t* chosen, const int32_t* tokens, const int64_t* masks, const int32_t* suffix_pages,
                   const int32_t* suffix_lens, int32_t* path, int32_t* count, int32_t* next_token, int64_t* from_slots,
                   int64_t* to_slots, int64_t batch, int32_t nodes, int32_t depth, int64_t suffix_width, int64_t pages,
                   int32_t page_size, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TREEACCEPT_H */
