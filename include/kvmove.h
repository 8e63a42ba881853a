/*
 * Moving tokens in a paged cache (kvcache.h) for AMD MI355X (gfx950): accepted tokens of a draft go
 * behind their sequence, a fork gets copies of pages, pages are filled up.
 *
 * Tokens come in groups.  In each group, token i's keys and values, of all heads, and their scales
 * go from slot from_slots[g][i] to slot to_slots[g][i], as if all of the group were read before
 * one was written: a group may move tokens to slots that others of it come from.  Groups run in
 * any order, so that no group may write a slot that another one reads or writes, and a group
 * writes a slot once (where two tokens go to one slot, it holds parts of either).  A token whose
 * slots are not both in the cache (a negative number is not) stays where it is.
 *
 * Status codes, pointer kinds and error text as in addrms.h.
 */
#ifndef KVMOVE_H
#define KVMOVE_H

#include "kvcache.h"

#ifdef __cplusplus
extern "C" {
#endif

#define KVMOVE_MAX_TOKENS 256

/* One asynchronous launch for keys and values.
 *   k_pages ...             device, as in kvcache.h; dtype is the type of the elements that KVCACHE_SAME holds
 *   from_slots, to_slots    device, int64 [groups][tokens]
 * tokens (of a group): up to KVMOVE_MAX_TOKENS; the other sizes as for kvcache_write; groups * heads below 2^21.
 * groups == 0 or tokens == 0 is a no-op.  Never synchronises, never allocates; can be captured: the slots are
 * read when the graph is replayed. */
int kvmove_run(void* k_pages, void* v_pages, uint8_t* k_scale, uint8_t* v_scale, const int64_t* from_slots,
               const int64_t* to_slots, int64_t groups, int32_t tokens, int32_t heads, int32_t d, int64_t pages,
               int32_t page_size, int dtype, int format, void* stream);

/* Bytes that a call must move of whose tokens `moved` have both slots in the cache: those once read and once written, the slots. */
int64_t kvmove_algorithmic_bytes(int64_t groups, int32_t tokens, int64_t moved, int32_t heads, int32_t d, int format);

#ifdef __cplusplus
}
#endif
#endif /* KVMOVE_H */
