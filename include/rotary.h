/*
 * Rotary positions with several axes for AMD MI355X (gfx950): what turns the queries and keys
 * of a decode step, a prefill chunk or a training step before they are attended with.
 *
 * A token has `axes` positions (one for text; time, height and width for images and video).
 * The first `rot` elements of each head are rot/2 pairs; pair i belongs to the axis
 * pair_axis[i] and turns by the angle
 *     a = positions[pair_axis[i]][t] * inv_freq[i]                       (64 bits)
 *     (x1, x2) -> (x1 cos a - x2 sin a, x1 sin a + x2 cos a)              (fp32, rounded once)
 * Pair i is the elements i and i + rot/2, or with ROTARY_INTERLEAVED 2i and 2i + 1.  Elements
 * from `rot` on are copied.  With ROTARY_INVERSE the angle is -a: the transposed map, that is,
 * the gradient of the inputs from the gradient of the outputs.
 *
 * Angles are formed and reduced to an eighth of a turn in 64 bits, so that positions of millions
 * turn by the right angle; sine and cosine are fp32, within 2 units in the last place.
 * Types: ADDRMS_BF16, ADDRMS_FP16, ADDRMS_FP32.  Status codes, pointer kinds and error text as
 * in addrms.h.
 */
#ifndef ROTARY_H
#define ROTARY_H

#include "addrms.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { ROTARY_INTERLEAVED = 1, ROTARY_INVERSE = 2 };
#define ROTARY_MAX_HEAD 256

/* One asynchronous launch for queries and keys.
 *   q, k         device, [tokens, heads, d], last axis contiguous, the others with strides in elements
 *                (q_strides, k_strides: host, {token, head}); k may be NULL with k_heads 0
 *   q_out, k_out device, as q and k with strides of their own; they may be q and k themselves
 *                (same pointer and strides: in place) and overlap the inputs in no other way
 *   positions    device, int64 [axes][tokens]
 *   inv_freq     device, fp64 [rot / 2], radians a position
 *   pair_axis    device, uint8 [rot / 2], below axes (a larger number counts as axes - 1)
 * rot is even, 2 <= rot <= d <= ROTARY_MAX_HEAD; 1 <= axes <= 255; q_heads + k_heads up to 65536; tokens below
 * 2^31, and of more than tokens * d = 2^32 some calls are refused.  tokens == 0 is a no-op.
 * Never synchronises, never allocates; can be captured into a HIP graph. */
int rotary_run(const void* q, const int64_t* q_strides, const void* k, const int64_t* k_strides,
               void* q_out, const int64_t* q_out_strides, void* k_out, const int64_t* k_out_strides,
               const int64_t* positions, const double* inv_freq, const uint8_t* pair_axis,
               int64_t tokens, int32_t q_heads, int32_t k_heads, int32_t d, int32_t rot, int32_t axes,
               int dtype, int flags, void* stream);

/* Bytes the operator must move: heads read and written once, positions read once. */
int64_t rotary_algorithmic_bytes(int64_t tokens, int32_t heads, int32_t d, int32_t axes, int dtype);

#ifdef __cplusplus
}
#endif
#endif /* ROTARY_H */
