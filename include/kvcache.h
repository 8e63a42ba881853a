/*
 * A paged cache of keys and values for AMD MI355X (gfx950), quantised as it is written and read
 * back into 16 bits; prefixattn.h attends to it where it lies.
 *
 * Pages: k_pages and v_pages are [pages][heads][page_size][d], so that the tokens of one head in
 * a page lie one behind the other.  A token's place is its slot: page * page_size + offset.
 *   KVCACHE_SAME   elements of the activations' type (ADDRMS_BF16 or ADDRMS_FP16), copied
 *   KVCACHE_E4M3   one byte an element (OCP e4m3) and one scale byte s for each token and head,
 *                  k_scale and v_scale [pages][heads][page_size]; the value is code * 2^(s - 127).  A write
 *                  gives s from 1 to 254; 0 is 2^-127 to those who read, and 255 makes the row NaN
 *
 * Quantisation of a row x of d elements: a = max |x|; e = the least whole number with
 * a * 2^-e <= 448 (448 is the format's largest value), at least -126 and at most 127, and 0 for a
 * row of zeros; s = e + 127; code = x * 2^-e rounded to nearest, ties to even.  A power of two
 * changes no digit, so that the code's rounding (half of 2^-3 relative, 2^-10 absolute below
 * 2^-6) is the only one.  Before that, magnitudes above the largest value of four significant
 * bits that the type holds (fp16: 61440, bf16: 15 * 2^124) are set to it, so that reading back
 * cannot overflow.  NaN stays NaN, an infinity becomes NaN (the format has none), and neither
 * counts in a.
 *
 * Status codes, pointer kinds and error text as in addrms.h.
 */
#ifndef KVCACHE_H
#define KVCACHE_H

#include "addrms.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { KVCACHE_SAME = 0, KVCACHE_E4M3 = 1 };
#define KVCACHE_MAX_HEAD 256

/* Writes tokens into the cache: one asynchronous launch for keys and values.
 *   k, v         device, [tokens, heads, d], last axis contiguous, the others with strides in
 *                elements (host, {token, head})
 *   slots        device, int64 [tokens]; a token whose slot is negative or beyond the cache is
 *                left out.  A slot is to be named once: where two tokens name one, its place holds
 *                parts of either, also one's codes with the other's scale, and no other place changes
 *   k_pages ...  device, 16-byte aligned; k_scale, v_scale NULL for KVCACHE_SAME
 * d: a multiple of 16 up to KVCACHE_MAX_HEAD; page_size: a power of two up to 65536; heads up to 65536; pages
 * below 2^31; tokens * heads * (d / 8, up to a power of two) below 2^32, and tokens * heads below 2^31.
 * tokens == 0 is a no-op.  Never synchronises, never allocates; can be captured. */
int kvcache_write(const void* k, const int64_t* k_strides, const void* v, const int64_t* v_strides,
                  const int64_t* slots, void* k_pages, void* v_pages, uint8_t* k_scale, uint8_t* v_scale,
                  int64_t tokens, int32_t heads, int32_t d, int64_t pages, int32_t page_size,
                  int dtype, int format, void* stream);

/* Reads tokens back: k_out, v_out device, [tokens, heads, d] contiguous, 16-byte aligned.  A token whose slot
 * is negative or beyond the cache reads as zeros.  Otherwise as kvcache_write.  A value that is
 * not representable (an e4m3 code times a small power of two, in fp16) is rounded to nearest. */
int kvcache_read(const void* k_pages, const void* v_pages, const uint8_t* k_scale, const uint8_t* v_scale,
                 const int64_t* slots, void* k_out, void* v_out, int64_t tokens, int32_t heads, int32_t d,
                 int64_t pages, int32_t page_size, int dtype, int format, void* stream);

/* Bytes that a write or a read must move: tokens once in the type, once in the format, the slots. */
int64_t kvcache_algorithmic_bytes(int64_t tokens, int32_t heads, int32_t d, int dtype, int format);

#ifdef __cplusplus
}
#endif
#endif /* KVCACHE_H */
