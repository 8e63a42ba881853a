// What the host side of prefixattn and its kernel units share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace serving {

// Partial results: part p of [prefix splits, then suffix splits], row = token * q_heads + head:
//   part_o [parts][rows][d] fp32, relative to part_ml [parts][rows] = (base-2 exponent, sum of weights).
struct AttnArgs {
    uint64_t q, k_pages, v_pages, k_scale, v_scale, prefix_pages, suffix_pages, suffix_lens, out, lse, part_o, part_ml;
    int64_t q_token, q_head;                          // strides in elements
    int32_t batch, q_len, q_heads, kv_heads, group, d, page_shift, pages;
    int32_t prefix_len, prefix_splits, prefix_chunk, prefix_tiles, prefix_blocks;
    int32_t suffix_width, suffix_splits, suffix_chunk, suffix_tiles;
    uint32_t page_bytes, page_rows, head_bytes;       // of a page: all its heads, and one
    int32_t inline_len;                               // keys of a short prefix that each suffix's workgroup sees itself, before its own
    int32_t finish;                                   // the suffixes' workgroups join the prefix's parts to their own, and write the output
    int32_t q_wide;                                   // queries can be read 16 bytes at a time
    float c;                                          // scale * log2(e): weights are powers of 2
    // Trees (treeattn.hip): masks of their nodes, whose keys follow suffix_lens; parts that the sequences' keys are cut into, together, but
    // for one more of each; the shortest; and whether sequences come in the order of their lengths.
    uint64_t masks;
    int32_t cut_parts, cut_least, sorted;
};

// Forms of a workgroup: 16 rows whose four (FEW_8: eight) waves take keys in turn; 64, 128 or 256 rows that share their keys (64:
// heads up to 128; 256: heads of 65 to 128).
enum : int { FEW = 0, MANY_64 = 1, MANY_128 = 2, MANY_256 = 3, FEW_8 = 4 };
// Threads of a workgroup; heads over 128 leave no registers for two of 128 rows on a CU.
constexpr int threads_of(int form, int padded_head) { return form == FEW_8 || form == MANY_256 || (form == MANY_128 && padded_head > 128) ? 512 : 256; }
constexpr int kJoinThreads = 256;
constexpr int kJoinColumns = 64;                      // of a tree's row, where several workgroups join it
constexpr int kFormRows[] = {16, 64, 128, 256, 16};
constexpr int kChunkStep = 128;                       // splits begin at multiples of this many keys: every tile is aligned
constexpr int kFinishSplits = 64;                     // of a prefix that is joined by the suffixes' workgroups: a part a lane
constexpr int kMaxSplits = 256;                       // of a prefix, and of a suffix

// One for each element type, format and padded head size (prefixattn_unit.hip; for trees treeattn_unit.hip).
typedef hipError_t (*AttnLaunch)(const AttnArgs&, int prefix_form, int suffix_form, unsigned blocks, hipStream_t);
#define ATTN_UNIT_NAME(dt, fmt, dp) attn_launch_d##dt##_f##fmt##_h##dp
#define ATTN_UNIT(dt, fmt, dp) ATTN_UNIT_NAME(dt, fmt, dp)
#define ATTN_DECLARE(dt, fmt) \
    hipError_t ATTN_UNIT(dt, fmt, 64)(const AttnArgs&, int, int, unsigned, hipStream_t);  \
    hipError_t ATTN_UNIT(dt, fmt, 128)(const AttnArgs&, int, int, unsigned, hipStream_t); \
    hipError_t ATTN_UNIT(dt, fmt, 256)(const AttnArgs&, int, int, unsigned, hipStream_t);
ATTN_DECLARE(0, 0) ATTN_DECLARE(0, 1) ATTN_DECLARE(1, 0) ATTN_DECLARE(1, 1)
#undef ATTN_DECLARE
#define TREE_UNIT_NAME(dt, fmt, dp) tree_launch_d##dt##_f##fmt##_h##dp
#define TREE_UNIT(dt, fmt, dp) TREE_UNIT_NAME(dt, fmt, dp)
#define TREE_DECLARE(dt, fmt) \
    hipError_t TREE_UNIT(dt, fmt, 64)(const AttnArgs&, int, int, unsigned, hipStream_t);  \
    hipError_t TREE_UNIT(dt, fmt, 128)(const AttnArgs&, int, int, unsigned, hipStream_t); \
    hipError_t TREE_UNIT(dt, fmt, 256)(const AttnArgs&, int, int, unsigned, hipStream_t);
TREE_DECLARE(0, 0) TREE_DECLARE(0, 1) TREE_DECLARE(1, 0) TREE_DECLARE(1, 1)
#undef TREE_DECLARE

}  // namespace serving
