// How calls of attention over a cache are checked and cut into workgroups: what prefixattn.hip and treeattn.hip share.
#pragma once
#include <math.h>

#include <algorithm>

#include "prefixattn.h"
#include "prefixattn_args.h"
#include "serving_internal.h"

namespace serving {

using namespace addrms_host;

constexpr int64_t kMaxRows = 1 << 24;        // queries by heads: their numbers, and those of what is formed of them, are 32 bits
// The shortest piece of keys; of a suffix as long as the prefix's, up to twice this.  128 beside 256, whole calls: 8 x 40 heads over
// 2000 bf16 keys 12.8 and 14.2 us, 2 x 40 over 900 e4m3 10.8 and 11.2, 8 x 40 over 8191 the same; a long prefix with the suffixes in
// pieces of 128 has too little room left: 4 x 32 heads over 131072 bf16 keys and suffixes of 2000 112 us, with pieces of 256 103.5.
constexpr int32_t kMinChunk = 128;
constexpr int64_t kInlineBytes = 1 << 27, kInlineChain = 3 << 16;      // of keys and values (see plan_of)
// From here on the suffixes alone fill the chip, and their workgroups join the prefix's parts.  From 64 on instead: 16 x 4 x 32 heads
// over 4096 fp16 keys and suffixes of 300 32 us a call in place of 25, 8 x 40 heads over 8191 e4m3 keys 28 in place of 16.
constexpr int64_t kFinishUnits = 256;
// From here on a wave joins a row, not four: 8192 rows of 128 46.8 us a call in place of 51.5, 2048 26.5 in place of 27.3, 1984 33.0 and
// 33.7, 1536 30.5 either way; 512 20.8 in place of 19.4.
constexpr int64_t kJoinRows = 1024;

inline int32_t splits_of(int64_t keys, int64_t units, int64_t wanted, int32_t shortest, int32_t* chunk)
{
    int64_t n = (wanted + units - 1) / units;
    if (n > (keys + shortest - 1) / shortest) n = (keys + shortest - 1) / shortest;
    if (n > kMaxSplits) n = kMaxSplits;
    if (n < 1) n = 1;
    const int64_t each = ((keys + n - 1) / n + kChunkStep - 1) / kChunkStep * kChunkStep;
    *chunk = static_cast<int32_t>(each);
    return static_cast<int32_t>((keys + each - 1) / each);
}

struct Plan {
    AttnArgs a;
    int prefix_form, suffix_form, dp;
    int64_t rows, prefix_blocks, suffix_blocks, bytes;
    bool finish;                             // the suffixes' workgroups are a launch of their own that joins the prefix's parts
};

// Whether launches hold a plan's workgroups.
inline int fits(const Plan& p)
{
    const int64_t beside = p.prefix_blocks + (p.finish ? 0 : p.suffix_blocks);
    if (launchable(beside, threads_of(p.prefix_form, p.dp)) && launchable(p.suffix_blocks, threads_of(p.suffix_form, p.dp))) return ADDRMS_OK;
    return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "the call is too large: %lld workgroups", (long long)(p.prefix_blocks + p.suffix_blocks));
}

// Checks a shape and fills in what does not depend on how the work is split; rows are 0 where there is none.
inline int shape_of(const prefixattn_shape* s, Plan* p)
{
    if (!s) return fail(ADDRMS_ERR_INVALID_ARG, "shape is NULL");
    if (s->dtype != ADDRMS_BF16 && s->dtype != ADDRMS_FP16) return fail(ADDRMS_ERR_UNSUPPORTED_DTYPE, "unsupported dtype %d for attention", s->dtype);
    if (s->format != KVCACHE_SAME && s->format != KVCACHE_E4M3) return fail(ADDRMS_ERR_INVALID_ARG, "unknown cache format %d", s->format);
    if (s->batch < 0 || s->q_len < 0 || s->q_heads <= 0 || s->kv_heads <= 0 || s->d <= 0 || s->pages < 0 || s->prefix_len < 0 || s->suffix_width < 0)
        return fail(ADDRMS_ERR_INVALID_ARG, "sizes must not be negative, heads and d must be > 0");
    if (s->q_heads % s->kv_heads != 0)
        return fail(ADDRMS_ERR_INVALID_ARG, "q_heads=%d is not a multiple of kv_heads=%d", s->q_heads, s->kv_heads);
    if (!power_of_two(s->page_size) || s->page_size > 65536)
        return fail(ADDRMS_ERR_INVALID_ARG, "page_size must be a power of two up to 65536 (got %d)", s->page_size);
    if (s->d % 16 != 0 || s->d > KVCACHE_MAX_HEAD)
        return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "d=%d is not a multiple of 16 up to %d", s->d, KVCACHE_MAX_HEAD);
    const int64_t width = s->suffix_width < (1ll << 30) ? s->suffix_width * s->page_size : 1ll << 30;
    if (s->pages >= (1ll << 31) || s->prefix_len >= (1ll << 30) || width >= (1ll << 30) || s->q_heads > 65536)
        return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "pages, keys or heads are beyond the limits (2^31, 2^30, 65536)");
    const int64_t page_rows = static_cast<int64_t>(s->page_size) * s->kv_heads, row_bytes = s->d * (s->format == KVCACHE_E4M3 ? 1 : 2);
    if (page_rows * row_bytes >= (1ll << 32)) return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "a page of %lld bytes is beyond the limit (2^32)", (long long)(page_rows * row_bytes));
    *p = Plan{};
    AttnArgs& a = p->a;
    a.batch = s->batch, a.q_len = s->q_len, a.q_heads = s->q_heads, a.kv_heads = s->kv_heads, a.group = s->q_heads / s->kv_heads, a.d = s->d;
    a.page_shift = log2_of(s->page_size), a.pages = static_cast<int32_t>(s->pages);
    a.prefix_len = static_cast<int32_t>(s->prefix_len), a.suffix_width = static_cast<int32_t>(s->suffix_width);
    a.page_rows = static_cast<uint32_t>(page_rows), a.page_bytes = static_cast<uint32_t>(page_rows * row_bytes);
    a.head_bytes = static_cast<uint32_t>(s->page_size * row_bytes);
    p->dp = s->d <= 64 ? 64 : s->d <= 128 ? 128 : 256;
    if (s->batch == 0 || s->q_len == 0) return ADDRMS_OK;
    const int64_t tokens = static_cast<int64_t>(s->batch) * s->q_len;
    if (tokens > kMaxRows || tokens * s->q_heads > kMaxRows)
        return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "%lld queries of %d heads are beyond the limit (2^24 together)", (long long)tokens, s->q_heads);
    p->rows = tokens * s->q_heads;
    return ADDRMS_OK;
}

// The least form that has the rows (with 64 rows in 128: 16 x 32 heads over 16384 keys, bf16 25.4 us and 26.0, e4m3 22.2 and 24.0).
// Heads over 128 go from 16 to 128: with 16 rows a wave, a form for 64 took 53 us in place of 41 for 20 rows over 16384 bf16 keys
// of 256, 54 and 53 for 32, 63 and 59 for 64 (in e4m3 36.5 and 41).  Heads up to 64 end with 128 rows: a tile of e4m3 keys has fewer
// pieces of 16 bytes than 512 threads, and in 16 bits a form for 256 rows takes 67.2 us in place of 72.1 for 64 x 64 heads over 32768
// keys, but 48.0 in place of 41.2 for 8 x 64 queries of 32 heads over 4096 and 46.1 in place of 39.3 for 2 x 512 over 1000.
inline int form_of(int64_t rows, int dp) { return rows <= 16 ? FEW : rows <= 64 && dp <= 128 ? MANY_64 : rows <= 128 || dp != 128 ? MANY_128 : MANY_256; }
inline int64_t tiles_of(int64_t rows, int form) { return (rows + kFormRows[form] - 1) / kFormRows[form]; }

// Checks the pointers of a call whose work is split, and hands them to the kernels.
inline int arguments_of(const void* q, const int64_t* q_strides, const void* k_pages, const void* v_pages, const uint8_t* k_scale, const uint8_t* v_scale,
                        const int32_t* prefix_pages, const int32_t* suffix_pages, const int32_t* suffix_lens, void* out, float* lse, float scale,
                        const prefixattn_shape* shape, void* workspace, int64_t workspace_bytes, Plan* p)
{
    const float c = scale * 1.44269504088896340736f;
    if (!(scale > 0.0f) || !(c < INFINITY)) return fail(ADDRMS_ERR_INVALID_ARG, "scale must be > 0, and finite times log2(e) (got %g)", static_cast<double>(scale));
    if (p->rows == 0) return ADDRMS_OK;
    AttnArgs& a = p->a;
    const bool codes = shape->format == KVCACHE_E4M3, keys = a.prefix_splits || a.suffix_splits, own = a.suffix_splits && shape->suffix_width;
    if (!q || !q_strides || !out || (keys && (!k_pages || !v_pages || (p->bytes && !workspace) || (codes && (!k_scale || !v_scale)))) ||
        ((a.prefix_splits || a.inline_len) && !prefix_pages) || (own && (!suffix_pages || !suffix_lens)))
        return fail(ADDRMS_ERR_INVALID_ARG, "no pointer may be NULL");
    if (workspace_bytes < p->bytes)
        return fail(ADDRMS_ERR_INVALID_ARG, "the workspace has %lld bytes, the call needs %lld", (long long)workspace_bytes, (long long)p->bytes);
    if (!aligned_to(q, 2) || !aligned_to(out, 16) || !aligned_to(lse, 4) || !aligned_to(k_pages, 16) || !aligned_to(v_pages, 16) ||
        !aligned_to(workspace, 16) || !aligned_to(prefix_pages, 4) || !aligned_to(suffix_pages, 4) || !aligned_to(suffix_lens, 4))
        return fail(ADDRMS_ERR_MISALIGNED, "pages, out and workspace must be 16-byte aligned, the others to their elements");
    a.q = addr(q), a.k_pages = addr(k_pages), a.v_pages = addr(v_pages), a.k_scale = addr(k_scale), a.v_scale = addr(v_scale);
    a.prefix_pages = addr(prefix_pages), a.suffix_pages = addr(suffix_pages), a.suffix_lens = addr(suffix_lens), a.out = addr(out), a.lse = addr(lse);
    a.part_o = addr(workspace);
    a.part_ml = a.part_o + 4ull * (p->bytes / (4ll * a.d + 8)) * a.d;
    a.q_token = q_strides[0], a.q_head = q_strides[1];
    a.q_wide = (a.q | static_cast<uint64_t>(q_strides[0] * 2) | static_cast<uint64_t>(q_strides[1] * 2)) % 16 == 0;
    a.c = c;
    a.prefix_blocks = static_cast<int32_t>(p->prefix_blocks);
    return ADDRMS_OK;
}

}  // namespace serving
