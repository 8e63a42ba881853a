// Moving tokens in a paged cache (include/kvmove.h).
//
// A unit is one head's keys, or values, of a group: all of a unit's rows are read by one workgroup before it writes one, which is
// what a group may ask for, and no unit needs another.  A row is 1 to 32 neighbouring lanes of 16 bytes.  Bound by memory: 2048 groups of
// 16 x 8 x 128 bf16 (269 MB) in 54.6 us, 4.9 TB/s, as fast as a copy; 64 groups of 6 tokens 2.8 on the device, a launch.
// One row of a thread, two and four: 64 x 6 tokens of 8 x 128 e4m3 2.77, 2.95 and 2.98 us, 256 x 8 bf16 4.23, 4.34 and 4.59; much to move 56.6, 56.5
// and 56.0, e4m3 33.9, 32.5 and 30.3.  Past the caches that is 55.0, 54.6 and 55.1, and 26.2, 23.2 and 23.2; rows that are no whole lines are
// slower so (1000 x 7 x 4 x 96 e4m3 4.9 us in place of 4.4).
#include "kvmove.h"
#include "serving_internal.h"

using namespace addrms_host;
using namespace serving;

namespace {

constexpr int64_t kPastBytes = 4 << 20;      // of keys and values

struct MoveArgs {
    addr_t pages[2], scale[2], from, to;
    int64_t cache_slots;
    uint32_t tokens, heads, units, spans, pieces, lanes_log2, page_shift;        // units of a workgroup; workgroups of a group; 16-byte pieces of a row
    float per_token;                                                             // 1 / tokens
};

template <int FORMAT, int THREADS, int PER, bool PAST>
__global__ __launch_bounds__(THREADS) void move_kernel(MoveArgs a)
{
    const uint32_t group = blockIdx.x / a.spans, unit0 = (blockIdx.x - group * a.spans) * a.units;
    const uint32_t lane = threadIdx.x & ((1u << a.lanes_log2) - 1), row0 = threadIdx.x >> a.lanes_log2, step = THREADS >> a.lanes_log2;
    const uint32_t rows = min(a.units, 2 * a.heads - unit0) * a.tokens;
    const int64_t list = static_cast<int64_t>(group) * a.tokens;
    const uint32_t piece = min(lane, a.pieces - 1);
    int64_t from[PER], to[PER];                                 // slots, then rows of the cache; -1: stays
    uint32_t head[PER];
    bool values[PER];
    // Slots first, then rows, neither in a branch, so that all of them are under way together: where there is nothing to move, row 0 is
    // read and not written.
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const uint32_t row = row0 + i * step;
        // exact: at most 2^13 rows, and half a token's distance from the next unit
        const uint32_t unit = static_cast<uint32_t>((static_cast<float>(row) + 0.5f) * a.per_token), u = unit0 + unit;
        const int64_t at = list + (row - unit * a.tokens);
        from[i] = at_global<const int64_t>(a.from)[row < rows ? at : 0];
        to[i] = at_global<const int64_t>(a.to)[row < rows ? at : 0];
        if (row >= rows) to[i] = -1;
        head[i] = u >> 1;
        values[i] = u & 1;
    }
    u32x4 x[PER];
    uint8_t scale[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const bool there = static_cast<uint64_t>(from[i]) < static_cast<uint64_t>(a.cache_slots) && static_cast<uint64_t>(to[i]) < static_cast<uint64_t>(a.cache_slots);
        const auto row_of = [&](int64_t slot) {
            return (((slot >> a.page_shift) * a.heads + head[i]) << a.page_shift) + (slot & ((1ll << a.page_shift) - 1));
        };
        from[i] = there ? row_of(from[i]) : 0;
        to[i] = there ? row_of(to[i]) : -1;
        x[i] = at_global<const u32x4>(values[i] ? a.pages[1] : a.pages[0])[from[i] * a.pieces + piece];
        if constexpr (FORMAT == KVCACHE_E4M3) scale[i] = at_global<const uint8_t>(values[i] ? a.scale[1] : a.scale[0])[from[i]];
    }
    // everything is in registers before a wave writes
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (to[i] < 0) continue;
        if (lane < a.pieces) {
            u32x4* const p = at_global<u32x4>(values[i] ? a.pages[1] : a.pages[0]) + (to[i] * a.pieces + lane);
            if constexpr (PAST) __builtin_nontemporal_store(x[i], p);
            else *p = x[i];
        }
        if constexpr (FORMAT == KVCACHE_E4M3)
            if (lane == 0) at_global<uint8_t>(values[i] ? a.scale[1] : a.scale[0])[to[i]] = scale[i];
    }
}

int check(int64_t groups, int32_t tokens, int32_t heads, int32_t d, int64_t pages, int32_t page_size, int dtype, int format)
{
    if (dtype != ADDRMS_BF16 && dtype != ADDRMS_FP16) return fail(ADDRMS_ERR_UNSUPPORTED_DTYPE, "unsupported dtype %d for a cache", dtype);
    if (format != KVCACHE_SAME && format != KVCACHE_E4M3) return fail(ADDRMS_ERR_INVALID_ARG, "unknown cache format %d", format);
    if (groups < 0 || tokens < 0 || heads <= 0 || d <= 0 || pages < 0)
        return fail(ADDRMS_ERR_INVALID_ARG, "groups, tokens and pages must be >= 0, heads and d > 0");
    if (!power_of_two(page_size) || page_size > 65536) return fail(ADDRMS_ERR_INVALID_ARG, "page_size must be a power of two up to 65536 (got %d)", page_size);
    if (d % 16 != 0 || d > KVCACHE_MAX_HEAD)
        return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "d=%d is not a multiple of 16 up to %d", d, KVCACHE_MAX_HEAD);
    if (tokens > KVMOVE_MAX_TOKENS) return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "a group of %d tokens is beyond the limit (%d)", tokens, KVMOVE_MAX_TOKENS);
    if (heads > 65536 || pages >= (1ll << 31) || groups >= (1ll << 21) || groups * heads >= (1ll << 21))
        return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "%lld groups of %d heads or %lld pages are beyond the limits", (long long)groups, heads, (long long)pages);
    return ADDRMS_OK;
}

}  // namespace

extern "C" {

int kvmove_run(void* k_pages, void* v_pages, uint8_t* k_scale, uint8_t* v_scale, const int64_t* from_slots, const int64_t* to_slots, int64_t groups,
               int32_t tokens, int32_t heads, int32_t d, int64_t pages, int32_t page_size, int dtype, int format, void* stream)
{
    if (const int st = check(groups, tokens, heads, d, pages, page_size, dtype, format)) return st;
    if (groups == 0 || tokens == 0 || pages == 0) return ADDRMS_OK;
    if (!k_pages || !v_pages || !from_slots || !to_slots || (format == KVCACHE_E4M3 && (!k_scale || !v_scale)))
        return fail(ADDRMS_ERR_INVALID_ARG, "no pointer may be NULL");
    if (!aligned_to(k_pages, 16) || !aligned_to(v_pages, 16) || !aligned_to(from_slots, 8) || !aligned_to(to_slots, 8))
        return fail(ADDRMS_ERR_MISALIGNED, "pages must be aligned to 16 bytes and slots to 8");
    MoveArgs a = {};
    a.pages[0] = addr(k_pages), a.pages[1] = addr(v_pages), a.scale[0] = addr(k_scale), a.scale[1] = addr(v_scale);
    a.from = addr(from_slots), a.to = addr(to_slots);
    a.cache_slots = pages * page_size;
    a.tokens = static_cast<uint32_t>(tokens), a.heads = static_cast<uint32_t>(heads), a.page_shift = static_cast<uint32_t>(log2_of(page_size));
    a.pieces = static_cast<uint32_t>(format == KVCACHE_E4M3 ? d / 16 : d / 8), a.lanes_log2 = static_cast<uint32_t>(log2_of(a.pieces));
    a.per_token = 1.0f / static_cast<float>(tokens);
    const uint32_t unit = a.tokens << a.lanes_log2;                              // lanes' pieces of a unit, up to 256 * 32
    // Rows of a thread: as few as hold a unit, two where there is much to move.  Much, in whole lines, goes past the caches.
    const bool much = 2ll * groups * tokens * heads * a.pieces * 16 >= kPastBytes, past = much && a.pieces % 8 == 0;
    const int per = unit > 1024 ? 8 : unit > 512 ? 4 : unit > 256 || much ? 2 : 1;
    const uint32_t threads = unit > 1024 ? 1024 : 256;
    a.units = threads * per / unit < 2 * a.heads ? threads * per / unit : 2 * a.heads;
    a.spans = (2 * a.heads + a.units - 1) / a.units;
    const dim3 grid(static_cast<unsigned>(groups) * a.spans);
    const hipStream_t s = static_cast<hipStream_t>(stream);
#define AS(F, T, P) launch_kernel(past ? move_kernel<F, T, P, true> : move_kernel<F, T, P, false>, grid, dim3(threads), s, a)
#define GO(F) (per == 8 ? AS(F, 1024, 8) : per == 4 ? AS(F, 256, 4) : per == 2 ? AS(F, 256, 2) : AS(F, 256, 1))
    SERVING_HIP_TRY(format == KVCACHE_E4M3 ? GO(KVCACHE_E4M3) : GO(KVCACHE_SAME));
#undef AS
#undef GO
    return ADDRMS_OK;
}

int64_t kvmove_algorithmic_bytes(int64_t groups, int32_t tokens, int64_t moved, int32_t heads, int32_t d, int format)
{
    if (const int st = check(groups, tokens, heads, d, 1, 1, ADDRMS_BF16, format)) return st;
    if (moved < 0 || moved > groups * tokens) return fail(ADDRMS_ERR_INVALID_ARG, "moved must be from 0 to %lld", (long long)(groups * tokens));
    return 4 * moved * heads * (format == KVCACHE_E4M3 ? d + 1 : 2 * d) + 16 * groups * tokens;
}

}  // extern "C"
