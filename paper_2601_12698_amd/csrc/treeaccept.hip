// The path through a tree of drafted tokens that agrees with the model (include/treeaccept.h).
//
// A wave has a sequence, a lane a node.  A step of the path compares all masks with that of the node it stands at and asks the
// wave's vote for the first child; the path grows by a bit of the mask a step, so that it ends.  Bound by the launch: 256 sequences of 64
// nodes 3.9 us a call, one of 8 the same.
#include "serving_internal.h"
#include "treeaccept.h"

using namespace addrms_host;
using namespace serving;

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

struct AcceptArgs {
    addr_t chosen, tokens, masks, suffix_pages, suffix_lens, path, count, next_token, from, to;
    int64_t suffix_width;
    uint32_t batch, nodes, depth, page_shift, pages;
};

__global__ __launch_bounds__(kThreads) void accept_kernel(AcceptArgs a)
{
    const uint32_t lane = threadIdx.x & 63, b = blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (b >= a.batch) return;
    const int64_t at = static_cast<int64_t>(b) * a.nodes + (lane < a.nodes ? lane : 0);
    const uint64_t mine = lane < a.nodes ? at_global<const uint64_t>(a.masks)[at] & (~0ull >> (64 - a.nodes)) : 0;
    const int32_t token = at_global<const int32_t>(a.tokens)[at], answer = at_global<const int32_t>(a.chosen)[at];
    const int32_t begin = a.suffix_lens ? max(at_global<const int32_t>(a.suffix_lens)[b], 0) : 0;
    const uint64_t bit = 1ull << lane;
    const auto of = [](uint32_t x, uint32_t l) { return static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(x), static_cast<int>(l))); };
    uint32_t here = 0, count = 0;
    int32_t on_path = -1, next = -1;                            // the path's node number `lane`
    uint64_t seen = static_cast<uint64_t>(of(static_cast<uint32_t>(mine >> 32), 0)) << 32 | of(static_cast<uint32_t>(mine), 0);
    if (seen & 1)
        for (;;) {
            if (lane == count) on_path = static_cast<int32_t>(here);
            ++count;
            next = static_cast<int32_t>(of(static_cast<uint32_t>(answer), here));
            if (count == a.depth) break;
            const uint64_t children = __ballot(lane < a.nodes && !(seen & bit) && mine == (seen | bit) && token == next);
            if (!children) break;
            here = static_cast<uint32_t>(__builtin_ctzll(children));
            seen |= 1ull << here;
        }
    const int64_t room = a.suffix_width << a.page_shift;
    const auto slot_at = [&](int64_t position) -> int64_t {
        if (position >= room) return -1;
        const int32_t page = at_global<const int32_t>(a.suffix_pages)[b * a.suffix_width + (position >> a.page_shift)];
        if (static_cast<uint32_t>(page) >= a.pages) return -1;
        return (static_cast<int64_t>(page) << a.page_shift) + (position & ((1ll << a.page_shift) - 1));
    };
    for (uint32_t k = lane; k < a.depth; k += 64) {
        const int64_t to = static_cast<int64_t>(b) * a.depth + k;
        const int32_t node = k < 64 ? on_path : -1;
        at_global<int32_t>(a.path)[to] = node;
        if (!a.from) continue;
        int64_t f = -1, t = -1;
        if (node >= 0 && node != static_cast<int32_t>(k)) {
            f = slot_at(static_cast<int64_t>(begin) + node);
            t = slot_at(static_cast<int64_t>(begin) + k);
            if (f < 0 || t < 0) f = t = -1;
        }
        at_global<int64_t>(a.from)[to] = f;
        at_global<int64_t>(a.to)[to] = t;
    }
    if (lane == 0) {
        at_global<int32_t>(a.count)[b] = static_cast<int32_t>(count);
        at_global<int32_t>(a.next_token)[b] = next;
    }
}

}  // namespace

extern "C" int treeaccept_run(const int32_t* chosen, const int32_t* tokens, const int64_t* masks, const int32_t* suffix_pages, const int32_t* suffix_lens,
                              int32_t* path, int32_t* count, int32_t* next_token, int64_t* from_slots, int64_t* to_slots, int64_t batch, int32_t nodes,
                              int32_t depth, int64_t suffix_width, int64_t pages, int32_t page_size, void* stream)
{
    if (batch < 0 || nodes <= 0 || depth <= 0 || suffix_width < 0 || pages < 0)
        return fail(ADDRMS_ERR_INVALID_ARG, "sizes must not be negative, nodes and depth must be > 0");
    if (!power_of_two(page_size) || page_size > 65536) return fail(ADDRMS_ERR_INVALID_ARG, "page_size must be a power of two up to 65536 (got %d)", page_size);
    if (nodes > TREE_MAX_NODES) return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "a tree of %d nodes is beyond the limit (%d)", nodes, TREE_MAX_NODES);
    if (depth > 65536 || batch >= (1 << 24) || pages >= (1ll << 31) || suffix_width >= (1ll << 30) / page_size)
        return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "batch, depth, pages or keys are beyond the limits (2^24, 65536, 2^31, 2^30)");
    if (batch == 0) return ADDRMS_OK;
    if ((from_slots == nullptr) != (to_slots == nullptr)) return fail(ADDRMS_ERR_INVALID_ARG, "from_slots and to_slots are given together");
    if (!chosen || !tokens || !masks || !path || !count || !next_token || (from_slots && ((suffix_width && !suffix_pages) || !suffix_lens)))
        return fail(ADDRMS_ERR_INVALID_ARG, "no pointer may be NULL");
    if (!aligned_to(chosen, 4) || !aligned_to(tokens, 4) || !aligned_to(masks, 8) || !aligned_to(suffix_pages, 4) || !aligned_to(suffix_lens, 4) ||
        !aligned_to(path, 4) || !aligned_to(count, 4) || !aligned_to(next_token, 4) || !aligned_to(from_slots, 8) || !aligned_to(to_slots, 8))
        return fail(ADDRMS_ERR_MISALIGNED, "arrays must be aligned to their elements");
    AcceptArgs a = {};
    a.chosen = addr(chosen), a.tokens = addr(tokens), a.masks = addr(masks), a.suffix_pages = addr(suffix_pages), a.suffix_lens = addr(suffix_lens);
    a.path = addr(path), a.count = addr(count), a.next_token = addr(next_token), a.from = addr(from_slots), a.to = addr(to_slots);
    a.suffix_width = suffix_width;
    a.batch = static_cast<uint32_t>(batch), a.nodes = static_cast<uint32_t>(nodes), a.depth = static_cast<uint32_t>(depth);
    a.page_shift = static_cast<uint32_t>(log2_of(page_size)), a.pages = static_cast<uint32_t>(pages);
    SERVING_HIP_TRY(launch_kernel(accept_kernel, dim3(static_cast<unsigned>((batch + kWaves - 1) / kWaves)), dim3(kThreads), static_cast<hipStream_t>(stream), a));
    return ADDRMS_OK;
}
