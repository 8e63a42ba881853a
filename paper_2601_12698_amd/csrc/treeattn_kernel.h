// Device side of attention of trees of drafted tokens (include/treeattn.h).
//
// A sequence's nodes are its rows, as in prefixattn_kernel.h, whose two forms of a workgroup are used here: the keys below the tree
// are seen by all rows, so that only a tile that holds nodes' keys (the last, or the last two) looks at masks, a row's 64 bits
// shifted to the tile's first key and met with the keys that are there.
#pragma once
#include "prefixattn_kernel.h"

namespace serving {

template <int DT, int FORMAT, int DP, int FORM, int WAVES> struct tree_form;
template <int DT, int FORMAT, int DP, int WAVES> struct tree_form<DT, FORMAT, DP, FEW, WAVES> { typedef Few<DT, FORMAT, DP, WAVES, true> type; };
template <int DT, int FORMAT, int DP, int WAVES> struct tree_form<DT, FORMAT, DP, FEW_8, WAVES> { typedef Few<DT, FORMAT, DP, 8, true> type; };
template <int DT, int FORMAT, int DP, int WAVES> struct tree_form<DT, FORMAT, DP, MANY_64, WAVES> { typedef Many<DT, FORMAT, DP, 32, 4, 2, true> type; };
template <int DT, int FORMAT, int DP, int WAVES> struct tree_form<DT, FORMAT, DP, MANY_128, WAVES> { typedef Many<DT, FORMAT, DP, (DP > 128 ? 16 : 32), (DP > 128 ? 8 : 4), 1, true> type; };
template <int DT, int FORMAT, int DP, int WAVES> struct tree_form<DT, FORMAT, DP, MANY_256, WAVES> { typedef Many<DT, FORMAT, DP, 32, 8, 1, true> type; };

// Workgroups of the prefix first, then those of the sequences.  Workgroups go round the 8 XCDs; the row tiles of one head and
// key range stand 8 apart, so that they read it through the same L2 at the same time.
template <int DT, int FORMAT, int DP, int PREFIX, int SUFFIX>
__global__ __launch_bounds__(threads_of(PREFIX, DP), (DP > 128 && PREFIX == FEW ? 1 : 2)) void tree_kernel(AttnArgs a)
{
    constexpr int WAVES = threads_of(PREFIX, DP) / 64;          // few rows use all of them, whatever the prefix's form
    typedef typename form<DT, FORMAT, DP, PREFIX, WAVES>::type P;
    typedef typename tree_form<DT, FORMAT, DP, SUFFIX, WAVES>::type S;
    __shared__ __attribute__((aligned(16))) char lds[P::LDS > S::SUFFIX_LDS ? P::LDS : S::SUFFIX_LDS];
    int32_t b = static_cast<int32_t>(blockIdx.x);
    Share s;
    s.table2 = 0;
    s.turn = kAll;
    if (b < a.prefix_blocks) {
        const int32_t j = b >> 3, tile = j % a.prefix_tiles, pair = (j / a.prefix_tiles) * 8 + (b & 7);
        if (pair >= a.prefix_splits * a.kv_heads) return;
        const int32_t split = pair / a.kv_heads;
        s.head = pair - split * a.kv_heads;
        s.table = a.prefix_pages;
        s.token0 = 0;
        s.row0 = tile * P::ROWS;
        s.rows = min(P::ROWS, a.batch * a.q_len * a.group - s.row0);
        s.first = split * a.prefix_chunk;
        s.end = min(s.first + a.prefix_chunk, a.prefix_len);
        s.part = split;
        s.last0 = kAll;
        if constexpr (PREFIX == FEW || PREFIX == FEW_8) P().template run<false>(a, s, P::page_of(a, s, s.first + P::TILE * (threadIdx.x >> 6), threadIdx.x & 63), lds);
        else P().template run<false>(a, s, lds);
        return;
    }
    if (threadIdx.x >= S::THREADS) return;                      // a form with more waves than the sequences' leaves the others idle
    b -= a.prefix_blocks;
    const int32_t j = b >> 3, tile = j % a.suffix_tiles, unit = (j / a.suffix_tiles) * 8 + (b & 7);
    const int32_t seq = unit / (a.suffix_splits * a.kv_heads);
    if (seq >= a.batch) return;
    const int32_t in_seq = unit - seq * a.suffix_splits * a.kv_heads, split = in_seq / a.kv_heads, room = a.suffix_width << a.page_shift;
    s.head = in_seq - split * a.kv_heads;
    s.token0 = seq * a.q_len;
    s.row0 = tile * S::ROWS;
    s.rows = min(S::ROWS, a.q_len * a.group - s.row0);
    s.part = a.prefix_splits + split;
    s.first = split * a.suffix_chunk;
    s.table = a.suffix_pages + 4 * static_cast<int64_t>(seq) * a.suffix_width;
    const auto context = [&] { return min(max(at_global<const int32_t>(a.suffix_lens)[seq], 0), room); };
    if constexpr (SUFFIX == FEW || SUFFIX == FEW_8) {
        if (a.inline_len) {
            s.table2 = s.table;
            s.table = a.prefix_pages;
            s.turn = a.inline_len;
        }
        // The first tile's pages are asked for together with the length, as if the row of pages were full: a page number is checked
        // before it is used, and what is beyond the length masked.
        s.end = a.inline_len + room;
        const int32_t page0 = s.first < s.end ? S::page_of(a, s, s.first + S::TILE * (threadIdx.x >> 6), threadIdx.x & 63) : 0;
        const int32_t before = room ? context() : 0, keys = min(before + a.q_len, room);
        s.end = a.inline_len ? a.inline_len + keys : min(s.first + a.suffix_chunk, keys);
        s.last0 = a.inline_len + before - 1;
        if (s.first >= s.end && !a.finish) return;              // the joining kernel knows the length, too
        S().template run<true>(a, s, page0, lds);
    } else {
        const int32_t before = context();
        s.end = min(s.first + a.suffix_chunk, min(before + a.q_len, room));
        s.last0 = before - 1;
        if (s.first >= s.end && !a.finish) return;
        S().template run<true>(a, s, lds);
    }
}

}  // namespace serving
