// Device side of attention of trees of drafted tokens (include/treeattn.h).
//
// A sequence's nodes are its rows, as in prefixattn_kernel.h, whose two forms of a workgroup are used here: the keys below the tree
// are seen by all rows, so that only a tile that holds nodes' keys (of the last two or three) looks at masks, a row's 64 bits
// shifted to the tile's first key and met with the keys that are there.
//
// Many rows are bound by matrix instructions and the softmax between them (64 x 64 nodes of 64 heads of 128 over up to 4096 bf16 keys, 248
// GFLOP, 321 us, 770 TFLOP/s), few rows by memory (40 sequences over up to 8000 e4m3 keys 71 us, 5.0 TB/s), small calls by their chain
// (8 nodes over 301 keys 9.4 us).
#pragma once
#include "prefixattn_kernel.h"
#include "treeattn_cut.h"

namespace serving {

template <int DT, int FORMAT, int DP, int FORM, int WAVES, bool TWO> struct tree_form;
template <int DT, int FORMAT, int DP, int WAVES, bool TWO> struct tree_form<DT, FORMAT, DP, FEW, WAVES, TWO> { typedef Few<DT, FORMAT, DP, WAVES, true> type; };
template <int DT, int FORMAT, int DP, int WAVES, bool TWO> struct tree_form<DT, FORMAT, DP, FEW_8, WAVES, TWO> { typedef Few<DT, FORMAT, DP, 8, true> type; };
template <int DT, int FORMAT, int DP, int WAVES, bool TWO> struct tree_form<DT, FORMAT, DP, MANY_64, WAVES, TWO> { typedef Many<DT, FORMAT, DP, 32, 4, 2, true, TWO> type; };
template <int DT, int FORMAT, int DP, int WAVES, bool TWO> struct tree_form<DT, FORMAT, DP, MANY_128, WAVES, TWO> { typedef Many<DT, FORMAT, DP, (DP > 128 ? 16 : 32), (DP > 128 ? 8 : 4), 1, true, TWO> type; };
template <int DT, int FORMAT, int DP, int WAVES, bool TWO> struct tree_form<DT, FORMAT, DP, MANY_256, WAVES, TWO> { typedef Many<DT, FORMAT, DP, 32, 8, 1, true, TWO> type; };

// Workgroups of the prefix first, then those of the sequences.  Workgroups go round the 8 XCDs; the row tiles of one head and
// key range stand 8 apart, so that they read it through the same L2 at the same time.
// TWO: the sequences' workgroups of many rows see the prefix first.  (Those of few rows may, in either case.)
template <int DT, int FORMAT, int DP, int PREFIX, int SUFFIX, bool TWO>
__global__ __launch_bounds__(threads_of(PREFIX, DP), 2) void tree_kernel(AttnArgs a)
{
    constexpr int WAVES = threads_of(PREFIX, DP) / 64;          // few rows use all of them, whatever the prefix's form
    typedef typename form<DT, FORMAT, DP, PREFIX, WAVES>::type P;
    typedef typename tree_form<DT, FORMAT, DP, SUFFIX, WAVES, TWO>::type S;
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
    const int32_t j = b >> 3, tile = j % a.suffix_tiles, unit = (j / a.suffix_tiles) * 8 + (b & 7), at = unit / a.kv_heads, room = a.suffix_width << a.page_shift;
    s.head = unit - at * a.kv_heads;
    int32_t seq = at, split = 0, piece = kAll;
    if (a.cut_parts) {
        const Piece p = piece_at(a, at);
        if (p.seq < 0) return;
        seq = p.seq, split = p.number, piece = p.keys;
    } else {
        if (at >= a.batch) return;
        if (a.sorted) seq = by_length(a, at);
    }
    seq = __builtin_amdgcn_readfirstlane(seq), split = __builtin_amdgcn_readfirstlane(split), piece = __builtin_amdgcn_readfirstlane(piece);
    s.token0 = seq * a.q_len;
    s.row0 = tile * S::ROWS;
    s.rows = min(S::ROWS, a.q_len * a.group - s.row0);
    s.part = a.prefix_splits * a.batch + at - seq;
    s.first = split * piece;
    s.table = a.suffix_pages + 4 * static_cast<int64_t>(seq) * a.suffix_width;
    const auto context = [&] { return min(max(at_global<const int32_t>(a.suffix_lens)[seq], 0), room); };
    constexpr bool MANY = SUFFIX != FEW && SUFFIX != FEW_8;
    const int32_t shared = !MANY ? a.inline_len : TWO ? (a.inline_len + 63) / 64 * 64 : 0;        // where the sequence's own keys begin
    if (shared) {
        s.table2 = s.table;
        s.table = a.prefix_pages;
        s.turn = shared;
    }
    if constexpr (!MANY) {
        // The first tile's pages are asked for together with the length, as if the row of pages were full: a page number is checked
        // before it is used, and what is beyond the length masked.
        s.end = shared + room;
        const int32_t page0 = s.first < s.end ? S::page_of(a, s, s.first + S::TILE * (threadIdx.x >> 6), threadIdx.x & 63) : 0;
        const int32_t before = room ? context() : 0, keys = min(before + a.q_len, room);
        s.end = shared ? shared + keys : min(piece < kAll ? s.first + piece : kAll, keys);
        s.last0 = shared + before - 1;
        S().template run<true>(a, s, page0, lds);
    } else {
        const int32_t before = room ? context() : 0, keys = min(before + a.q_len, room);
        s.end = shared ? shared + keys : min(piece < kAll ? s.first + piece : kAll, keys);
        s.last0 = shared + before - 1;
        S().template run<true>(a, s, lds);
    }
}

// As prefixattn.hip's: out = sum_p 2^(m_p - m) O_p / sum_p 2^(m_p - m) l_p, lse = ln 2 (m + log2 of that sum), over the prefix's parts and
// those of the row's sequence.  WAVES waves join a row, lanes being columns of four elements by groups of parts.  NARROW: a workgroup has
// kJoinColumns of a row's elements, so that more lanes share its parts.
template <int DT, int WAVES, bool NARROW>
__global__ __launch_bounds__(kJoinThreads) void tree_join_kernel(AttnArgs a)
{
    typedef typename elem<DT>::type T;
    typedef T T4 __attribute__((ext_vector_type(4)));
    constexpr int ROWS = kJoinThreads / 64 / WAVES, THREADS = 64 * WAVES, AHEAD = 4;
    __shared__ float weight[ROWS][2 * kMaxSplits], red[2][4];
    __shared__ f32x4 sums[kJoinThreads];
    const int32_t tid = static_cast<int32_t>(threadIdx.x) % THREADS, slot = static_cast<int32_t>(threadIdx.x) / THREADS, wave = tid >> 6;
    const int32_t each = a.q_len * a.q_heads, rows = a.batch * each;
    const int32_t pieces = NARROW ? (a.d + kJoinColumns - 1) / kJoinColumns : 1, block = static_cast<int32_t>(blockIdx.x) / pieces, piece = static_cast<int32_t>(blockIdx.x) - block * pieces;
    const int32_t row = __builtin_amdgcn_readfirstlane(block * ROWS + slot);
    if (row >= rows) return;                                    // with one wave a row: no barrier follows
    const auto meet = [] {
        if constexpr (WAVES > 1) __syncthreads();
        else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    };
    int32_t parts = a.prefix_splits;
    int64_t own = 0;                                            // the row's place in its sequence's first part
    if (a.cut_parts) {
        const int32_t seq = row / each;
        const Cut cut = cut_of(a, seq);
        parts += cut.pieces;
        own = (static_cast<int64_t>(a.prefix_splits) * a.batch + cut.before - seq) * each + row;
    }
    const auto place = [&](int32_t p) { return p < a.prefix_splits ? static_cast<int64_t>(p) * rows + row : own + static_cast<int64_t>(p - a.prefix_splits) * each; };
    const int32_t cols = NARROW ? kJoinColumns / 4 : a.d / 4, groups = THREADS / cols, grp = tid / cols, lane_col = tid - grp * cols;
    const int32_t col = NARROW ? min(lane_col + piece * cols, a.d / 4 - 1) : lane_col;            // lanes beyond the head do as the last one does
    const float* o = at_global<const float>(a.part_o) + 4 * col;
    const int32_t mine = grp < groups && grp < parts ? (parts - grp + groups - 1) / groups : 0;      // parts that this lane adds
    f32x4 first[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) first[i] = i < mine ? *reinterpret_cast<const f32x4*>(o + place(grp + i * groups) * a.d) : f32x4{0, 0, 0, 0};
    const float2* ml = at_global<const float2>(a.part_ml);
    float m = kNone;
    for (int32_t p = tid; p < parts; p += THREADS) m = fmaxf(m, ml[place(p)].x);
#pragma unroll
    for (int x = 32; x; x >>= 1) m = fmaxf(m, __shfl_xor(m, x));
    if constexpr (WAVES > 1) {
        if ((tid & 63) == 0) red[0][wave] = m;
        __syncthreads();
        m = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
    }
    float l = 0.0f;
    for (int32_t p = tid; p < parts; p += THREADS) {
        const float2 x = ml[place(p)];
        // a part that saw no key has m = -inf, l = 0 and O = 0 (l is NaN where its scores were)
        const float w = x.x == kNone ? 1.0f : __builtin_amdgcn_exp2f(x.x - m);
        weight[slot][p] = w;
        l += w * x.y;
    }
#pragma unroll
    for (int x = 32; x; x >>= 1) l += __shfl_xor(l, x);
    if constexpr (WAVES > 1) {
        if ((tid & 63) == 0) red[1][wave] = l;
    }
    meet();
    if constexpr (WAVES > 1) l = (red[1][0] + red[1][1]) + (red[1][2] + red[1][3]);
    f32x4 x = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (i < mine) x += weight[slot][grp + i * groups] * first[i];
    for (int32_t i = AHEAD; i < mine; i += AHEAD) {
        f32x4 next[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) next[j] = *reinterpret_cast<const f32x4*>(o + place(grp + min(i + j, mine - 1) * groups) * a.d);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (i + j < mine) x += weight[slot][grp + (i + j) * groups] * next[j];
    }
    sums[threadIdx.x] = x;
    meet();
    if (grp == 0) {
        for (int32_t g = 1; g < groups; ++g) x += sums[slot * THREADS + g * cols + lane_col];
        const float inverse = l == 0.0f ? 0.0f : 1.0f / l;              // no key was seen: zeros
        T4 y;
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = static_cast<T>(x[j] * inverse);
        *reinterpret_cast<T4*>(at_global<T>(a.out) + static_cast<int64_t>(row) * a.d + 4 * col) = y;
        if (a.lse && col == 0) at_global<float>(a.lse)[row] = lse_of(m, l);
    }
}

}  // namespace serving
