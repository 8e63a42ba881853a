// The kernel that joins the parts of attention over splits of the keys.
#pragma once
#include "prefixattn_plan.h"

namespace serving {

// out = sum_p 2^(m_p - m) O_p / sum_p 2^(m_p - m) l_p, lse = ln 2 (m + log2 of that sum), over the parts that were run: a suffix
// has as many as its length says (TREE: with its nodes).  WAVES waves join a row, lanes being columns of four elements by groups of parts; the first parts
// are under way while their weights are found.  One wave where there are rows enough to fill the chip (no barrier, four rows a
// workgroup), four where there are few rows, which then have many parts.
template <int DT, int WAVES, bool TREE = false>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(AttnArgs a)
{
    typedef typename elem<DT>::type T;
    typedef T T4 __attribute__((ext_vector_type(4)));
    constexpr int ROWS = kJoinThreads / 64 / WAVES, THREADS = 64 * WAVES, AHEAD = 4;
    __shared__ float weight[ROWS][2 * kMaxSplits], red[2][4];
    __shared__ f32x4 sums[kJoinThreads];
    const int32_t tid = static_cast<int32_t>(threadIdx.x) % THREADS, slot = static_cast<int32_t>(threadIdx.x) / THREADS, wave = tid >> 6;
    const int64_t rows = static_cast<int64_t>(a.batch) * a.q_len * a.q_heads;
    const int32_t row = static_cast<int32_t>(blockIdx.x) * ROWS + slot;
    if (row >= rows) return;                                    // with one wave a row: no barrier follows
    const auto meet = [] {
        if constexpr (WAVES > 1) __syncthreads();
        else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    };
    int32_t parts = a.prefix_splits;
    if (a.suffix_splits) {
        const int32_t room = a.suffix_width << a.page_shift;
        int32_t keys = min(max(at_global<const int32_t>(a.suffix_lens)[row / (a.q_len * a.q_heads)], 0), room);
        if constexpr (TREE) keys = min(keys + a.q_len, room);
        parts += (keys + a.suffix_chunk - 1) / a.suffix_chunk;
    }
    const int32_t cols = a.d / 4, groups = THREADS / cols, grp = tid / cols, col = tid - grp * cols;
    const int64_t step = static_cast<int64_t>(groups) * rows * a.d;
    const float* o = at_global<const float>(a.part_o) + (grp * rows + row) * a.d + 4 * col;
    const int32_t mine = grp < groups && grp < parts ? (parts - grp + groups - 1) / groups : 0;      // parts that this lane adds
    f32x4 first[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) first[i] = i < mine ? *reinterpret_cast<const f32x4*>(o + i * step) : f32x4{0, 0, 0, 0};
    const float2* ml = at_global<const float2>(a.part_ml);
    float m = -__builtin_huge_valf();
    for (int32_t p = tid; p < parts; p += THREADS) m = fmaxf(m, ml[p * rows + row].x);
#pragma unroll
    for (int x = 32; x; x >>= 1) m = fmaxf(m, __shfl_xor(m, x));
    if constexpr (WAVES > 1) {
        if ((tid & 63) == 0) red[0][wave] = m;
        __syncthreads();
        m = fmaxf(fmaxf(red[0][0], red[0][1]), fmaxf(red[0][2], red[0][3]));
    }
    float l = 0.0f;
    for (int32_t p = tid; p < parts; p += THREADS) {
        const float2 x = ml[p * rows + row];
        // a part that saw no key has m = -inf, l = 0 and O = 0 (l is NaN where its scores were)
        const float w = x.x == -__builtin_huge_valf() ? 1.0f : __builtin_amdgcn_exp2f(x.x - m);
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
        for (int j = 0; j < AHEAD; ++j) next[j] = *reinterpret_cast<const f32x4*>(o + min(i + j, mine - 1) * step);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (i + j < mine) x += weight[slot][grp + (i + j) * groups] * next[j];
    }
    sums[threadIdx.x] = x;
    meet();
    if (grp == 0) {
        for (int32_t g = 1; g < groups; ++g) x += sums[slot * THREADS + g * cols + col];
        const float inverse = l == 0.0f ? 0.0f : 1.0f / l;              // no key was seen: zeros
        T4 y;
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = static_cast<T>(x[j] * inverse);
        *reinterpret_cast<T4*>(at_global<T>(a.out) + static_cast<int64_t>(row) * a.d + 4 * col) = y;
        if (a.lse && col == 0) at_global<float>(a.lse)[row] = (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
    }
}

template <bool TREE>
hipError_t launch_join(const Plan& p, int dtype, hipStream_t s)
{
    const bool many = p.rows >= kJoinRows;
    const unsigned groups = static_cast<unsigned>(many ? (p.rows + 3) / 4 : p.rows);
    return launch_kernel(dtype == ADDRMS_FP16 ? (many ? join_kernel<DT_FP16, 1, TREE> : join_kernel<DT_FP16, 4, TREE>)
                                              : (many ? join_kernel<DT_BF16, 1, TREE> : join_kernel<DT_BF16, 4, TREE>),
                         dim3(groups), dim3(kJoinThreads), s, p.a);
}

}  // namespace serving
