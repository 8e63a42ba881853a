// Host side of attention over a shared prefix (include/prefixattn.h): argument checks, how the work is split, and the kernel
// that joins the splits' results.
#include "prefixattn.h"
#include "prefixattn_plan.h"

using namespace addrms_host;
using namespace serving;

namespace {

// out = sum_p 2^(m_p - m) O_p / sum_p 2^(m_p - m) l_p, lse = ln 2 (m + log2 of that sum), over the parts that were run: a suffix
// has as many as its length says.  WAVES waves join a row, lanes being columns of four elements by groups of parts; the first parts
// are under way while their weights are found.  One wave where there are rows enough to fill the chip (no barrier, four rows a
// workgroup), four where there are few rows, which then have many parts.
template <int DT, int WAVES>
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
        const int32_t keys = min(max(at_global<const int32_t>(a.suffix_lens)[row / (a.q_len * a.q_heads)], 0), a.suffix_width << a.page_shift);
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

// Checks a shape and splits its work.  A key range is split until there are as many workgroups as `wanted` says,
// in pieces of kMinChunk keys or more; what a suffix may hold at most counts, for its length is known on the device alone.
int plan_of(const prefixattn_shape* s, Plan* p)
{
    if (const int st = shape_of(s, p)) return st;
    if (p->rows == 0) return ADDRMS_OK;
    AttnArgs& a = p->a;
    const int64_t width = s->suffix_width * s->page_size, all = static_cast<int64_t>(s->batch) * s->q_len * a.group, own = static_cast<int64_t>(s->q_len) * a.group;
    p->suffix_form = form_of(own, p->dp);
    p->prefix_form = form_of(all, p->dp);
    // a cache without a page has no key (the kernels read row 0 in the place of one that is not there)
    // A CU holds one workgroup of eight waves and two of four.  (Of few rows three for some types, but 4 x 32 heads over 131072 keys take
    // 57.4 us with 512, 59.0 with 768, 67.2 with 384 in e4m3, 103.0, 104.0 and 100.5 in bf16, 2 x 32 over 32768 bf16 33.6, 33.9 and 35.6.)
    auto wanted = [p](int form) { return form == MANY_256 || (form == MANY_128 && p->dp > 128) ? 256 : 512; };
    // one workgroup a CU, or fewer: eight waves each (32 x 8 heads of e4m3 keys, 16 and then up to 1024: 15.0 us a call with four, 12.5
    // with eight; 64 x 8: 17.6 with four, 21.8 with eight)
    auto few = [](int64_t units) { return units <= kFinishUnits ? FEW_8 : FEW; };
    // A short prefix is seen by each suffix's workgroup, through the L2s, in one launch: as long as all of them read up to 128 MB of it;
    // with fewer workgroups than CUs, as long as one reads up to 192 KB with its suffix, or 384 from half the CUs on, for more of them
    // would then share the work.  32 query and 8 key heads of 128, a prefix and suffixes of 64, one launch and two, us:
    //   sequences   2 e4m3: 700 keys 9.2, 10.9; 1400 13.0, 10.7   2 bf16: 200 7.5, 9.2; 400 9.3, 9.5; 700 12.1, 9.8
    //              16 e4m3: 1400 13.6, 13.7                      16 bf16: 400 9.6, 12.6; 700 12.3, 12.5; 1400 19.4, 12.9
    //              64 e4m3: 700 14.7, 20.5; 1400 22.3, 22.3      64 bf16: 400 14.4, 20.1; 700 19.5, 20.8; 1400 31.7, 23.0
    // (a key counts for 256 bytes at least: less is not faster)
    const int64_t units = static_cast<int64_t>(a.kv_heads) * s->batch, key_bytes = std::max(256, 2 * p->dp * (s->format == KVCACHE_E4M3 ? 1 : 2));
    const int64_t prefix_bytes = a.prefix_len * key_bytes, chain = prefix_bytes + width * key_bytes;
    if (a.pages && a.prefix_len && p->suffix_form == FEW &&
        (units >= kFinishUnits ? units * prefix_bytes <= kInlineBytes : chain <= (units >= kFinishUnits / 2 ? 2 * kInlineChain : kInlineChain))) {
        p->prefix_form = p->suffix_form = few(units);
        p->finish = true;
        a.inline_len = a.prefix_len;
        a.suffix_tiles = a.suffix_splits = 1;
        a.suffix_chunk = static_cast<int32_t>(width);
        p->suffix_blocks = units;
        return fits(*p);
    }
    const bool prefix = a.prefix_len && a.pages, suffix = width && a.pages;
    if (!prefix) p->prefix_form = p->suffix_form;
    a.prefix_tiles = static_cast<int32_t>(tiles_of(all, p->prefix_form));
    a.suffix_tiles = static_cast<int32_t>(tiles_of(own, p->suffix_form));
    const int64_t prefix_units = static_cast<int64_t>(a.prefix_tiles) * a.kv_heads, suffix_units = static_cast<int64_t>(a.suffix_tiles) * a.kv_heads * s->batch;
    const int64_t slots = wanted(p->prefix_form);
    auto split_prefix = [&](int64_t n) { a.prefix_splits = prefix ? splits_of(a.prefix_len, prefix_units, n, kMinChunk, &a.prefix_chunk) : 0; };
    split_prefix(slots);
    p->finish = suffix && suffix_units >= kFinishUnits && a.prefix_splits <= kFinishSplits;
    if (p->finish && p->suffix_form == FEW) p->suffix_form = few(suffix_units);
    if (suffix) {
        a.suffix_splits = splits_of(width, suffix_units, p->finish ? 1 : wanted(p->suffix_form), std::clamp(a.prefix_chunk, kMinChunk, 2 * kMinChunk), &a.suffix_chunk);
        p->suffix_blocks = suffix_units * a.suffix_splits;
        // One launch for both: the prefix leaves the suffixes their places, up to half of all.  Where a workgroup's own pace is the bound
        // (not with few rows, where memory is), only if its pieces grow by no more keys than a suffix's piece has, and as many as its
        // start takes the time of (about kMinChunk), for it else runs behind them: 16 x 4 queries over 4001 fp16 keys of 256 and
        // suffixes of 300 take 43.9 us with them behind, 38.2 beside, of one page 37.8 and 37.0; 8 x 40 heads over 8191 e4m3 keys and one
        // page 19.9 behind, 15.9 beside; over 131072 and suffixes of 500 70.6 behind, 80.5 beside; 4 x 16 queries of 32 heads over 20000
        // bf16 keys and suffixes of 1000 53.0 behind, 54.7 beside; with few rows, 4 x 32 heads over 131072 bf16 keys and suffixes of 2000,
        // 103.0 behind, 101.8 beside.
        if (!p->finish && prefix) {
            const int32_t splits = a.prefix_splits, chunk = a.prefix_chunk;
            split_prefix(std::max(slots / 2, slots - p->suffix_blocks));
            if (p->prefix_form != FEW && a.prefix_chunk - chunk > std::min<int64_t>(width, a.suffix_chunk) + kMinChunk)
                a.prefix_splits = splits, a.prefix_chunk = chunk;
        }
    }
    p->prefix_blocks = (static_cast<int64_t>(a.prefix_splits) * a.kv_heads + 7) / 8 * 8 * a.prefix_tiles;
    const int64_t parts = a.prefix_splits + (p->finish ? 0 : a.suffix_splits);
    p->bytes = parts * p->rows * (4ll * a.d + 8);
    return fits(*p);
}

}  // namespace

extern "C" {

int64_t prefixattn_workspace_bytes(const prefixattn_shape* shape)
{
    Plan p;
    if (const int st = plan_of(shape, &p)) return st;
    return p.bytes;
}

int64_t prefixattn_algorithmic_bytes(const prefixattn_shape* shape, int64_t suffix_keys)
{
    Plan p;
    if (const int st = plan_of(shape, &p)) return st;
    if (suffix_keys < 0) return fail(ADDRMS_ERR_INVALID_ARG, "suffix_keys must be >= 0");
    const int64_t key = 2ll * shape->kv_heads * (shape->format == KVCACHE_E4M3 ? shape->d + 1 : 2 * shape->d);
    return (shape->prefix_len + suffix_keys) * key + p.rows * (4ll * shape->d + 4);
}

int prefixattn_run(const void* q, const int64_t* q_strides, const void* k_pages, const void* v_pages, const uint8_t* k_scale, const uint8_t* v_scale,
                   const int32_t* prefix_pages, const int32_t* suffix_pages, const int32_t* suffix_lens, void* out, float* lse, float scale,
                   const prefixattn_shape* shape, void* workspace, int64_t workspace_bytes, void* stream)
{
    Plan p;
    if (const int st = plan_of(shape, &p)) return st;
    if (const int st = arguments_of(q, q_strides, k_pages, v_pages, k_scale, v_scale, prefix_pages, suffix_pages, suffix_lens, out, lse, scale, shape, workspace,
                                    workspace_bytes, &p))
        return st;
    if (p.rows == 0) return ADDRMS_OK;
    AttnArgs& a = p.a;
    const bool codes = shape->format == KVCACHE_E4M3;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    static constexpr AttnLaunch kUnits[2][2][3] = {
        {{ATTN_UNIT(0, 0, 64), ATTN_UNIT(0, 0, 128), ATTN_UNIT(0, 0, 256)}, {ATTN_UNIT(0, 1, 64), ATTN_UNIT(0, 1, 128), ATTN_UNIT(0, 1, 256)}},
        {{ATTN_UNIT(1, 0, 64), ATTN_UNIT(1, 0, 128), ATTN_UNIT(1, 0, 256)}, {ATTN_UNIT(1, 1, 64), ATTN_UNIT(1, 1, 128), ATTN_UNIT(1, 1, 256)}}};
    const AttnLaunch unit = kUnits[shape->dtype == ADDRMS_FP16][codes][p.dp == 64 ? 0 : p.dp == 128 ? 1 : 2];
    a.prefix_blocks = static_cast<int32_t>(p.prefix_blocks);
    if (p.finish) {
        if (p.prefix_blocks) SERVING_HIP_TRY(unit(a, p.prefix_form, p.suffix_form, static_cast<unsigned>(p.prefix_blocks), s));
        a.finish = 1;
        a.prefix_blocks = 0;
        SERVING_HIP_TRY(unit(a, p.suffix_form, p.suffix_form, static_cast<unsigned>(p.suffix_blocks), s));
        return ADDRMS_OK;
    }
    if (p.prefix_blocks + p.suffix_blocks) SERVING_HIP_TRY(unit(a, p.prefix_form, p.suffix_form, static_cast<unsigned>(p.prefix_blocks + p.suffix_blocks), s));
    const bool many = p.rows >= kJoinRows;
    const unsigned groups = static_cast<unsigned>(many ? (p.rows + 3) / 4 : p.rows);
    SERVING_HIP_TRY(launch_kernel(shape->dtype == ADDRMS_FP16 ? (many ? join_kernel<DT_FP16, 1> : join_kernel<DT_FP16, 4>)
                                                              : (many ? join_kernel<DT_BF16, 1> : join_kernel<DT_BF16, 4>),
                                  dim3(groups), dim3(kJoinThreads), s, a));
    return ADDRMS_OK;
}

}  // extern "C"
