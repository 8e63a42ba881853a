// Device side of attention over a shared prefix (include/prefixattn.h).
//
// Rows are queries of one key and value head: of a token, `group` query heads.  A workgroup takes a tile of rows and a range
// of keys, goes over the keys once with a running maximum m and sum l of weights,
//     S = K Q^T;  m' = max(m, S);  P = 2^(c S - c m');  O = O 2^(c m - c m') + V^T P;  l = l 2^(c m - c m') + sum P
// and leaves O, c m and l (fp32) for the joining kernel.  Both products are matrix instructions, and both are formed
// transposed (keys by rows, then head elements by rows), because then
//   * a lane's scores belong to one row: maxima and sums are the lane's own, up to one exchange between lane groups;
//   * the scores lie in a lane as the second product wants its right operand, up to the order of keys, which a sum over keys
//     does not see: the values are fetched in that order, and no weight crosses a lane;
//   * values come out of LDS through the transposing read, four keys of one element a lane.
// O is scaled down only when a maximum grows by more than 2^8 (weights stay below that, and l and O are relative to the same
// number): most tiles leave 16 to 128 multiplications a lane out.
//
// Two forms.  FEW (up to 16 rows): every wave has all rows and takes every fourth tile of 32 keys by itself, keys straight from
// memory into registers, values through LDS of its own, no barrier until the waves' results are joined.  MANY: each of four waves
// has 32 rows, the tile of 64 keys and values is staged in LDS for all of them, two tiles deep.
#pragma once
#include "kvcache.h"
#include "prefixattn_args.h"
#include "serving_internal.h"

namespace serving {

template <int DT> struct mat;
template <> struct mat<DT_BF16> {
    typedef __bf16 T;
    typedef T T8 __attribute__((ext_vector_type(8)));
    typedef T T2 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ auto mul16(T8 a, T8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    template <typename C> static __device__ __forceinline__ C mul32(T8 a, T8 b, C c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    template <bool HI> static __device__ __forceinline__ T2 of_codes(uint32_t w, float s) { return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, HI); }
};
template <> struct mat<DT_FP16> {
    typedef _Float16 T;
    typedef T T8 __attribute__((ext_vector_type(8)));
    typedef T T2 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ auto mul16(T8 a, T8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    template <typename C> static __device__ __forceinline__ C mul32(T8 a, T8 b, C c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    template <bool HI> static __device__ __forceinline__ T2 of_codes(uint32_t w, float s) { return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, s, HI); }
};
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr float kLazy = 8.0f;                                   // a maximum may lag behind by this power of 2
// fp16 weights are 2^7 times larger (at most 2^15), so that they are normal numbers down to 2^-21 of the largest.
template <int DT> constexpr float kLift = DT == DT_FP16 ? 7.0f : 0.0f;
constexpr float kNone = -__builtin_huge_valf();

__device__ __forceinline__ float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

// Eight codes as elements, times their row's power of two.
template <int DT>
__device__ __forceinline__ typename mat<DT>::T8 elements_of(uint32_t lo, uint32_t hi, float s)
{
    const auto a = mat<DT>::template of_codes<false>(lo, s), b = mat<DT>::template of_codes<true>(lo, s);
    const auto c = mat<DT>::template of_codes<false>(hi, s), d = mat<DT>::template of_codes<true>(hi, s);
    return typename mat<DT>::T8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A transposing read: 16 lanes give the places of 4 rows of 16 elements, 8 bytes each; lane i gets element i of the four rows.
template <int DT>
__device__ __forceinline__ typename mat<DT>::T8 two_transposed(const char* lds_a, const char* lds_b)
{
    typedef __attribute__((address_space(3))) s16x4* P;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(lds_a)), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(lds_b));
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(typename mat<DT>::T8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

__device__ __forceinline__ float other_half_max(float x) { const pair p = with_half(x); return fmaxf(p.a, p.b); }
__device__ __forceinline__ float other_half_sum(float x) { const pair p = with_half(x); return p.a + p.b; }
__device__ __forceinline__ float other_row_max(float x) { const pair p = with_row(x); return fmaxf(p.a, p.b); }
__device__ __forceinline__ float other_row_sum(float x) { const pair p = with_row(x); return p.a + p.b; }

// A workgroup's share: rows [row0, row0 + rows) of a key head, rows counted token by token from token `token0`, keys
// [first, end) of a table of pages.  Query i of its sequence sees keys up to last0 + i.
struct Share {
    const int32_t* table;
    int32_t head, token0, row0, rows, first, end, part, last0;
};
constexpr int32_t kAll = 1 << 30;

struct Row {
    bool in;
    int32_t global;                                             // token * q_heads + head
    int32_t last;                                               // the last key that it sees
    int64_t q;                                                  // offset of its elements
};
__device__ __forceinline__ Row row_of(const AttnArgs& a, const Share& s, int32_t r)
{
    Row row;
    row.in = r < s.rows;
    const int32_t at = s.row0 + (row.in ? r : 0);
    const int32_t i = at / a.group, head = s.head * a.group + (at - i * a.group), token = s.token0 + i;
    row.global = token * a.q_heads + head;
    row.last = s.last0 + (s.last0 >= kAll ? 0 : i);
    row.q = token * a.q_token + head * a.q_head;
    return row;
}

// The cache row of a key: -1 where its page is outside the cache.
__device__ __forceinline__ int64_t cache_row(const AttnArgs& a, int32_t head, int32_t page, int32_t key)
{
    const int64_t row = ((static_cast<int64_t>(page) * a.kv_heads + head) << a.page_shift) + (key & ((1 << a.page_shift) - 1));
    return static_cast<uint32_t>(page) < static_cast<uint32_t>(a.pages) ? row : -1;
}

template <int DT, int FORMAT, int DP>
struct Few {
    typedef mat<DT> M;
    typedef typename M::T T;
    typedef typename M::T8 T8;
    static constexpr bool CODES = FORMAT == KVCACHE_E4M3;
    static constexpr int ES = CODES ? 1 : 2;
    static constexpr int TILE = 32;                             // keys of a wave at a time
    static constexpr int NC = DP / 32;                          // steps of 32 elements in S
    static constexpr int NK = CODES ? NC / 2 : NC;              // 16-byte loads of a lane for 16 keys
    static constexpr int NT = DP / 16;                          // tiles of 16 elements in O
    static constexpr int PIECES = DP * ES / 16;                 // 16-byte pieces of a key's values
    static constexpr int NV = TILE * PIECES / 64;
    static constexpr int VROW = DP * 2 + 32;                    // bytes from key to key in LDS: 4 keys' 32 bytes fall on 4 groups of banks
    static constexpr int WAVE_LDS = TILE * VROW;
    static constexpr int OROW = DP + 4;                         // floats from row to row where waves are joined
    static constexpr int LDS = 4 * WAVE_LDS > 4 * kFewRows * OROW * 4 ? 4 * WAVE_LDS : 4 * kFewRows * OROW * 4;

    u32x4 k[2][NK], v[NV];
    uint32_t scales;                                            // of key lane % 32: the key's byte, and the value's above it
    uint32_t valid;                                             // keys of the tile that are there

    __device__ __forceinline__ void load(const AttnArgs& a, const Share& s, int32_t key0, int32_t page, int lane)
    {
        const int32_t mine = key0 + (lane & 31);
        const int64_t row = mine < s.end ? cache_row(a, s.head, page, mine) : -1;
        valid = static_cast<uint32_t>(__ballot(row >= 0));
        scales = 0;
        if constexpr (CODES) {
            if (row >= 0) scales = at_global<const uint8_t>(a.k_scale)[row] | (at_global<const uint8_t>(a.v_scale)[row] << 8);
        }
        const char* kp = at_global<const char>(a.k_pages);
        const char* vp = at_global<const char>(a.v_pages);
        const int32_t row_bytes = a.d * ES;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int at = 16 * t + (lane & 15);
            const int64_t r = cache_row(a, s.head, __shfl(page, at), key0 + at);
            const bool in = (valid >> at) & 1;
#pragma unroll
            for (int c = 0; c < NK; ++c) {
                const int32_t b = 64 * c + 16 * (lane >> 4);    // 16 bytes: 8 elements, or 16 codes
                k[t][c] = u32x4{0, 0, 0, 0};
                if (in && b < row_bytes) k[t][c] = *reinterpret_cast<const u32x4*>(kp + r * row_bytes + b);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = (64 / PIECES) * i + lane / PIECES;
            const int32_t b = 16 * (lane % PIECES);
            const int64_t r = cache_row(a, s.head, __shfl(page, at), key0 + at);
            v[i] = u32x4{0, 0, 0, 0};
            if (((valid >> at) & 1) && b < row_bytes) v[i] = *reinterpret_cast<const u32x4*>(vp + r * row_bytes + b);
        }
    }

    static __device__ __forceinline__ int32_t page_of(const AttnArgs& a, const Share& s, int32_t key0, int lane)
    {
        const int32_t key = key0 + (lane & 31);
        return key < s.end ? s.table[key >> a.page_shift] : -1;
    }

    __device__ __forceinline__ void run(const AttnArgs& a, const Share& s, char* lds)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4;
        const Row row = row_of(a, s, lane & 15);
        T8 q[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int32_t e = CODES ? 64 * (c >> 1) + 16 * g + 8 * (c & 1) : 32 * c + 8 * g;
            const T* p = at_global<const T>(a.q) + row.q + e;
#pragma unroll
            for (int j = 0; j < 8; ++j) q[c][j] = row.in && e < a.d ? p[j] : static_cast<T>(0.0f);
        }
        f32x4 o[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) o[t] = f32x4{0, 0, 0, 0};
        float m = kNone, l = 0.0f;
        const float lag = kLazy / a.c;
        char* mine = lds + wave * WAVE_LDS;
        // where this lane's 8 bytes of a transposing read begin: key 4 g + (lane % 16) / 4 of 16, elements 4 (lane % 4) of 16
        const char* from = mine + (4 * g + ((lane & 15) >> 2)) * VROW + 8 * (lane & 3);

        int32_t key0 = s.first + TILE * wave;
        if (key0 < s.end) load(a, s, key0, page_of(a, s, key0, lane), lane);
        int32_t page = key0 + 4 * TILE < s.end ? page_of(a, s, key0 + 4 * TILE, lane) : -1;
        while (key0 < s.end) {
            // values to LDS, as elements
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int at = (64 / PIECES) * i + lane / PIECES, b = lane % PIECES;
                if constexpr (CODES) {
                    const float sc = scale_of((__shfl(scales, at) >> 8) & 255);
                    T8* to = reinterpret_cast<T8*>(mine + at * VROW + 32 * b);
                    to[0] = elements_of<DT>(v[i][0], v[i][1], sc);
                    to[1] = elements_of<DT>(v[i][2], v[i][3], sc);
                } else {
                    *reinterpret_cast<u32x4*>(mine + at * VROW + 16 * b) = v[i];
                }
            }
            // S^T: 32 keys by 16 rows; this lane has keys 16 t + 4 g + r of row lane % 16
            f32x4 z[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                z[t] = f32x4{0, 0, 0, 0};
                if constexpr (CODES) {
                    const float sc = scale_of(__shfl(scales, 16 * t + (lane & 15)) & 255);
#pragma unroll
                    for (int c = 0; c < NK; ++c) {
                        z[t] = M::mul16(elements_of<DT>(k[t][c][0], k[t][c][1], sc), q[2 * c], z[t]);
                        z[t] = M::mul16(elements_of<DT>(k[t][c][2], k[t][c][3], sc), q[2 * c + 1], z[t]);
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < NK; ++c) z[t] = M::mul16(__builtin_bit_cast(T8, k[t][c]), q[c], z[t]);
                }
            }
            const uint32_t there = valid;
            const int32_t now = key0;
            key0 += 4 * TILE;
            if (key0 < s.end) {
                load(a, s, key0, page, lane);
                page = key0 + 4 * TILE < s.end ? page_of(a, s, key0 + 4 * TILE, lane) : -1;
            }
            if (there != 0xffffffffu || now + TILE - 1 > s.last0) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int at = 16 * t + 4 * g + r;
                        if (!((there >> at) & 1) || now + at > row.last) z[t][r] = kNone;
                    }
            }
            float top = fmaxf(fmaxf(fmaxf(z[0][0], z[0][1]), fmaxf(z[0][2], z[0][3])), fmaxf(fmaxf(z[1][0], z[1][1]), fmaxf(z[1][2], z[1][3])));
            top = other_half_max(other_row_max(top));
            if (__any(top > m + lag)) {
                const float next = fmaxf(m, top);
                const float down = m == kNone ? 0.0f : __builtin_amdgcn_exp2f((m - next) * a.c);
                l *= down;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[t][r] *= down;
                m = next;
            }
            const float base = m == kNone ? 0.0f : m * a.c - kLift<DT>;
            T8 p;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(z[j >> 2][j & 3], a.c, -base));
                l += w;
                p[j] = static_cast<T>(w);
            }
            // the wave's own LDS, written by other lanes of it above
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int t = 0; t < NT; ++t) o[t] = M::mul16(two_transposed<DT>(from + 32 * t, from + 32 * t + 16 * VROW), p, o[t]);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }

        // the four waves' results, joined
        l = other_half_sum(other_row_sum(l));
        __shared__ float2 ml[4][kFewRows];
        if (lane < 16) ml[wave][lane] = make_float2(m, l);
        __syncthreads();
        float best = kNone, sum = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) best = fmaxf(best, ml[w][lane & 15].x);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float2 x = ml[w][lane & 15];
            if (x.x != kNone || x.y != x.y) sum += x.y * (x.x == kNone ? 1.0f : __builtin_amdgcn_exp2f((x.x - best) * a.c));
        }
        const float down = m == kNone ? 1.0f : __builtin_amdgcn_exp2f((m - best) * a.c);
        float* join = reinterpret_cast<float*>(lds);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            f32x4 x = o[t];
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] *= down;
            *reinterpret_cast<f32x4*>(join + (wave * kFewRows + (lane & 15)) * OROW + 16 * t + 4 * g) = x;
        }
        const int64_t rows = static_cast<int64_t>(a.batch) * a.q_len * a.q_heads;
        if (wave == 0 && lane < 16 && row.in)
            at_global<float2>(a.part_ml)[s.part * rows + row.global] = make_float2(best == kNone ? kNone : best * a.c - kLift<DT>, sum);
        __syncthreads();
        for (int i = threadIdx.x; i < kFewRows * DP / 4; i += kAttnThreads) {
            const int r = i / (DP / 4), e = 4 * (i % (DP / 4));
            if (r >= s.rows || e >= a.d) continue;
            f32x4 x = *reinterpret_cast<const f32x4*>(join + r * OROW + e);
#pragma unroll
            for (int w = 1; w < 4; ++w) x += *reinterpret_cast<const f32x4*>(join + (w * kFewRows + r) * OROW + e);
            *reinterpret_cast<f32x4*>(at_global<float>(a.part_o) + (s.part * rows + row_of(a, s, r).global) * a.d + e) = x;
        }
    }
};

template <int DT, int FORMAT, int DP>
struct Many {
    typedef mat<DT> M;
    typedef typename M::T T;
    typedef typename M::T8 T8;
    static constexpr bool CODES = FORMAT == KVCACHE_E4M3;
    static constexpr int ES = CODES ? 1 : 2;
    static constexpr int TILE = 64;
    static constexpr int NC = DP / 16;                          // steps of 16 elements in S
    static constexpr int NT = DP / 32;                          // tiles of 32 elements in O
    static constexpr int PIECES = DP * ES / 16;
    static constexpr int NP = TILE * PIECES / kAttnThreads;     // pieces of keys, and of values, that a thread stages
    static constexpr int KROW = DP * 2 + 16, VROW = DP * 2 + 32;   // bytes from key to key: 8 keys' 16, or 4 keys' 32, fall on all banks
    static constexpr int BUF = TILE * (KROW + VROW) + TILE;     // keys, values, a byte for each key that is there
    static constexpr int LDS = 2 * BUF;

    u32x4 k[NP], v[NP];
    uint32_t scales[NP];                                        // the key's byte, the value's above it, and 2^16 if the key is there

    static __device__ __forceinline__ int key_of(int i) { return (kAttnThreads / PIECES) * i + static_cast<int>(threadIdx.x) / PIECES; }
    static __device__ __forceinline__ int piece() { return static_cast<int>(threadIdx.x) % PIECES; }

    __device__ __forceinline__ void pages_of(const AttnArgs& a, const Share& s, int32_t key0, int32_t (&page)[NP]) const
    {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int32_t key = key0 + key_of(i);
            page[i] = key < s.end ? s.table[key >> a.page_shift] : -1;
        }
    }
    __device__ __forceinline__ void load(const AttnArgs& a, const Share& s, int32_t key0, const int32_t (&page)[NP])
    {
        const char* kp = at_global<const char>(a.k_pages);
        const char* vp = at_global<const char>(a.v_pages);
        const int32_t row_bytes = a.d * ES, b = 16 * piece();
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int64_t row = cache_row(a, s.head, page[i], key0 + key_of(i));
            k[i] = v[i] = u32x4{0, 0, 0, 0};
            scales[i] = 0;
            if (row >= 0) {
                if (b < row_bytes) {
                    k[i] = *reinterpret_cast<const u32x4*>(kp + row * row_bytes + b);
                    v[i] = *reinterpret_cast<const u32x4*>(vp + row * row_bytes + b);
                }
                scales[i] = 1u << 16;
                if constexpr (CODES) scales[i] |= at_global<const uint8_t>(a.k_scale)[row] | (at_global<const uint8_t>(a.v_scale)[row] << 8);
            }
        }
    }
    __device__ __forceinline__ void stage(char* buf) const
    {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            char* kt = buf + key_of(i) * KROW + (CODES ? 32 : 16) * piece();
            char* vt = buf + TILE * KROW + key_of(i) * VROW + (CODES ? 32 : 16) * piece();
            if constexpr (CODES) {
                const float ks = scale_of(scales[i] & 255), vs = scale_of((scales[i] >> 8) & 255);
                reinterpret_cast<T8*>(kt)[0] = elements_of<DT>(k[i][0], k[i][1], ks);
                reinterpret_cast<T8*>(kt)[1] = elements_of<DT>(k[i][2], k[i][3], ks);
                reinterpret_cast<T8*>(vt)[0] = elements_of<DT>(v[i][0], v[i][1], vs);
                reinterpret_cast<T8*>(vt)[1] = elements_of<DT>(v[i][2], v[i][3], vs);
            } else {
                *reinterpret_cast<u32x4*>(kt) = k[i];
                *reinterpret_cast<u32x4*>(vt) = v[i];
            }
            if (piece() == 0) buf[TILE * (KROW + VROW) + key_of(i)] = static_cast<char>(scales[i] >> 16);
        }
    }

    __device__ __forceinline__ void run(const AttnArgs& a, const Share& s, char* lds)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
        const Row row = row_of(a, s, 32 * wave + (lane & 31));
        const bool busy = 32 * wave < s.rows;                   // waves without rows only help to stage
        T8 q[NC];
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int32_t e = 16 * c + 8 * h;
            const T* p = at_global<const T>(a.q) + row.q + e;
#pragma unroll
            for (int j = 0; j < 8; ++j) q[c][j] = row.in && e < a.d ? p[j] : static_cast<T>(0.0f);
        }
        f32x16 o[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) o[t] = f32x16{};
        float m = kNone, l = 0.0f;
        const float lag = kLazy / a.c;

        int32_t page[NP];
        int32_t key0 = s.first;
        pages_of(a, s, key0, page);
        load(a, s, key0, page);
        pages_of(a, s, key0 + TILE, page);
        stage(lds);
        __syncthreads();
        for (int cur = 0; key0 < s.end; key0 += TILE, cur ^= 1) {
            const bool more = key0 + TILE < s.end;
            if (more) {
                load(a, s, key0 + TILE, page);
                pages_of(a, s, key0 + 2 * TILE, page);
            }
            const char* buf = lds + cur * BUF;
            if (busy) {
                const char* kt = buf + (lane & 31) * KROW + 16 * h;
                f32x16 z[2];
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    z[t] = f32x16{};
#pragma unroll
                    for (int c = 0; c < NC; ++c) z[t] = M::mul32(*reinterpret_cast<const T8*>(kt + 32 * t * KROW + 32 * c), q[c], z[t]);
                }
                const uint64_t there = __ballot(buf[TILE * (KROW + VROW) + lane] != 0);
                if (there != ~0ull || key0 + TILE - 1 > s.last0) {
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int at = 32 * t + 8 * (i >> 2) + 4 * h + (i & 3);
                            if (!((there >> at) & 1) || key0 + at > row.last) z[t][i] = kNone;
                        }
                }
                float top = z[0][0];
#pragma unroll
                for (int i = 1; i < 32; ++i) top = fmaxf(top, z[i >> 4][i & 15]);
                top = other_half_max(top);
                if (__any(top > m + lag)) {
                    const float next = fmaxf(m, top);
                    const float down = m == kNone ? 0.0f : __builtin_amdgcn_exp2f((m - next) * a.c);
                    l *= down;
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[t][i] *= down;
                    m = next;
                }
                const float base = m == kNone ? 0.0f : m * a.c - kLift<DT>;
                // where this lane's 8 bytes of a transposing read begin: key 4 h + (lane % 16) / 4, elements 16 ((lane / 16) % 2) + 4 (lane % 4)
                const char* vt = buf + TILE * KROW + (4 * h + ((lane & 15) >> 2)) * VROW + 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
#pragma unroll
                for (int u = 0; u < TILE / 16; ++u) {
                    T8 p;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(z[u >> 1][8 * (u & 1) + j], a.c, -base));
                        l += w;
                        p[j] = static_cast<T>(w);
                    }
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const char* at = vt + 16 * u * VROW + 64 * t;
                        o[t] = M::mul32(two_transposed<DT>(at, at + 8 * VROW), p, o[t]);
                    }
                }
            }
            if (more) stage(lds + (cur ^ 1) * BUF);
            __syncthreads();
        }
        if (!busy) return;
        l = other_half_sum(l);
        if (!row.in) return;
        const int64_t rows = static_cast<int64_t>(a.batch) * a.q_len * a.q_heads, at = s.part * rows + row.global;
        if (h == 0) at_global<float2>(a.part_ml)[at] = make_float2(m == kNone ? kNone : m * a.c - kLift<DT>, l);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int32_t e = 32 * t + 8 * i + 4 * h;
                if (e < a.d)
                    *reinterpret_cast<f32x4*>(at_global<float>(a.part_o) + at * a.d + e) = f32x4{o[t][4 * i], o[t][4 * i + 1], o[t][4 * i + 2], o[t][4 * i + 3]};
            }
    }
};

// Workgroups of the prefix first, then those of the suffixes.  Workgroups go round the 8 XCDs; the row tiles of one head and
// key range stand 8 apart, so that they read it through the same L2 at the same time.
template <int DT, int FORMAT, int DP, int PREFIX, int SUFFIX>
__global__ __launch_bounds__(kAttnThreads, DP > 128 ? 1 : 2) void attn_kernel(const AttnArgs a)
{
    typedef Few<DT, FORMAT, DP> F;
    typedef Many<DT, FORMAT, DP> N;
    constexpr int LDS = PREFIX == MANY || SUFFIX == MANY ? (N::LDS > F::LDS || SUFFIX == MANY ? N::LDS : F::LDS) : F::LDS;
    __shared__ __attribute__((aligned(16))) char lds[LDS];
    int32_t b = static_cast<int32_t>(blockIdx.x);
    Share s;
    if (b < a.prefix_blocks) {
        const int32_t j = b >> 3, tile = j % a.prefix_tiles, pair = (j / a.prefix_tiles) * 8 + (b & 7);
        if (pair >= a.prefix_splits * a.kv_heads) return;
        const int32_t split = pair / a.kv_heads;
        constexpr int ROWS = PREFIX == MANY ? kManyRows : kFewRows;
        s.head = pair - split * a.kv_heads;
        s.table = at_global<const int32_t>(a.prefix_pages);
        s.token0 = 0;
        s.row0 = tile * ROWS;
        s.rows = min(ROWS, a.batch * a.q_len * a.group - s.row0);
        s.first = split * a.prefix_chunk;
        s.end = min(s.first + a.prefix_chunk, a.prefix_len);
        s.part = split;
        s.last0 = kAll;
        if constexpr (PREFIX == MANY) N().run(a, s, lds);
        else F().run(a, s, lds);
        return;
    }
    b -= a.prefix_blocks;
    const int32_t seq = b / (a.suffix_tiles * a.suffix_splits * a.kv_heads);
    b -= seq * a.suffix_tiles * a.suffix_splits * a.kv_heads;
    const int32_t split = b / (a.suffix_tiles * a.kv_heads);
    b -= split * a.suffix_tiles * a.kv_heads;
    const int32_t tile = b / a.kv_heads;
    constexpr int ROWS = SUFFIX == MANY ? kManyRows : kFewRows;
    const int32_t keys = min(max(at_global<const int32_t>(a.suffix_lens)[seq], 0), a.suffix_width << a.page_shift);
    s.head = b - tile * a.kv_heads;
    s.table = at_global<const int32_t>(a.suffix_pages) + static_cast<int64_t>(seq) * a.suffix_width;
    s.token0 = seq * a.q_len;
    s.row0 = tile * ROWS;
    s.rows = min(ROWS, a.q_len * a.group - s.row0);
    s.first = split * a.suffix_chunk;
    s.end = min(s.first + a.suffix_chunk, keys);
    s.part = a.prefix_splits + split;
    s.last0 = keys - a.q_len;
    if (s.first >= s.end) return;                               // the joining kernel knows the length, too
    if constexpr (SUFFIX == MANY) N().run(a, s, lds);
    else F().run(a, s, lds);
}

}  // namespace serving
