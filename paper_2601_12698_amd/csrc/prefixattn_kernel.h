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
// The second product's weights are rounded to the activations' type, which is what a matrix instruction takes at its full rate beside
// values of that type: half a unit in the last place of each, 1.9e-3 to 2.2e-3 of the outputs' norm in bf16 where weights in fp32 and the
// outputs' own rounding leave 1.6e-3.  Their sum l is of the weights before that.
// O is scaled down only when a maximum grows by more than 2^8 (weights stay below that, and l and O are relative to the same
// number): most tiles leave 16 to 128 multiplications a lane out.
//
// FEW (up to 16 rows; four or eight waves): every wave has all rows and takes every fourth (eighth) tile of 32 keys by itself, keys straight
// from memory into registers, values through LDS of its own, no barrier until the waves' results are joined.  Bound by memory:
// 4 x 32 heads over 131072 bf16 keys of 128, 537 MB in 95 us, 5.6 TB/s (e4m3 270 MB in 54 us).
//
// MANY (64, 128 or 256 rows): the tile of keys and values is staged in LDS for all waves, as elements, two tiles deep, and asked for
// two turns before that.  A wave has 32 rows and all keys of the tile; where there are 64 rows, two waves share rows and halve the
// keys, and are joined at the end (16 rows a wave and all keys: each wave reads all of the tile from LDS, 8 x 40 heads over 131072
// e4m3 keys 87 us a call, so 70).  More rows a workgroup mean fewer reads of a head's keys: 256 rows read a tile from LDS once for
// 128 operations a byte, one workgroup a CU.  Heads over 128 leave no registers for 32 rows a wave (32 x 256 sums are half of them):
// 16 rows, eight waves.
//   64 x 64 heads over 32768 e4m3 keys, 69 GFLOP: 85 to 93 us, 740 to 810 TFLOP/s, of 1211 that a large matrix product reaches here
//   (and 1340 of matrix instructions alone: power is the limit).  What is between is the softmax: exponentials, conversions and maxima
//   are as many cycles as the products, and waves that share a SIMD overlap them in part.  16 x 4 x 32 heads of 256 over 65536
//   fp16 keys: 600 TFLOP/s.
// Tried at the 256-row form and not faster: the next tile's scores before this one's sums, 64 rows a wave, half the waves a phase
// behind, wave priorities, fixed instruction orders.  At heads of 256, two waves that share weights through LDS and halve the elements
// of O: half the LDS reads, two barriers a tile, 3 to 7 % faster over 65536 keys and up to 6 % slower over 4001.
//
// A short prefix is seen by each suffix's workgroup before its own keys (`turn`): one launch.  Where the suffixes'
// workgroups fill the chip, they join the prefix's parts themselves (`finish`): two launches.  Else the joining kernel does.
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
constexpr float kMost = 0x1.fffffep127f;
// fp16 weights are 2^7 times larger (at most 2^15), so that they are normal numbers down to 2^-21 of the largest.
template <int DT> constexpr float kLift = DT == DT_FP16 ? 7.0f : 0.0f;
constexpr uint64_t full_of(int bits) { return bits == 64 ? ~0ull : (1ull << bits) - 1; }
constexpr float kNone = -__builtin_huge_valf();

// A row's scale as the conversions take it: they look at the exponent alone, to which 0 is 2^-127 and 255 NaN.
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

// The larger of two, NaN if one is NaN: three operands an instruction, and unlike fmaxf without making signalling NaNs quiet first.
__device__ __forceinline__ float larger(float x, float y) { return __builtin_elementwise_maximum(x, y); }
// ln 2 (m + log2 l): -infinity where no key was seen.
__device__ __forceinline__ float lse_of(float m, float l) { return (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f; }

template <int ROWS> struct acc;
template <> struct acc<16> { typedef f32x4 type; };
template <> struct acc<32> { typedef f32x16 type; };

__device__ __forceinline__ float other_half_max(float x) { const pair p = with_half(x); return larger(p.a, p.b); }
__device__ __forceinline__ float other_half_sum(float x) { const pair p = with_half(x); return p.a + p.b; }
__device__ __forceinline__ float other_row_max(float x) { const pair p = with_row(x); return larger(p.a, p.b); }
__device__ __forceinline__ float other_row_sum(float x) { const pair p = with_row(x); return p.a + p.b; }

// Values that are no finite numbers, of keys that some rows of a tile see and others do not.  A weight of zero does not take such a
// value out of a product.  A share that holds such keys looks at its sums when it is done, and if one is not finite goes over its keys
// again with SAFE: the value becomes a zero in LDS, and `first` keeps, for each element, the first key at which it was NaN, +inf or
// -inf.  Rows see the keys up to a last one: those from that first key on get the value added to their sum.  Looking at the sums costs
// a meeting of the waves, where there are several queries a sequence: 2 x 64 queries of 32 heads over 1000 and 1000 keys 0.4 us of 17
// (e4m3, heads of 64), 0.6 of 39 (bf16, 256), 2 x 2 over 301 and 17 0.35 of 8.  Looking through every such tile as it is staged takes 2
// of 17 and 3 of 39.  TREE: such keys are nodes of a tree (include/treeattn.h), and `nodes` keeps for each
// element those at which it was +inf or NaN, and those at which it was -inf or NaN.
template <int DP, bool TREE> struct StrayKeys { int32_t first[3][DP]; };
template <int DP> struct StrayKeys<DP, true> { uint64_t nodes[2][DP]; };
template <int DT, int DP, bool TREE = false>
struct Strays : StrayKeys<DP, TREE> {
    static constexpr uint32_t EXPONENT = DT == DT_BF16 ? 0x7f80u : 0x7c00u;
    int32_t odd[16];                                            // of each wave: a sum was not finite

    // Each wave says whether one of its sums is not finite (look); the waves meet; if one said so, all go over the keys again (found).
    template <int N, typename V>
    __device__ __forceinline__ void look(const V (&o)[N], int wave, bool mine)
    {
        constexpr int EACH = sizeof(V) / 4;
        float top[2] = {0, 0};                                  // NaN if one is
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int i = 0; i < EACH; ++i) top[i / 2 % 2] = larger(top[i / 2 % 2], __builtin_fabsf(o[t][i]));
        const bool some = __any(mine && !(larger(top[0], top[1]) < __builtin_huge_valf()));
        if (threadIdx.x % 64 == 0) odd[wave] = some;
    }
    template <int WAVES>
    __device__ __forceinline__ bool found()
    {
        int32_t any = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) any |= odd[w];
        if (__builtin_expect(any == 0, 1)) return false;
        for (int i = threadIdx.x; i < (TREE ? 2 : 3) * DP; i += 64 * WAVES) {
            if constexpr (TREE) this->nodes[0][i] = 0;
            else this->first[0][i] = 0x7fffffff;
        }
        __syncthreads();
        return true;
    }
    // Eight elements in LDS, those of `key` (TREE: of the node of this number) from e on.
    __device__ __forceinline__ void take_out(char* at, int32_t key, int32_t e)
    {
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
            uint16_t* p = reinterpret_cast<uint16_t*>(at) + i;
            const uint32_t w = *p;
            if ((w & EXPONENT) != EXPONENT) continue;
            const int kind = (w & (EXPONENT ^ 0x7fffu)) ? 0 : w >> 15 ? 2 : 1;
            if constexpr (TREE) {
                if (kind != 2) atomicOr(reinterpret_cast<unsigned long long*>(&this->nodes[0][e + i]), 1ull << key);
                if (kind != 1) atomicOr(reinterpret_cast<unsigned long long*>(&this->nodes[1][e + i]), 1ull << key);
            } else atomicMin(&this->first[kind][e + i], key);
            *p = 0;
        }
    }
    // What element e of a row's sum gets; the row sees keys up to `last` (TREE: and the nodes `seen`).
    __device__ __forceinline__ float of(int32_t e, int32_t last, uint64_t seen) const
    {
        if constexpr (TREE) {
            const float x = this->nodes[0][e] & seen ? __builtin_huge_valf() : 0.0f;
            return this->nodes[1][e] & seen ? x - __builtin_huge_valf() : x;         // both: NaN
        } else {
            float x = this->first[1][e] <= last ? __builtin_huge_valf() : 0.0f;
            x = this->first[2][e] <= last ? x - __builtin_huge_valf() : x;
            return this->first[0][e] <= last ? __builtin_nanf("") : x;
        }
    }
};

// The thread's number; ANEW: as if it had not been known, so that what follows from it is not held in registers meanwhile.
template <bool ANEW>
__device__ __forceinline__ int thread()
{
    int t = threadIdx.x;
    if constexpr (ANEW) asm volatile("" : "+v"(t));
    return t;
}

// A workgroup's share: rows [row0, row0 + rows) of a key head, rows counted token by token from token `token0`, keys
// [first, end) of a table of pages.  Query i of its sequence sees keys up to last0 + i.
// Keys from `turn` on are those of a second table, counted from 0 there (a short prefix, then a suffix; kAll: none).
struct Share {
    addr_t table, table2;
    int32_t turn, head, token0, row0, rows, first, end, part, last0;
};
constexpr int32_t kAll = 0x7fffffff;
// The last key that all queries of a suffix's sequence see; kAll if those are all of the share's.
__device__ __forceinline__ int32_t sure_of(const Share& s)
{
    const int32_t last = max(s.last0, s.turn < kAll ? s.turn - 1 : -1);
    return last >= s.end - 1 ? kAll : last;
}
__device__ __forceinline__ int32_t page_at(const AttnArgs& a, const Share& s, int32_t key)
{
    const bool second = key >= s.turn;
    return at_global<const int32_t>(second ? s.table2 : s.table)[(second ? key - s.turn : key) >> a.page_shift];
}

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
    row.last = s.last0 >= kAll ? kAll : max(s.last0 + i, s.turn < kAll ? s.turn - 1 : -1);     // a prefix is seen whole, also by a query before its suffix
    row.q = token * a.q_token + head * a.q_head;
    return row;
}
// Of a tree: the nodes that row r of a share sees, whose keys follow last0, and which of the 64 keys from key0 on it sees with that.
__device__ __forceinline__ uint64_t nodes_of(const AttnArgs& a, const Share& s, int32_t r)
{
    return at_global<const uint64_t>(a.masks)[s.token0 + (s.row0 + (r < s.rows ? r : 0)) / a.group] & full_of(a.q_len);
}
__device__ __forceinline__ uint64_t seen_from(const Share& s, uint64_t nodes, int32_t key0)
{
    const int32_t node = key0 - 1 - s.last0;                    // that key's number among the nodes; below 0 it is before them
    if (node >= 0) return node < 64 ? nodes >> node : 0;
    return node > -64 ? nodes << -node | full_of(-node) : ~0ull;
}

// Where a key's elements and its scale lie.  Where its page is not in the cache, or the key is beyond the share's end, callers
// take page 0 and set the piece to zeros afterwards: loads stand in no branch, so that all of a tile's are under way together.
struct Place {
    uint64_t bytes, row;
};
__device__ __forceinline__ Place place_of(const AttnArgs& a, int32_t head, int32_t page, int32_t key, int32_t row_bytes)
{
    // 32-bit factors, and one of 24 bits (an offset in a page times a row's bytes): a 64-bit product is four slow instructions
    const uint32_t in = static_cast<uint32_t>(key) & ((1u << a.page_shift) - 1);
    return Place{static_cast<uint64_t>(static_cast<uint32_t>(page)) * a.page_bytes + (static_cast<uint32_t>(head) * a.head_bytes + __umul24(in, row_bytes)),
                 static_cast<uint64_t>(static_cast<uint32_t>(page)) * a.page_rows + ((static_cast<uint32_t>(head) << a.page_shift) + in)};
}
__device__ __forceinline__ bool in_cache(const AttnArgs& a, int32_t page) { return static_cast<uint32_t>(page) < static_cast<uint32_t>(a.pages); }

// Eight elements of a row's query from e on, zeros beyond the row or the head.
template <int DT>
__device__ __forceinline__ typename mat<DT>::T8 query_piece(const AttnArgs& a, const Row& row, int32_t e)
{
    typedef typename mat<DT>::T8 T8;
    const auto* p = at_global<const typename mat<DT>::T>(a.q) + row.q + (e < a.d ? e : 0);
    T8 x;
    if (a.q_wide) x = *reinterpret_cast<const T8*>(p);
    else
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = p[j];
    return row.in && e < a.d ? x : T8{};
}

template <int DT, int FORMAT, int DP, int WAVES, bool TREE = false>
struct Few {
    typedef mat<DT> M;
    typedef typename M::T T;
    typedef typename M::T8 T8;
    static constexpr bool CODES = FORMAT == KVCACHE_E4M3;
    static constexpr int ES = CODES ? 1 : 2;
    static constexpr int THREADS = 64 * WAVES, ROWS = 16;
    static constexpr int TILE = 32;                             // keys of a wave at a time
    static constexpr int NC = DP / 32;                          // steps of 32 elements in S
    static constexpr int NK = CODES ? NC / 2 : NC;              // 16-byte loads of a lane for 16 keys
    static constexpr int NT = DP / 16;                          // tiles of 16 elements in O
    static constexpr int PIECES = DP * ES / 16;                 // 16-byte pieces of a key's values
    static constexpr int NV = TILE * PIECES / 64;
    static constexpr int VROW = DP * 2 + 32;                    // bytes from key to key in LDS: 4 keys' 32 bytes fall on 4 groups of banks
    static constexpr int WAVE_LDS = TILE * VROW;
    static constexpr int OROW = DP + 4;                         // floats from row to row where waves are joined
    static constexpr int JOIN_LDS = WAVES * (WAVE_LDS > ROWS * OROW * 4 ? WAVE_LDS : ROWS * OROW * 4);
    // Eight waves' 256 registers do not hold keys and values of 32 x 256 elements in 16 bits, sums and queries: the queries stay in LDS,
    // what follows from the lane is made anew in every turn and after the last, and the places of values are scalars until they are
    // loaded from (32 x 8 heads over a page and 500 fp16 keys at most 19.3 us; with a place for each lane, and so scratch memory between
    // the loads, 22.4; with the queries in registers, too, 32.4).
    static constexpr bool Q_LDS = !CODES && DP > 128 && WAVES == 8;
    static constexpr int QROW = DP * 2 + 32;
    static constexpr int MASKS_LDS = JOIN_LDS + ROWS * QROW;    // and so do a tree's masks
    static constexpr int LDS = JOIN_LDS + (Q_LDS ? ROWS * (QROW + (TREE ? 8 : 0)) : 0);
    typedef Strays<DT, DP, TREE> St;
    static __device__ __forceinline__ int32_t nodes_at(const Share& s) { return TREE ? s.last0 + 1 : 0; }
    static constexpr int SUFFIX_LDS = LDS + static_cast<int>(sizeof(St));
    // What the waves tell each other at the end, once for both kinds of shares.
    struct Ends {
        float2 ml[WAVES][ROWS];
        float weight[ROWS][kFinishSplits], own[ROWS], inverse[ROWS];
    };
    static __device__ __forceinline__ Ends& ends()
    {
        __shared__ Ends e;
        return e;
    }

    u32x4 k[2][NK], v[NV];
    uint32_t k_scale, v_scale;                                  // of key lane % 32
    uint32_t valid;                                             // keys of the tile that are there

    static __device__ __forceinline__ int32_t local(const Share& s, int32_t key) { return key >= s.turn ? key - s.turn : key; }

    // `page` is that of key lane % 32.
    __device__ __forceinline__ void load(const AttnArgs& a, const Share& s, int32_t key0, int32_t page, int lane)
    {
        const int32_t mine = key0 + (lane & 31);
        const bool there = mine < s.end && in_cache(a, page);
        valid = static_cast<uint32_t>(__ballot(there));
        if (!there) page = 0;
        if constexpr (CODES) {
            const uint64_t row = place_of(a, s.head, page, local(s, mine), 0).row;
            k_scale = at_global<const uint8_t>(a.k_scale)[row];
            v_scale = at_global<const uint8_t>(a.v_scale)[row];
        }
        const char* kp = at_global<const char>(a.k_pages);
        const char* vp = at_global<const char>(a.v_pages);
        const int32_t row_bytes = a.d * ES;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int at = 16 * t + (lane & 15);
            const char* r = kp + place_of(a, s.head, __shfl(page, at), local(s, key0 + at), row_bytes).bytes;
#pragma unroll
            for (int c = 0; c < NK; ++c) {
                const int32_t b = 64 * c + 16 * (lane >> 4);    // 16 bytes: 8 elements, or 16 codes
                k[t][c] = *reinterpret_cast<const u32x4*>(r + (b < row_bytes ? b : 0));
            }
        }
        const int32_t b = 16 * (lane % PIECES);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            uint64_t from;
            if constexpr (PIECES == 32) {                       // two keys a load, one for each half of the lanes: their places are scalars
                const int32_t first = __builtin_amdgcn_readfirstlane(key0) + 2 * i;
                const uint64_t lo = place_of(a, s.head, __builtin_amdgcn_readlane(page, 2 * i), local(s, first), row_bytes).bytes;
                const uint64_t hi = place_of(a, s.head, __builtin_amdgcn_readlane(page, 2 * i + 1), local(s, first + 1), row_bytes).bytes;
                from = lane < 32 ? lo : hi;
            } else {
                const int at = (64 / PIECES) * i + lane / PIECES;
                from = place_of(a, s.head, __shfl(page, at), local(s, key0 + at), row_bytes).bytes;
            }
            v[i] = *reinterpret_cast<const u32x4*>(vp + from + (b < row_bytes ? b : 0));
        }
    }
    // Zeros in the place of keys that are not there and of elements beyond the head.
    __device__ __forceinline__ void clear(const AttnArgs& a, int lane)
    {
        const int32_t row_bytes = a.d * ES;
        if (valid == 0xffffffffu && row_bytes == DP * ES) return;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < NK; ++c)
                if (!((valid >> (16 * t + (lane & 15))) & 1) || 64 * c + 16 * (lane >> 4) >= row_bytes) k[t][c] = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (!((valid >> ((64 / PIECES) * i + lane / PIECES)) & 1)) v[i] = u32x4{0, 0, 0, 0};
        if (!((valid >> (lane & 31)) & 1)) k_scale = v_scale = 127;
    }

    static __device__ __forceinline__ int32_t page_of(const AttnArgs& a, const Share& s, int32_t key0, int lane)
    {
        return page_at(a, s, min(key0 + (lane & 31), s.end - 1));
    }

    // Over the share's keys: sums O, maximum and sum of weights of this wave's tiles.  `page0`: that of key lane % 32 of the first.
    // SAFE: strays are taken out (see Strays).
    template <bool SAFE>
    __device__ __forceinline__ void pass(const AttnArgs& a, const Share& s, int32_t page0, char* lds, f32x4 (&o)[DP / 16], float& m, float& l)
    {
        const int first = thread<SAFE>(), lane = first & 63, wave = first >> 6;
        const Row row = row_of(a, s, lane & 15);
        const uint64_t nodes = TREE ? nodes_of(a, s, lane & 15) : 0;
        if constexpr (SAFE) page0 = s.first + TILE * wave < s.end ? page_of(a, s, s.first + TILE * wave, lane) : 0;
        T8 q[NC];
        if constexpr (Q_LDS) {
            static_assert(NC == WAVES, "a wave brings one piece of the queries");
            *reinterpret_cast<T8*>(lds + JOIN_LDS + (lane & 15) * QROW + 64 * wave + 16 * (lane >> 4)) = query_piece<DT>(a, row, 32 * wave + 8 * (lane >> 4));
            if constexpr (TREE) *reinterpret_cast<uint64_t*>(lds + MASKS_LDS + 8 * (lane & 15)) = nodes;
            __syncthreads();
        } else
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int32_t e = CODES ? 64 * (c >> 1) + 16 * (lane >> 4) + 8 * (c & 1) : 32 * c + 8 * (lane >> 4);
            q[c] = query_piece<DT>(a, row, e);
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) o[t] = f32x4{0, 0, 0, 0};
        m = kNone, l = 0.0f;
        const float lag = fminf(kLazy / a.c, kMost);

        int32_t key0 = s.first + TILE * wave, page = 0;
        if (key0 < s.end) {
            load(a, s, key0, page0, lane);
            page = page_of(a, s, key0 + WAVES * TILE, lane);
        }
        while (key0 < s.end) {
            // made anew in every turn, so that what follows from it is not held in registers (from where it would go to scratch memory,
            // whose loads wait for those of keys and values)
            const int tid = thread<Q_LDS>(), here = tid & 63, g = here >> 4;
            char* const mine = lds + (tid >> 6) * WAVE_LDS;
            const char* const at_q = lds + JOIN_LDS + (here & 15) * QROW + 16 * g;
            // where this lane's 8 bytes of a transposing read begin: key 4 g + (lane % 16) / 4 of 16, elements 4 (lane % 4) of 16
            const char* const from = mine + (4 * g + ((here & 15) >> 2)) * VROW + 8 * (here & 3);
            clear(a, here);
            // values to LDS, as elements
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int at = (64 / PIECES) * i + here / PIECES, b = here % PIECES;
                if constexpr (CODES) {
                    const float sc = scale_of(__shfl(v_scale, at));
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
                    const float sc = scale_of(__shfl(k_scale, 16 * t + (lane & 15)));
#pragma unroll
                    for (int c = 0; c < NK; ++c) {
                        z[t] = M::mul16(elements_of<DT>(k[t][c][0], k[t][c][1], sc), q[2 * c], z[t]);
                        z[t] = M::mul16(elements_of<DT>(k[t][c][2], k[t][c][3], sc), q[2 * c + 1], z[t]);
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < NK; ++c) z[t] = M::mul16(__builtin_bit_cast(T8, k[t][c]), Q_LDS ? *reinterpret_cast<const T8*>(at_q + 64 * c) : q[c], z[t]);
                }
            }
            const uint32_t there = valid;
            const int32_t now = key0;
            key0 += WAVES * TILE;
            if (key0 < s.end) {
                load(a, s, key0, page, here);
                page = page_of(a, s, key0 + WAVES * TILE, here);
            }
            if (there != 0xffffffffu || now + TILE - 1 > s.last0) {
                // this lane's keys, shifted so that each is a fixed bit
                const uint32_t mine_there = (TREE ? there & static_cast<uint32_t>(seen_from(s, Q_LDS ? *reinterpret_cast<const uint64_t*>(lds + MASKS_LDS + 8 * (here & 15)) : nodes, now)) : there) >> (4 * g);
                const int32_t last = TREE ? TILE : row.last - now - 4 * g;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (!((mine_there >> (16 * t + r)) & 1) || 16 * t + r > last) z[t][r] = kNone;
                if (SAFE && now + TILE - 1 > sure_of(s)) {
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
                    for (int at = here / (DP / 8); at < TILE; at += 64 / (DP / 8))
                        if (now + at > sure_of(s)) reinterpret_cast<St*>(lds + LDS)->take_out(mine + at * VROW + 16 * (here % (DP / 8)), now + at - nodes_at(s), 8 * (here % (DP / 8)));
                }
            }
            float top = z[0][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top = larger(top, z[i >> 2][i & 3]);
            top = other_half_max(other_row_max(top));
            if (__any(top > m + lag)) {
                const float next = larger(m, top);
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
                l += w;                                         // all of it; what the product takes has the activations' bits
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
    }

    // SUFFIX: there may be keys that not all rows see, and the prefix's parts to join.
    template <bool SUFFIX>
    __device__ __forceinline__ void run(const AttnArgs& a, const Share& s, int32_t page0, char* lds)
    {
        f32x4 o[NT];
        float m, l;
        pass<false>(a, s, page0, lds, o, m, l);
        const int tid = thread<true>(), lane = tid & 63, wave = tid >> 6, g = lane >> 4;
        St* const strays = reinterpret_cast<St*>(lds + LDS);
        bool strayed = false;
        if (SUFFIX && __builtin_expect(sure_of(s) < kAll, !Q_LDS)) {     // where registers are few, said to be rare: the pass above gets them
            strays->look(o, wave, true);
            __syncthreads();
            strayed = strays->template found<WAVES>();
            if (__builtin_expect(strayed, 0)) Few().template pass<true>(a, s, 0, lds, o, m, l);
        }

        // the waves' results, joined
        const Row row = row_of(a, s, lane & 15);
        l = other_half_sum(other_row_sum(l));
        auto& [ml, weight, own, inverse] = ends();
        if (lane < 16) ml[wave][lane] = make_float2(m, l);
        __syncthreads();
        float best = kNone, sum = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) best = larger(best, ml[w][lane & 15].x);
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
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
            *reinterpret_cast<f32x4*>(join + (wave * ROWS + (lane & 15)) * OROW + 16 * t + 4 * g) = x;
        }
        const int64_t rows = static_cast<int64_t>(a.batch) * a.q_len * a.q_heads;
        const int64_t each = TREE ? static_cast<int64_t>(a.q_len) * a.q_heads : rows;      // of a part: a sequence's, or all
        const float most = best == kNone ? kNone : best * a.c - kLift<DT>;
        const bool finish = SUFFIX && a.finish;
        if (!finish) {
            if (wave == 0 && lane < 16 && row.in) at_global<float2>(a.part_ml)[s.part * each + row.global] = make_float2(most, sum);
        } else {
            // the rows' weights of the prefix's parts: a wave takes rows in turn, its lanes the parts
            for (int r = wave; r < s.rows; r += WAVES) {
                const int32_t global = row_of(a, s, r).global;
                const float2 mine = make_float2(__shfl(most, r), __shfl(sum, r));
                const float2 x = lane < a.prefix_splits ? at_global<const float2>(a.part_ml)[lane * rows + global] : make_float2(kNone, 0.0f);
                float top = x.x;
#pragma unroll
                for (int i = 32; i; i >>= 1) top = larger(top, __shfl_xor(top, i));
                top = larger(top, mine.x);
                const float w = x.x == kNone ? 1.0f : __builtin_amdgcn_exp2f(x.x - top), w0 = mine.x == kNone ? 1.0f : __builtin_amdgcn_exp2f(mine.x - top);
                float all = w * x.y;
#pragma unroll
                for (int i = 32; i; i >>= 1) all += __shfl_xor(all, i);
                all += w0 * mine.y;
                if (lane < kFinishSplits) weight[r][lane] = w;
                if (lane == 0) {
                    own[r] = w0;
                    inverse[r] = all == 0.0f ? 0.0f : 1.0f / all;
                    if (a.lse) at_global<float>(a.lse)[global] = lse_of(top, all);
                }
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < ROWS * DP / 4; i += THREADS) {
            const int r = i / (DP / 4), e = 4 * (i % (DP / 4));
            if (r >= s.rows || e >= a.d) continue;
            const Row row = row_of(a, s, r);
            const int32_t global = row.global;
            f32x4 x = *reinterpret_cast<const f32x4*>(join + r * OROW + e);
#pragma unroll
            for (int w = 1; w < WAVES; ++w) x += *reinterpret_cast<const f32x4*>(join + (w * ROWS + r) * OROW + e);
            if (SUFFIX && strayed)
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] += strays->of(e + j, row.last, TREE ? nodes_of(a, s, r) : 0);
            if (!finish) {
                *reinterpret_cast<f32x4*>(at_global<float>(a.part_o) + (s.part * each + global) * a.d + e) = x;
                continue;
            }
            x *= own[r];
            const float* o = at_global<const float>(a.part_o) + static_cast<int64_t>(global) * a.d + e;
            for (int32_t p = 0; p < a.prefix_splits; p += 8) {
                f32x4 y[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = *reinterpret_cast<const f32x4*>(o + min(p + j, a.prefix_splits - 1) * rows * a.d);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (p + j < a.prefix_splits) x += weight[r][p + j] * y[j];
            }
            typedef T T4 __attribute__((ext_vector_type(4)));
            T4 y;
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = static_cast<T>(x[j] * inverse[r]);
            *reinterpret_cast<T4*>(at_global<T>(a.out) + static_cast<int64_t>(global) * a.d + e) = y;
        }
    }
};

// TWO: a prefix is seen before a tree's sequence's own keys.
template <int DT, int FORMAT, int DP, int RW, int WAVES, int KS = 1, bool TREE = false, bool TWO = false>
struct Many {
    typedef mat<DT> M;
    typedef typename M::T T;
    typedef typename M::T8 T8;
    static constexpr bool CODES = FORMAT == KVCACHE_E4M3, WIDE = RW == 32;
    static constexpr int ES = CODES ? 1 : 2, THREADS = 64 * WAVES, GROUPS = WAVES / KS, ROWS = RW * GROUPS;
    static constexpr int TILE = 64;                             // keys at a time: two workgroups' tiles, or one of eight waves, fit a CU
    static constexpr int KEYS = TILE / KS;                      // of a wave
    typedef typename acc<RW>::type A;                           // of a lane: WIDE 16 of 32 keys (or elements) by rows, else 4 of 16
    static constexpr int AN = WIDE ? 16 : 4;
    static constexpr int NS = KEYS / RW;                        // pieces of S
    static constexpr int KC = WIDE ? 16 : 32;                   // elements, or keys, that one matrix instruction sums over
    static constexpr int NC = DP / KC;
    static constexpr int NT = DP / RW;                          // pieces of O
    static constexpr int PIECES = DP * ES / 16;
    static constexpr int NP = TILE * PIECES / THREADS;          // 16-byte pieces of keys, and of values, that a thread stages
    static_assert(NP >= 1, "fewer pieces than threads");
    // Bytes from key to key in LDS: lanes that are served together fall on different banks, for the keys 16 bytes of 16 keys (WIDE) or
    // 32 of 8, and for a transposing read of the values 4 keys' 64 bytes (WIDE) or 8 keys' 32.  (16 rows a wave with 16 bytes between
    // the keys: a quarter of the LDS's time goes to conflicts, and 16 x 4 x 32 heads of 256 over 65536 fp16 keys take 260 us, not 249.)
    static constexpr int KROW = DP * 2 + (WIDE ? 16 : 32), VROW = DP * 2 + (WIDE ? 64 : 32);
    static constexpr int BUF = TILE * (KROW + VROW) + TILE;     // keys, values, a byte for each key that is there
    static constexpr int LDS = 2 * BUF + (TREE && !CODES && DP == 128 ? 8 * ROWS : 0);
    typedef Strays<DT, DP, TREE> St;
    static __device__ __forceinline__ int32_t nodes_at(const Share& s) { return TREE ? s.last0 + 1 : 0; }
    static constexpr int SUFFIX_LDS = LDS + static_cast<int>(sizeof(St));
    static constexpr bool ONE = DP > 128;                       // one set of pieces on their way
    static constexpr bool LATE = !CODES && DP == 128;           // a tree's masks wait in LDS: no register is left for them

    static __device__ __forceinline__ int key_of(int i) { return (THREADS / PIECES) * i + static_cast<int>(threadIdx.x) / PIECES; }
    static __device__ __forceinline__ int piece() { return static_cast<int>(threadIdx.x) % PIECES; }

    // The keys that a tile is of: their table of pages, the first one's number, and their end.  TWO: the prefix ends with a whole tile, those of
    // its keys that are not there masked, so that a tile is of one table.  (A form of its own: this costs the others 1.5 %.)
    struct From {
        addr_t table;
        int32_t base, end;
    };
    static __device__ __forceinline__ From from_of(const AttnArgs& a, const Share& s, int32_t key0)
    {
        if constexpr (TWO) return key0 >= s.turn ? From{s.table2, s.turn, s.end} : From{s.table, 0, a.inline_len};
        else return From{s.table, 0, s.end};
    }
    static __device__ __forceinline__ void pages_of(const AttnArgs& a, const Share& s, int32_t key0, int32_t (&page)[NP])
    {
        const From from = from_of(a, s, key0);
#pragma unroll
        for (int i = 0; i < NP; ++i) page[i] = at_global<const int32_t>(from.table)[(min(key0 + key_of(i), from.end - 1) - from.base) >> a.page_shift];
    }
    // What a thread stages of a tile: pieces on their way from memory, then written to LDS as elements.
    struct Staged {
        u32x4 k[NP], v[NP];
        uint32_t k_scale[NP], v_scale[NP];
        uint32_t valid;                                             // bit i: the key of piece i is there

        __device__ __forceinline__ void load(const AttnArgs& a, const Share& s, int32_t key0, const int32_t (&page)[NP])
        {
            const int32_t row_bytes = a.d * ES, b = 16 * piece() < row_bytes ? 16 * piece() : 0;
            const From from = from_of(a, s, key0);
            valid = 0;
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const bool there = key0 + key_of(i) < from.end && in_cache(a, page[i]);
                valid |= there ? 1u << i : 0u;
                const Place p = place_of(a, s.head, there ? page[i] : 0, key0 + key_of(i) - from.base, row_bytes);
                k[i] = *reinterpret_cast<const u32x4*>(at_global<const char>(a.k_pages) + (p.bytes + b));
                v[i] = *reinterpret_cast<const u32x4*>(at_global<const char>(a.v_pages) + (p.bytes + b));
                if constexpr (CODES) {
                    k_scale[i] = at_global<const uint8_t>(a.k_scale)[p.row];
                    v_scale[i] = at_global<const uint8_t>(a.v_scale)[p.row];
                }
            }
        }
        // Zeros in the place of keys that are not there and of elements beyond the head.
        __device__ __forceinline__ void clear(const AttnArgs& a)
        {
            const bool in = 16 * piece() < a.d * ES;
            if (__all(in && valid == (1u << NP) - 1)) return;
#pragma unroll
            for (int i = 0; i < NP; ++i)
                if (!in || !((valid >> i) & 1)) {
                    k[i] = v[i] = u32x4{0, 0, 0, 0};
                    k_scale[i] = v_scale[i] = 127;
                }
        }
        __device__ __forceinline__ void stage(char* buf) const
        {
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                char* kt = buf + key_of(i) * KROW + (CODES ? 32 : 16) * piece();
                char* vt = buf + TILE * KROW + key_of(i) * VROW + (CODES ? 32 : 16) * piece();
                if constexpr (CODES) {
                    const float ks = scale_of(k_scale[i]), vs = scale_of(v_scale[i]);
                    reinterpret_cast<T8*>(kt)[0] = elements_of<DT>(k[i][0], k[i][1], ks);
                    reinterpret_cast<T8*>(kt)[1] = elements_of<DT>(k[i][2], k[i][3], ks);
                    reinterpret_cast<T8*>(vt)[0] = elements_of<DT>(v[i][0], v[i][1], vs);
                    reinterpret_cast<T8*>(vt)[1] = elements_of<DT>(v[i][2], v[i][3], vs);
                } else {
                    *reinterpret_cast<u32x4*>(kt) = k[i];
                    *reinterpret_cast<u32x4*>(vt) = v[i];
                }
                if (piece() == 0) buf[TILE * (KROW + VROW) + key_of(i)] = static_cast<char>((valid >> i) & 1);
            }
        }
    };

    // Strays of the pieces that this thread staged.
    static __device__ __forceinline__ void look_through(const Share& s, int32_t key0, char* buf, char* lds)
    {
        const int b = piece() * (CODES ? 2 : 1);
#pragma unroll 1
        for (int key = key_of(0); key < TILE; key += THREADS / PIECES)
            if (key0 + key > sure_of(s))
#pragma unroll 1
                for (int h = 0; h < (CODES ? 2 : 1); ++h) reinterpret_cast<St*>(lds + LDS)->take_out(buf + TILE * KROW + key * VROW + 16 * (b + h), key0 + key - nodes_at(s), 8 * (b + h));
    }

    static __device__ __forceinline__ A mul(T8 a, T8 b, A c)
    {
        if constexpr (WIDE) return M::template mul32<A>(a, b, c);
        else return M::mul16(a, b, c);
    }

    // Over the share's keys: sums O, maximum and sum of weights of this wave's rows and keys of the tiles.
    template <bool SAFE>
    __device__ __forceinline__ void pass(const AttnArgs& a, const Share& s, const Row& row, bool busy, char* lds, A (&o)[DP / RW], float& m, float& l)
    {
        // lane = row, and one of 2 (WIDE) or 4 groups of keys or elements
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane % RW, g = lane / RW;
        const int part = wave / GROUPS * KEYS;                   // its keys of a tile
        const int at_row = RW * (wave % GROUPS) + r;
        const uint64_t nodes = TREE && !LATE ? nodes_of(a, s, at_row) : 0;
        if constexpr (TREE && LATE)
            if (static_cast<int>(threadIdx.x) < ROWS) *reinterpret_cast<uint64_t*>(lds + 2 * BUF + 8 * threadIdx.x) = nodes_of(a, s, threadIdx.x);
        T8 q[NC];
#pragma unroll
        for (int t = 0; t < NT; ++t) o[t] = A{};
        m = kNone, l = 0.0f;
        const float lag = fminf(kLazy / a.c, kMost);

        const auto attend = [&](const char* buf, int32_t key0) {
            const char* kt = buf + (part + r) * KROW + 16 * g;
            A z[NS];
#pragma unroll
            for (int t = 0; t < NS; ++t) {
                z[t] = A{};
#pragma unroll
                for (int c = 0; c < NC; ++c) z[t] = mul(*reinterpret_cast<const T8*>(kt + RW * t * KROW + 2 * KC * c), q[c], z[t]);
            }
            // Four of LDS's answers under way, then one asked for with each matrix instruction (left to the compiler, two at a time and
            // both waited for: 16 x 4 x 32 heads of 256 over 65536 fp16 keys 245 us, so 238; 64 x 64 of 128 over 32768 e4m3 91.9 and 90.8;
            // heads of 64, with four instructions a piece, are 1 % slower so).
            if constexpr (DP > 64) {
                __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
                for (int i = 4; i < NS * NC; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
            }
            const uint64_t there = __ballot(buf[TILE * (KROW + VROW) + lane % TILE] != 0) & full_of(TILE);
            if (there != full_of(TILE) || key0 + TILE - 1 > s.last0) {
                // this lane's keys, shifted so that each is a fixed bit (a mask made for every score would be held in registers)
                const uint64_t mine = (TREE ? there & seen_from(s, LATE ? *reinterpret_cast<const uint64_t*>(lds + 2 * BUF + 8 * at_row) : nodes, key0) : there) >> (part + 4 * g);
                const int32_t last = TREE ? TILE : row.last - key0 - part - 4 * g;
#pragma unroll
                for (int t = 0; t < NS; ++t)
#pragma unroll
                    for (int i = 0; i < AN; ++i) {
                        const int at = RW * t + (WIDE ? 8 * (i >> 2) : 0) + (i & 3);
                        if (!((mine >> at) & 1) || at > last) z[t][i] = kNone;
                    }
            }
            float top = z[0][0];
#pragma unroll
            for (int i = 1; i < NS * AN; ++i) top = larger(top, z[i / AN][i % AN]);
            if constexpr (!WIDE) top = other_row_max(top);
            top = other_half_max(top);
            if (__any(top > m + lag)) {
                const float next = larger(m, top);
                const float down = m == kNone ? 0.0f : __builtin_amdgcn_exp2f((m - next) * a.c);
                l *= down;
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < AN; ++i) o[t][i] *= down;
                m = next;
            }
            const float base = m == kNone ? 0.0f : m * a.c - kLift<DT>;
            // where this lane's 8 bytes of a transposing read begin: of 4 keys, its (lane % 16) / 4 th, elements 4 (lane % 4) of 16
            const char* vt = buf + TILE * KROW + (part + 4 * g + ((lane & 15) >> 2)) * VROW + (WIDE ? 32 * ((lane >> 4) & 1) : 0) + 8 * (lane & 3);
#pragma unroll
            for (int u = 0; u < KEYS / KC; ++u) {
                T8 p;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float x = WIDE ? z[u / 2][(8 * u + j) % AN] : z[2 * u + j / 4][j % 4];
                    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(x, a.c, -base));
                    l += w;
                    p[j] = static_cast<T>(w);
                }
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const char* at = vt + KC * u * VROW + 2 * RW * t;
                    o[t] = mul(two_transposed<DT>(at, at + KC / 2 * VROW), p, o[t]);
                }
            }
        };

        if (s.first < s.end) {
            // Tiles are asked for two turns before they are staged (a turn is shorter than memory takes), in two sets of registers.  Heads
            // over 128 have longer turns and no registers for that: one set, asked for again as soon as it is staged.
            // Page numbers are asked for before the pieces, and both in every turn, also for tiles that are beyond the end (whose keys
            // then are not there): loads come back in their order and are waited for by their number, so that a page number behind its
            // turn's pieces, or loads in a branch, would make every wait one for the newest.
            Staged even, odd;
            int32_t page[NP];
            const auto ask = [&](Staged& to, int32_t key0) {
                int32_t now[NP];
#pragma unroll
                for (int i = 0; i < NP; ++i) now[i] = page[i];
                pages_of(a, s, key0 + TILE, page);
                to.load(a, s, key0, now);
            };
            pages_of(a, s, s.first, page);
            ask(even, s.first);
#pragma unroll
            for (int c = 0; c < NC; ++c) q[c] = query_piece<DT>(a, row, KC * c + 8 * g);
            if constexpr (!ONE) ask(odd, s.first + TILE);
            even.clear(a);
            even.stage(lds);
            if (SAFE && s.first + TILE - 1 > sure_of(s)) look_through(s, s.first, lds, lds);
            if constexpr (ONE) ask(even, s.first + TILE);
            __syncthreads();
            // one turn: `key0`'s tile is in `buf`, the next one arrives in `next`, the one after is asked for into `after`
            const auto turn = [&](int32_t key0, char* buf, char* other, Staged& next, Staged& after) {
                if constexpr (!ONE) ask(after, key0 + 2 * TILE);
                if (busy) attend(buf, key0);
                if (key0 + TILE < s.end) {
                    next.clear(a);
                    next.stage(other);
                    if (SAFE && key0 + 2 * TILE - 1 > sure_of(s)) look_through(s, key0 + TILE, other, lds);
                }
                if constexpr (ONE) ask(after, key0 + 2 * TILE);
                __syncthreads();
            };
            Staged& second = ONE ? even : odd;
            int32_t key0 = s.first;
            for (; key0 + TILE < s.end; key0 += 2 * TILE) {
                turn(key0, lds, lds + BUF, second, even);
                turn(key0 + TILE, lds + BUF, lds, even, second);
            }
            if (key0 < s.end) turn(key0, lds, lds + BUF, second, even);
        }
    }

    // SUFFIX: there may be keys that not all rows see, and the prefix's parts to join.
    template <bool SUFFIX>
    __device__ __forceinline__ void run(const AttnArgs& a, const Share& s, char* lds)
    {
        A o[NT];
        float m, l;
        int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane % RW, g = lane / RW;
        int group = wave % GROUPS, part = wave / GROUPS * KEYS;  // its rows, and its keys of a tile
        Row row = row_of(a, s, RW * group + r);
        bool busy = RW * group < s.rows;                         // waves without rows only help to stage
        pass<false>(a, s, row, busy, lds, o, m, l);
        const auto anew = [&] {                                  // not held in registers over a pass, where a tree leaves none
            if constexpr (TREE) {
                const int t = thread<true>();
                lane = t & 63, wave = t >> 6, r = lane % RW, g = lane / RW;
                group = wave % GROUPS, part = wave / GROUPS * KEYS;
                row = row_of(a, s, RW * group + r);
                busy = RW * group < s.rows;
            }
        };
        anew();
        St* const strays = reinterpret_cast<St*>(lds + LDS);
        bool strayed = false;
        if (SUFFIX && sure_of(s) < kAll) {
            strays->look(o, wave, busy);
            __syncthreads();
            strayed = strays->template found<WAVES>();
            if (__builtin_expect(strayed, 0)) {
                pass<true>(a, s, row, busy, lds, o, m, l);
                anew();
            }
        }
        if constexpr (KS == 2) {
            // what the waves of a tile's other half found, register by register
            constexpr int N = NT * AN;
            static_assert(GROUPS * (N + 2) * 64 * 4 <= LDS, "the other half's results do not fit");
            float* at = reinterpret_cast<float*>(lds) + group * (N + 2) * 64 + lane;
            if (part && busy) {
#pragma unroll
                for (int i = 0; i < N; ++i) at[64 * i] = o[i / AN][i % AN];
                at[64 * N] = m;
                at[64 * (N + 1)] = l;
            }
            __syncthreads();
            if (part) return;
            if (busy) {
                const float other = at[64 * N], most = larger(m, other);
                const float mine = m == kNone ? 1.0f : __builtin_amdgcn_exp2f((m - most) * a.c), its = other == kNone ? 1.0f : __builtin_amdgcn_exp2f((other - most) * a.c);
#pragma unroll
                for (int i = 0; i < N; ++i) o[i / AN][i % AN] = o[i / AN][i % AN] * mine + at[64 * i] * its;
                l = l * mine + at[64 * (N + 1)] * its;
                m = most;
            }
        }
        if (!busy) return;
        if constexpr (!WIDE) l = other_row_sum(l);
        l = other_half_sum(l);
        if (!row.in) return;
        if (SUFFIX && strayed)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < AN; ++i) o[t][i] += strays->of(RW * t + 8 * (i >> 2) + 4 * g + (i & 3), row.last, TREE ? nodes_of(a, s, RW * group + r) : 0);
        const int64_t rows = static_cast<int64_t>(a.batch) * a.q_len * a.q_heads;
        float most = m == kNone ? kNone : m * a.c - kLift<DT>;
        if (!SUFFIX || !a.finish) {
            const int64_t at = s.part * (TREE ? static_cast<int64_t>(a.q_len) * a.q_heads : rows) + row.global;
            if (g == 0) at_global<float2>(a.part_ml)[at] = make_float2(most, l);
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < AN / 4; ++i) {
                    const int32_t e = RW * t + 8 * i + 4 * g;
                    if (e < a.d)
                        *reinterpret_cast<f32x4*>(at_global<float>(a.part_o) + at * a.d + e) = f32x4{o[t][4 * i], o[t][4 * i + 1], o[t][4 * i + 2], o[t][4 * i + 3]};
                }
            return;
        }
        // the prefix's parts, and the result
        for (int32_t p = 0; p < a.prefix_splits; ++p) {
            const int64_t at = p * rows + row.global;
            const float2 x = at_global<const float2>(a.part_ml)[at];
            const float next = larger(most, x.x);
            const float mine = most == kNone ? 1.0f : __builtin_amdgcn_exp2f(most - next), its = x.x == kNone ? 1.0f : __builtin_amdgcn_exp2f(x.x - next);
            most = next;
            l = l * mine + x.y * its;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < AN / 4; ++i) {
                    const int32_t e = RW * t + 8 * i + 4 * g;
                    const f32x4 y = *reinterpret_cast<const f32x4*>(at_global<const float>(a.part_o) + at * a.d + (e < a.d ? e : 0));
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[t][4 * i + j] = o[t][4 * i + j] * mine + y[j] * its;
                }
        }
        const float inverse = l == 0.0f ? 0.0f : 1.0f / l;
        if (a.lse && g == 0) at_global<float>(a.lse)[row.global] = lse_of(most, l);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < AN / 4; ++i) {
                const int32_t e = RW * t + 8 * i + 4 * g;
                typedef T T4 __attribute__((ext_vector_type(4)));
                T4 y;
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = static_cast<T>(o[t][4 * i + j] * inverse);
                if (e < a.d) *reinterpret_cast<T4*>(at_global<T>(a.out) + static_cast<int64_t>(row.global) * a.d + e) = y;
            }
    }
};

// Workgroups of the prefix first, then those of the suffixes.  Workgroups go round the 8 XCDs; the row tiles of one head and
// key range stand 8 apart, so that they read it through the same L2 at the same time.
// FORM: see prefixattn_args.h.
template <int DT, int FORMAT, int DP, int FORM, int WAVES> struct form;
template <int DT, int FORMAT, int DP, int WAVES> struct form<DT, FORMAT, DP, FEW, WAVES> { typedef Few<DT, FORMAT, DP, WAVES> type; };
template <int DT, int FORMAT, int DP, int WAVES> struct form<DT, FORMAT, DP, FEW_8, WAVES> { typedef Few<DT, FORMAT, DP, 8> type; };
template <int DT, int FORMAT, int DP, int WAVES> struct form<DT, FORMAT, DP, MANY_64, WAVES> { typedef Many<DT, FORMAT, DP, 32, 4, 2> type; };
template <int DT, int FORMAT, int DP, int WAVES> struct form<DT, FORMAT, DP, MANY_128, WAVES> { typedef Many<DT, FORMAT, DP, (DP > 128 ? 16 : 32), (DP > 128 ? 8 : 4)> type; };
template <int DT, int FORMAT, int DP, int WAVES> struct form<DT, FORMAT, DP, MANY_256, WAVES> { typedef Many<DT, FORMAT, DP, 32, 8> type; };

template <int DT, int FORMAT, int DP, int PREFIX, int SUFFIX>
__global__ __launch_bounds__(threads_of(PREFIX, DP), (DP > 128 && PREFIX == FEW ? 1 : 2)) void attn_kernel(AttnArgs a)
{
    constexpr int WAVES = threads_of(PREFIX, DP) / 64;          // few rows use all of them, whatever the prefix's form
    typedef typename form<DT, FORMAT, DP, PREFIX, WAVES>::type P;
    typedef typename form<DT, FORMAT, DP, SUFFIX, WAVES>::type S;
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
    if (threadIdx.x >= S::THREADS) return;                      // a form with more waves than the suffixes' leaves the others idle
    b -= a.prefix_blocks;
    const int32_t seq = b / (a.suffix_tiles * a.suffix_splits * a.kv_heads);
    b -= seq * a.suffix_tiles * a.suffix_splits * a.kv_heads;
    const int32_t split = b / (a.suffix_tiles * a.kv_heads);
    b -= split * a.suffix_tiles * a.kv_heads;
    const int32_t tile = b / a.kv_heads, room = a.suffix_width << a.page_shift;
    s.head = b - tile * a.kv_heads;
    s.token0 = seq * a.q_len;
    s.row0 = tile * S::ROWS;
    s.rows = min(S::ROWS, a.q_len * a.group - s.row0);
    s.part = a.prefix_splits + split;
    s.first = split * a.suffix_chunk;
    s.table = a.suffix_pages + 4 * static_cast<int64_t>(seq) * a.suffix_width;
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
        const int32_t keys = room ? min(max(at_global<const int32_t>(a.suffix_lens)[seq], 0), room) : 0;
        s.end = a.inline_len ? a.inline_len + keys : min(s.first + a.suffix_chunk, keys);
        s.last0 = a.inline_len + keys - a.q_len;
        if (s.first >= s.end && !a.finish) return;              // the joining kernel knows the length, too
        S().template run<true>(a, s, page0, lds);
    } else {
        const int32_t keys = min(max(at_global<const int32_t>(a.suffix_lens)[seq], 0), room);
        s.end = min(s.first + a.suffix_chunk, keys);
        s.last0 = keys - a.q_len;
        if (s.first >= s.end && !a.finish) return;
        S().template run<true>(a, s, lds);
    }
}

}  // namespace serving
