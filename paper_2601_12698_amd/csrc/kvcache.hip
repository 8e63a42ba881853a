// Writing tokens into a paged cache, quantised, and reading them back (include/kvcache.h).
//
// A row is one head of one token.  Both kernels move each byte once and are bound by that: e4m3, 16384 tokens x 8 x 128 fp16 written
// (101 MB) in 18.8 us, 5.4 TB/s; 131072 x 8 x 128 bf16 read back (808 MB) in 136, 5.9 TB/s; 64 tokens 2.7.
// A row is 2 to 32 neighbouring lanes of 8 elements each, keys and values together.  A row that is written stays in registers: its
// lanes find the largest magnitude by exchanges and then round.  (A lane of 16 elements loads 16 bytes of codes at once, but then
// its two stores of 16 bytes each fill every other half line: 131072 tokens x 8 x 128 bf16 165 us, with 8 elements 146.)
// Results of 4 MB and more (keys and values in 16 bits) go past the caches: 131072 tokens read back 146 -> 138 us, 16384 22.5 -> 17.3
// (5.8 TB/s), 4999 x 4 x 256 fp16 6.5 -> 6.4; written, 16384 x 8 x 128 23.2 -> 20.2 us, 4999 x 4 x 256 8.5 -> 7.9, 131072 151 -> 148; 512
// to 2048 tokens the same.  What comes next reads them from memory: a write of 131072 tokens and attention of 4 x 32 heads to them 192
// us, not 199, of 16384 33.6 and 33.1; 16384 read back and copied 42.4 and 37.3, 131072 339 and 334, 8192 and two matrix products
// 46.5 and 45.4, 2048 41.0 and 41.2.  Loads that go past the caches lose 2 to 20 %.
#include "kvcache.h"
#include "serving_internal.h"

using namespace addrms_host;
using namespace serving;

namespace {

constexpr int kThreads = 256;
constexpr uint32_t kBlock = 8;               // tokens of a head that are written side by side (16384 x 8 x 128: 21.4 us token by token, 19.8 with 8 or 16)
constexpr int64_t kPastBytes = 4 << 20;      // of keys and values in 16 bits

struct CacheArgs {
    addr_t k, v, slots, k_pages, v_pages, k_scale, v_scale;
    int64_t tokens, rows, cache_slots;
    int64_t ks[2], vs[2];                    // strides of k and v: token, head
    uint32_t heads, d, lanes_log2, page_shift;
};

template <bool PAST, typename P>
__device__ __forceinline__ void put(P* p, P v)
{
    if constexpr (PAST) __builtin_nontemporal_store(v, p);
    else *p = v;
}

// Row of the cache that a slot's head is: pages are [heads][page_size].
__device__ __forceinline__ int64_t cache_row(int64_t slot, uint32_t head, const CacheArgs& a)
{
    const int64_t page = slot >> a.page_shift, offset = slot & ((1ll << a.page_shift) - 1);
    return ((page * a.heads + head) << a.page_shift) + offset;
}

// Scale byte of a row whose largest magnitude is `top`: with top = m 2^x, 1 <= m < 2, the least e with top 2^-e <= 448 = 1.75 * 2^8
// is x - 8, or x - 7 where m > 1.75.  Adding the fraction's distance from 1.75 to the bits carries into the exponent exactly then.
__device__ __forceinline__ uint32_t scale_byte(float top)
{
    const int32_t x = static_cast<int32_t>((__builtin_bit_cast(uint32_t, top) + 0x1fffffu) >> 23) - 8;
    return top > 0.0f ? static_cast<uint32_t>(min(max(x, 1), 254)) : 127u;
}

// Eight elements, those beyond the row zeros.
template <int DT> using vec8 = typename elem<DT>::type __attribute__((ext_vector_type(8)));
template <int DT, bool WIDE>
__device__ __forceinline__ vec8<DT> load8(const typename elem<DT>::type* p, bool in)
{
    vec8<DT> raw = {};
    if (in) {
        if constexpr (WIDE) raw = *reinterpret_cast<const vec8<DT>*>(p);
        else
#pragma unroll
            for (int j = 0; j < 8; ++j) raw[j] = p[j];
    }
    return raw;
}

template <int DT, bool PAST>
__device__ __forceinline__ void quantise(vec8<DT> raw, bool in, uint32_t lanes, bool first, char* codes, uint8_t* scale)
{
    // the largest magnitude of four significant bits that the type holds
    constexpr float kMost = DT == DT_FP16 ? 61440.0f : 0x1.ep127f;
    float x[8], top = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        x[j] = static_cast<float>(raw[j]);
        const float m = __builtin_fabsf(x[j]);
        if (m < __builtin_huge_valf()) {                             // neither infinite nor NaN
            x[j] = __builtin_copysignf(fminf(m, kMost), x[j]);
            top = fmaxf(top, fminf(m, kMost));
        }
    }
    top = max_of_lanes(top, lanes);
    const uint32_t s = scale_byte(top);
    const float inverse = __builtin_bit_cast(float, (254u - s) << 23);   // 2^-(s - 127); s = 254 is not reached: kMost is below 2^128
    u32x2 out;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * j] * inverse, x[4 * j + 1] * inverse, 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * j + 2] * inverse, x[4 * j + 3] * inverse, w, true);
        out[j] = static_cast<uint32_t>(w);
    }
    if (in) put<PAST>(reinterpret_cast<u32x2*>(codes), out);
    if (first) *scale = static_cast<uint8_t>(s);
}

template <int DT, int FORMAT, bool WIDE, bool PAST>
__global__ __launch_bounds__(kThreads) void write_kernel(CacheArgs a)
{
    typedef typename elem<DT>::type T;
    const uint32_t lanes = 1u << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
    // eight tokens of one head, then of the next: their codes and scale bytes lie side by side
    const uint32_t at = blockIdx.x * (kThreads >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2), block = at / (kBlock * a.heads), in_block = at - block * (kBlock * a.heads);
    const uint32_t h = in_block / kBlock;
    const int64_t t = static_cast<int64_t>(block) * kBlock + in_block % kBlock;
    if (t >= a.tokens) return;                                       // all lanes of a row together
    const bool in = 8 * lane < a.d;
    const int64_t slot = at_global<const int64_t>(a.slots)[t];
    const vec8<DT> k = load8<DT, WIDE>(at_global<const T>(a.k) + t * a.ks[0] + h * a.ks[1] + 8 * lane, in);
    const vec8<DT> v = load8<DT, WIDE>(at_global<const T>(a.v) + t * a.vs[0] + h * a.vs[1] + 8 * lane, in);
    if (slot < 0 || slot >= a.cache_slots) return;
    const int64_t to = cache_row(slot, h, a);
    if constexpr (FORMAT == KVCACHE_E4M3) {
        const int64_t at = to * a.d + 8 * lane;
        quantise<DT, PAST>(k, in, lanes, lane == 0, at_global<char>(a.k_pages) + at, at_global<uint8_t>(a.k_scale) + to);
        quantise<DT, PAST>(v, in, lanes, lane == 0, at_global<char>(a.v_pages) + at, at_global<uint8_t>(a.v_scale) + to);
    } else if (in) {
        put<PAST>(reinterpret_cast<vec8<DT>*>(at_global<T>(a.k_pages) + to * a.d + 8 * lane), k);
        put<PAST>(reinterpret_cast<vec8<DT>*>(at_global<T>(a.v_pages) + to * a.d + 8 * lane), v);
    }
}

// Eight elements of a row as they are read back.
template <int DT, int FORMAT>
struct Piece {
    u32x2 codes;
    vec8<DT> same;
    uint32_t scale;

    __device__ __forceinline__ void load(addr_t pages, addr_t scales, int64_t from, uint32_t e, const CacheArgs& a)
    {
        if constexpr (FORMAT == KVCACHE_E4M3) {
            codes = *reinterpret_cast<const u32x2*>(at_global<const char>(pages) + from * a.d + e);
            scale = at_global<const uint8_t>(scales)[from];
        } else {
            same = *reinterpret_cast<const vec8<DT>*>(at_global<const typename elem<DT>::type>(pages) + from * a.d + e);
        }
    }
    __device__ __forceinline__ vec8<DT> values() const
    {
        typedef typename elem<DT>::type T;
        if constexpr (FORMAT != KVCACHE_E4M3) return same;
        vec8<DT> x;
        // the exponent; with the fraction's first bit, 0 is 2^-127 and 255 NaN
        const float by = __builtin_bit_cast(float, scale << 23 | (scale - 1 >= 254 ? 0x400000u : 0u));
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(codes[j]), false);
            const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(codes[j]), true);
            x[4 * j] = static_cast<T>(lo[0] * by);
            x[4 * j + 1] = static_cast<T>(lo[1] * by);
            x[4 * j + 2] = static_cast<T>(hi[0] * by);
            x[4 * j + 3] = static_cast<T>(hi[1] * by);
        }
        return x;
    }
};

template <int DT, int FORMAT, bool PAST>
__global__ __launch_bounds__(kThreads) void read_kernel(CacheArgs a)
{
    const uint32_t lanes = 1u << a.lanes_log2, lane = threadIdx.x & (lanes - 1);
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (kThreads >> a.lanes_log2) + (threadIdx.x >> a.lanes_log2);
    if (row >= a.rows || 8 * lane >= a.d) return;
    const int64_t t = static_cast<int64_t>(static_cast<uint32_t>(row) / a.heads);
    const uint32_t h = static_cast<uint32_t>(row - t * a.heads);
    const int64_t slot = at_global<const int64_t>(a.slots)[t];
    vec8<DT> k = {}, v = {};
    if (slot >= 0 && slot < a.cache_slots) {
        const int64_t from = cache_row(slot, h, a);
        Piece<DT, FORMAT> kp, vp;
        kp.load(a.k_pages, a.k_scale, from, 8 * lane, a);
        vp.load(a.v_pages, a.v_scale, from, 8 * lane, a);
        k = kp.values();
        v = vp.values();
    }
    typedef typename elem<DT>::type T;
    put<PAST>(reinterpret_cast<vec8<DT>*>(at_global<T>(a.k) + row * a.d + 8 * lane), k);
    put<PAST>(reinterpret_cast<vec8<DT>*>(at_global<T>(a.v) + row * a.d + 8 * lane), v);
}

// Workgroups of a launch; a write goes by blocks of tokens.
int64_t groups_of(int64_t tokens, int32_t heads, int32_t d)
{
    const int64_t per = kThreads >> log2_of(d / 8);
    return (tokens * heads + per - 1) / per;
}
int64_t whole_blocks(int64_t tokens) { return (tokens + kBlock - 1) / kBlock * kBlock; }

int check(int64_t tokens, int32_t heads, int32_t d, int64_t pages, int32_t page_size, int dtype, int format)
{
    if (dtype != ADDRMS_BF16 && dtype != ADDRMS_FP16) return fail(ADDRMS_ERR_UNSUPPORTED_DTYPE, "unsupported dtype %d for a cache", dtype);
    if (format != KVCACHE_SAME && format != KVCACHE_E4M3) return fail(ADDRMS_ERR_INVALID_ARG, "unknown cache format %d", format);
    if (tokens < 0 || heads <= 0 || d <= 0 || pages < 0) return fail(ADDRMS_ERR_INVALID_ARG, "tokens and pages must be >= 0, heads and d > 0");
    if (!power_of_two(page_size) || page_size > 65536) return fail(ADDRMS_ERR_INVALID_ARG, "page_size must be a power of two up to 65536 (got %d)", page_size);
    if (d % 16 != 0 || d > KVCACHE_MAX_HEAD)
        return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "d=%d is not a multiple of 16 up to %d", d, KVCACHE_MAX_HEAD);
    if (heads > 65536 || pages >= (1ll << 31) || tokens >= (1ll << 31) / heads - kBlock || !launchable(groups_of(whole_blocks(tokens), heads, d), kThreads))
        return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "%lld tokens of %d heads or %lld pages are beyond the limits", (long long)tokens, heads, (long long)pages);
    return ADDRMS_OK;
}

int launched(hipError_t e) { return e == hipSuccess ? ADDRMS_OK : fail(ADDRMS_ERR_HIP, "the launch failed: %s", hipGetErrorString(e)); }

CacheArgs args_of(const int64_t* slots, int64_t tokens, int32_t heads, int32_t d, int64_t pages, int32_t page_size)
{
    CacheArgs a = {};
    a.slots = addr(slots);
    a.tokens = tokens, a.rows = tokens * heads, a.cache_slots = pages * page_size;
    a.heads = static_cast<uint32_t>(heads), a.d = static_cast<uint32_t>(d);
    a.page_shift = static_cast<uint32_t>(log2_of(page_size)), a.lanes_log2 = static_cast<uint32_t>(log2_of(d / 8));
    return a;
}

}  // namespace

extern "C" {

int kvcache_write(const void* k, const int64_t* k_strides, const void* v, const int64_t* v_strides, const int64_t* slots, void* k_pages, void* v_pages,
                  uint8_t* k_scale, uint8_t* v_scale, int64_t tokens, int32_t heads, int32_t d, int64_t pages, int32_t page_size, int dtype, int format,
                  void* stream)
{
    if (const int st = check(tokens, heads, d, pages, page_size, dtype, format)) return st;
    if (tokens == 0) return ADDRMS_OK;
    if (!k || !v || !k_strides || !v_strides || !slots || !k_pages || !v_pages || (format == KVCACHE_E4M3 && (!k_scale || !v_scale)))
        return fail(ADDRMS_ERR_INVALID_ARG, "no pointer may be NULL");
    if (!aligned_to(k, 2) || !aligned_to(v, 2) || !aligned_to(slots, 8) || !aligned_to(k_pages, 16) || !aligned_to(v_pages, 16))
        return fail(ADDRMS_ERR_MISALIGNED, "k and v must be aligned to their elements, slots to 8 bytes and pages to 16");
    CacheArgs a = args_of(slots, tokens, heads, d, pages, page_size);
    a.k = addr(k), a.v = addr(v), a.k_pages = addr(k_pages), a.v_pages = addr(v_pages), a.k_scale = addr(k_scale), a.v_scale = addr(v_scale);
    uint64_t bits = a.k | a.v;
    for (int i = 0; i < 2; ++i) {
        a.ks[i] = k_strides[i], a.vs[i] = v_strides[i];
        bits |= static_cast<uint64_t>(a.ks[i] | a.vs[i]) * 2;
    }
    const bool wide = bits % 16 == 0;        // else element by element
    const dim3 grid(static_cast<unsigned>(groups_of(whole_blocks(tokens), heads, d)));
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const bool past = a.rows * d * 4 >= kPastBytes;
#define GO(DT, F) launch_kernel(!wide ? write_kernel<DT, F, false, false> : past ? write_kernel<DT, F, true, true> : write_kernel<DT, F, true, false>, grid, kThreads, s, a)
    if (dtype == ADDRMS_BF16) return launched(format == KVCACHE_E4M3 ? GO(DT_BF16, KVCACHE_E4M3) : GO(DT_BF16, KVCACHE_SAME));
    return launched(format == KVCACHE_E4M3 ? GO(DT_FP16, KVCACHE_E4M3) : GO(DT_FP16, KVCACHE_SAME));
#undef GO
}

int kvcache_read(const void* k_pages, const void* v_pages, const uint8_t* k_scale, const uint8_t* v_scale, const int64_t* slots, void* k_out, void* v_out,
                 int64_t tokens, int32_t heads, int32_t d, int64_t pages, int32_t page_size, int dtype, int format, void* stream)
{
    if (const int st = check(tokens, heads, d, pages, page_size, dtype, format)) return st;
    if (tokens == 0) return ADDRMS_OK;
    if (!k_out || !v_out || !slots || !k_pages || !v_pages || (format == KVCACHE_E4M3 && (!k_scale || !v_scale)))
        return fail(ADDRMS_ERR_INVALID_ARG, "no pointer may be NULL");
    if (!aligned_to(k_out, 16) || !aligned_to(v_out, 16) || !aligned_to(slots, 8) || !aligned_to(k_pages, 16) || !aligned_to(v_pages, 16))
        return fail(ADDRMS_ERR_MISALIGNED, "pages and outputs must be 16-byte aligned and slots 8-byte");
    CacheArgs a = args_of(slots, tokens, heads, d, pages, page_size);
    a.k = addr(k_out), a.v = addr(v_out), a.k_pages = addr(k_pages), a.v_pages = addr(v_pages), a.k_scale = addr(k_scale), a.v_scale = addr(v_scale);
    const dim3 grid(static_cast<unsigned>(groups_of(tokens, heads, d)));
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const bool past = a.rows * d * 4 >= kPastBytes;
#define GO(DT, F) launch_kernel(past ? read_kernel<DT, F, true> : read_kernel<DT, F, false>, grid, kThreads, s, a)
    if (dtype == ADDRMS_BF16) return launched(format == KVCACHE_E4M3 ? GO(DT_BF16, KVCACHE_E4M3) : GO(DT_BF16, KVCACHE_SAME));
    return launched(format == KVCACHE_E4M3 ? GO(DT_FP16, KVCACHE_E4M3) : GO(DT_FP16, KVCACHE_SAME));
#undef GO
}

int64_t kvcache_algorithmic_bytes(int64_t tokens, int32_t heads, int32_t d, int dtype, int format)
{
    if (const int st = check(tokens, heads, d, 1, 1, dtype, format)) return st;
    const int64_t rows = 2 * tokens * heads;
    return rows * d * 2 + (format == KVCACHE_E4M3 ? rows * (d + 1) : rows * d * 2) + 8 * tokens;
}

}  // extern "C"
