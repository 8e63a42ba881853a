// Rotary positions with several axes (include/rotary.h).
//
// A pair (x1, x2) of a head is a complex number; the operator multiplies it by exp(i a), a = position of the pair's
// axis * its frequency.  All heads of a token turn by the same angles, so a workgroup forms them once, for its tokens,
// in LDS, and then walks the tokens' heads; queries and keys are one launch.  Bound by memory: 2 elements moved for
// every 3 operations.  While the angles are formed the first pieces of the heads are already under way.
// 8191 tokens x 40 heads x 128 bf16 (168 MB) 29.0 us, 5.8 TB/s; 2048 x 40 x 96 fp32, interleaved and inverse (63 MB) 11.1; one token 2.7.
#include <math.h>

#include "rotary.h"
#include "serving_internal.h"

using namespace addrms_host;
using namespace serving;

namespace {

constexpr int kThreads = 256;
constexpr int kMaxTurns = 2048;              // angles of one workgroup: 16 KiB of LDS
constexpr int kAhead = 2;                    // pieces of a thread that are under way together (8191 x 40 x 128 bf16: 2 38.5 us, 4 42.5, 8 48)
constexpr int64_t kPastBytes = 4 << 20;      // of output (see rotary_run)

struct RotaryArgs {
    addr_t q, k, q_out, k_out, positions, inv_freq, pair_axis;
    int64_t tokens;
    int64_t qs[2], ks[2], qos[2], kos[2];    // strides: token, head
    int32_t q_heads, heads, pairs, pair_pieces, pieces, axes, tokens_per_wg, heads_per_wg, sign;
};

// cos and sin of an angle in fp64, within 2 units in the last place of fp32.  Where the angle is near a whole number of quarter turns
// its sine or cosine is what remains after they are taken off, so 1 / (2 pi) is two numbers here and the product's rounding is kept: of
// an angle of a million one number leaves 10^-10, and the sine near a half turn, 1e-6 say, would have three digits too few.  What
// remains is at most an eighth of a turn, pi/4 = 0.785, and goes through the series of sine and cosine in fp32, cut after x^9 and x^10:
// what is left out is x^11 / 11! = 1.8e-9 and x^12 / 12! = 1.2e-10, a seventeenth of an fp32 half step at 0.707, and less.
__device__ __forceinline__ float2 turn_of(double angle)
{
    constexpr double kTurn = 0x1.45f306dc9c883p-3, kTurnRest = -0x1.6b01ec5417056p-57;        // 1 / (2 pi)
    const double r = angle * kTurn, rest = __builtin_fma(angle, kTurnRest, __builtin_fma(angle, kTurn, -r));
    const double quarters = r * 4.0, whole = __builtin_rint(quarters);
    const double near = __builtin_fma(4.0, rest, quarters - whole), more = __builtin_rint(near);   // more: 0 below 2^50 quarters, but for borders
    const float x = static_cast<float>((near - more) * 1.57079632679489661923);
    const double turns = whole - 4.0 * __builtin_floor(whole * 0.25) + more;
    const int which = static_cast<int>(turns - 4.0 * __builtin_floor(turns * 0.25));          // 0..3
    const float y = x * x;
    const float s = __builtin_fmaf(
        x * y, __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, 2.75573192e-6f, -1.98412698e-4f), 8.33333333e-3f), -1.66666667e-1f), x);
    const float c = __builtin_fmaf(
        y, __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, __builtin_fmaf(y, -2.75573192e-7f, 2.48015873e-5f), -1.38888889e-3f), 4.16666667e-2f), -0.5f),
        1.0f);
    const float a = (which & 1) ? s : c, b = (which & 1) ? c : s;
    return make_float2((which == 1 || which == 2) ? -a : a, which >= 2 ? -b : b);
}

template <bool PAST, typename T, typename P>
__device__ __forceinline__ void put(T* p, P v)
{
    if constexpr (PAST) __builtin_nontemporal_store(v, reinterpret_cast<P*>(p));
    else *reinterpret_cast<P*>(p) = v;
}

// V elements as one access of V * sizeof(T) bytes.
template <typename T, int V> struct piece { typedef T type __attribute__((ext_vector_type(V))); };

// A piece is V pairs, the elements [j, j + V) and [j + pairs, j + pairs + V), or with INTER the V / 2 pairs of the V elements from
// 2 j on (V = 1: one pair, both elements).  blockDim.x = pieces of a head (pairs, or V elements that are copied), blockDim.y = heads
// side by side.  PAST: outputs are written past the caches.
template <int DT, int V, bool INTER, bool PAST>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a)
{
    typedef typename elem<DT>::type T;
    typedef typename piece<T, V>::type P;
    __shared__ float2 turns[kMaxTurns];

    const int64_t t0 = static_cast<int64_t>(blockIdx.x) * a.tokens_per_wg;
    const int32_t nt = static_cast<int32_t>(min(static_cast<int64_t>(a.tokens_per_wg), a.tokens - t0));
    const int32_t h0 = static_cast<int32_t>(blockIdx.y) * a.heads_per_wg;
    const int32_t nh = min(a.heads_per_wg, a.heads - h0);
    const int32_t px = static_cast<int32_t>(threadIdx.x), step = static_cast<int32_t>(blockDim.y);
    const bool turned = px < a.pair_pieces;
    // where this thread's piece of a head begins, and its second half
    constexpr bool SECOND = !INTER || V == 1;        // a piece has a second half
    const int32_t e0 = turned ? (INTER && V == 1 ? 2 : V) * px : 2 * a.pairs + V * (px - a.pair_pieces);
    const int32_t e1 = turned ? (INTER ? e0 + 1 : e0 + a.pairs) : e0;

    uint32_t at = threadIdx.y;                       // of the tokens' heads, one token's behind the other's
    bool first = true;
    for (int32_t base = 0; base < nt * nh; base += kAhead * step) {
        P x[kAhead], y[kAhead];
        int32_t tt[kAhead], hh[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            tt[i] = static_cast<int32_t>(at / static_cast<uint32_t>(nh));
            hh[i] = h0 + static_cast<int32_t>(at) - tt[i] * nh;
            at += static_cast<uint32_t>(step);
            if (tt[i] < nt) {
                const bool is_k = hh[i] >= a.q_heads;
                const T* p = at_global<const T>(is_k ? a.k : a.q) + (t0 + tt[i]) * (is_k ? a.ks[0] : a.qs[0]) +
                             static_cast<int64_t>(is_k ? hh[i] - a.q_heads : hh[i]) * (is_k ? a.ks[1] : a.qs[1]);
                x[i] = *reinterpret_cast<const P*>(p + e0);
                if (SECOND && turned) y[i] = *reinterpret_cast<const P*>(p + e1);
            }
        }
        if (first) {
            first = false;
            const int32_t threads = static_cast<int32_t>(blockDim.x) * step;
            const int64_t* pos = at_global<const int64_t>(a.positions);
            for (int32_t i = static_cast<int32_t>(threadIdx.y * blockDim.x + threadIdx.x); i < nt * a.pairs; i += threads) {
                const int32_t token = i / a.pairs, pair = i - token * a.pairs;
                const int32_t axis = min(static_cast<int32_t>(at_global<const uint8_t>(a.pair_axis)[pair]), a.axes - 1);
                const double angle = static_cast<double>(pos[axis * a.tokens + t0 + token]) * at_global<const double>(a.inv_freq)[pair];
                float2 cs = turn_of(angle);
                if (a.sign < 0) cs.y = -cs.y;
                turns[i] = cs;
            }
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            if (tt[i] >= nt) continue;
            const bool is_k = hh[i] >= a.q_heads;
            T* p = at_global<T>(is_k ? a.k_out : a.q_out) + (t0 + tt[i]) * (is_k ? a.kos[0] : a.qos[0]) +
                   static_cast<int64_t>(is_k ? hh[i] - a.q_heads : hh[i]) * (is_k ? a.kos[1] : a.qos[1]);
            if (turned) {
                constexpr int N = SECOND ? V : V / 2;       // pairs of the piece
                const float2* cs = turns + tt[i] * a.pairs + px * N;
                T in[2 * N], out[2 * N];
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    in[j] = x[i][j];
                    if (SECOND) in[V + j] = y[i][j];
                }
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const int lo = INTER ? 2 * j : j, hi = INTER ? 2 * j + 1 : V + j;
                    const float u = static_cast<float>(in[lo]), v = static_cast<float>(in[hi]);
                    const float2 w = cs[j];
                    out[lo] = static_cast<T>(__builtin_fmaf(u, w.x, -(v * w.y)));
                    out[hi] = static_cast<T>(__builtin_fmaf(u, w.y, v * w.x));
                }
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    x[i][j] = out[j];
                    if (SECOND) y[i][j] = out[V + j];
                }
                if (SECOND) put<PAST>(p + e1, y[i]);
            }
            put<PAST>(p + e0, x[i]);
        }
    }
}

template <int DT, int V>
hipError_t launch(const RotaryArgs& a, bool inter, bool past, dim3 grid, dim3 block, hipStream_t s)
{
    if (inter) return launch_kernel(past ? rotary_kernel<DT, V, true, true> : rotary_kernel<DT, V, true, false>, grid, block, s, a);
    return launch_kernel(past ? rotary_kernel<DT, V, false, true> : rotary_kernel<DT, V, false, false>, grid, block, s, a);
}

// False where [tokens, heads, d] with these strides may put two elements at one place.  (True only where one axis's steps enclose
// the other axis whole; strides that interleave without meeting are taken for such that meet.)
bool strides_fit(const int64_t* st, int64_t tokens, int64_t heads, int64_t d)
{
    const int64_t a = st[0] < 0 ? -st[0] : st[0], b = st[1] < 0 ? -st[1] : st[1];
    if (heads > 1 && b < d) return false;
    if (tokens > 1 && a < d) return false;
    if (tokens > 1 && heads > 1) return a >= b ? a >= (heads - 1) * b + d : b >= (tokens - 1) * a + d;
    return true;
}

}  // namespace

extern "C" {

int rotary_run(const void* q, const int64_t* q_strides, const void* k, const int64_t* k_strides, void* q_out, const int64_t* q_out_strides,
               void* k_out, const int64_t* k_out_strides, const int64_t* positions, const double* inv_freq, const uint8_t* pair_axis,
               int64_t tokens, int32_t q_heads, int32_t k_heads, int32_t d, int32_t rot, int32_t axes, int dtype, int flags, void* stream)
{
    if (dtype != ADDRMS_BF16 && dtype != ADDRMS_FP16 && dtype != ADDRMS_FP32)
        return fail(ADDRMS_ERR_UNSUPPORTED_DTYPE, "unsupported dtype %d for rotary positions", dtype);
    if (flags & ~(ROTARY_INTERLEAVED | ROTARY_INVERSE)) return fail(ADDRMS_ERR_INVALID_ARG, "unknown flags %d", flags);
    if (tokens < 0 || q_heads < 0 || k_heads < 0) return fail(ADDRMS_ERR_INVALID_ARG, "tokens and heads must be >= 0");
    if (d <= 0 || rot <= 0 || rot > d || rot % 2 != 0 || axes < 1 || axes > 255)
        return fail(ADDRMS_ERR_INVALID_ARG, "rot must be even, 2 <= rot <= d, and 1 <= axes <= 255 (got rot=%d d=%d axes=%d)", rot, d, axes);
    if (d > ROTARY_MAX_HEAD || tokens > (1ll << 31) - 1 || static_cast<int64_t>(q_heads) + k_heads > 65536)
        return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "d=%d, tokens=%lld or %lld heads are beyond the limits (%d, 2^31-1, 65536)", d, (long long)tokens,
                    (long long)q_heads + k_heads, ROTARY_MAX_HEAD);
    if (tokens == 0 || (q_heads == 0 && k_heads == 0)) return ADDRMS_OK;
    if ((q_heads && (!q || !q_out || !q_strides || !q_out_strides)) || (k_heads && (!k || !k_out || !k_strides || !k_out_strides)) || !positions ||
        !inv_freq || !pair_axis)
        return fail(ADDRMS_ERR_INVALID_ARG, "no pointer may be NULL");
    if ((q_heads && !strides_fit(q_out_strides, tokens, q_heads, d)) || (k_heads && !strides_fit(k_out_strides, tokens, k_heads, d)))
        return fail(ADDRMS_ERR_INVALID_ARG, "the strides of an output put two elements at one place");
    const int es = x_bytes(dtype);
    RotaryArgs a = {};
    a.q = addr(q), a.k = addr(k), a.q_out = addr(q_out), a.k_out = addr(k_out);
    a.positions = addr(positions), a.inv_freq = addr(inv_freq), a.pair_axis = addr(pair_axis);
    a.tokens = tokens;
    uint64_t bits = 0;                       // of everything that a piece of V elements must divide
    for (int i = 0; i < 2; ++i) {
        if (q_heads) a.qs[i] = q_strides[i], a.qos[i] = q_out_strides[i];
        if (k_heads) a.ks[i] = k_strides[i], a.kos[i] = k_out_strides[i];
        bits |= static_cast<uint64_t>(a.qs[i] | a.qos[i] | a.ks[i] | a.kos[i]) * es;
    }
    if (q_heads) bits |= a.q | a.q_out;
    if (k_heads) bits |= a.k | a.k_out;
    if (bits % es != 0 || !aligned_to(positions, 8) || !aligned_to(inv_freq, 8))
        return fail(ADDRMS_ERR_MISALIGNED, "tensors must be aligned to their element size");
    a.q_heads = q_heads, a.heads = q_heads + k_heads, a.pairs = rot / 2, a.axes = axes, a.sign = (flags & ROTARY_INVERSE) ? -1 : 1;
    const bool inter = flags & ROTARY_INTERLEAVED;
    bits |= static_cast<uint64_t>(a.pairs | (d - rot)) * es;
    // Pieces of 16 bytes where everything is a multiple of that, of 8 where it is of that, single elements else.
    const int v = bits % 16 == 0 ? 16 / es : bits % 8 == 0 && es == 2 ? 4 : 1;
    a.pair_pieces = inter && v > 1 ? 2 * a.pairs / v : a.pairs / v;
    a.pieces = a.pair_pieces + (d - rot) / v;
    // A workgroup is as many heads side by side as 256 threads hold; each thread has about kAhead pieces, of several tokens where
    // their heads alone do not give them.  Few tokens: one a workgroup, and their heads over several, until there are 2 workgroups a CU.
    const int ix = a.pieces, iy = kThreads / ix;                 // ix <= ROTARY_MAX_HEAD = kThreads
    const int64_t many = 512;
    int64_t per = (static_cast<int64_t>(iy) * kAhead + a.heads - 1) / a.heads;
    if (per > tokens / many) per = tokens / many;
    if (per > kMaxTurns / a.pairs) per = kMaxTurns / a.pairs;
    if (per < 1) per = 1;
    a.tokens_per_wg = static_cast<int32_t>(per);
    a.heads_per_wg = a.heads;
    const int64_t groups = (tokens + per - 1) / per;
    if (groups < many && a.heads > iy) a.heads_per_wg = iy;
    if (!launchable(groups, ix)) return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "%lld tokens of d=%d are too many for a launch", (long long)tokens, d);
    const dim3 grid(static_cast<unsigned>(groups), static_cast<unsigned>((a.heads + a.heads_per_wg - 1) / a.heads_per_wg)), block(ix, iy);
    // Large outputs go past the caches where every store fills its 16-byte pieces' lines: 8192 tokens x 40 heads x 128 bf16 26.7 us, not
    // 32.3, 2048 tokens 8.9 and 9.9, 1024 and 512 (5 MB) the same, 200 (2 MB) too.  What comes next then reads them from memory: with the
    // write of the keys into a cache behind it 8192 tokens take 42.6 and 43.9, 2048 13.8 and 14.8, 1024 10.1 and 11.2; with that and
    // attention, 2048 tokens 111.0 and 110.4.  A copy of all outputs loses more than was won: 8192 62.0 and 55.7, 2048 20.2 and 18.8.
    // Loads that go past the caches, too, gain 2 % at the largest and lose a quarter at the others.
    const bool past = v * es == 16 && tokens * a.heads * static_cast<int64_t>(d) * es >= kPastBytes;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    hipError_t e;
    if (dtype == ADDRMS_FP32) e = v == 4 ? launch<DT_FP32, 4>(a, inter, past, grid, block, s) : launch<DT_FP32, 1>(a, inter, past, grid, block, s);
    else if (dtype == ADDRMS_BF16)
        e = v == 8 ? launch<DT_BF16, 8>(a, inter, past, grid, block, s) : v == 4 ? launch<DT_BF16, 4>(a, inter, past, grid, block, s) : launch<DT_BF16, 1>(a, inter, past, grid, block, s);
    else
        e = v == 8 ? launch<DT_FP16, 8>(a, inter, past, grid, block, s) : v == 4 ? launch<DT_FP16, 4>(a, inter, past, grid, block, s) : launch<DT_FP16, 1>(a, inter, past, grid, block, s);
    if (e != hipSuccess) return fail(ADDRMS_ERR_HIP, "the launch failed: %s", hipGetErrorString(e));
    return ADDRMS_OK;
}

int64_t rotary_algorithmic_bytes(int64_t tokens, int32_t heads, int32_t d, int32_t axes, int dtype)
{
    if (dtype != ADDRMS_BF16 && dtype != ADDRMS_FP16 && dtype != ADDRMS_FP32)
        return fail(ADDRMS_ERR_UNSUPPORTED_DTYPE, "unsupported dtype %d for rotary positions", dtype);
    if (tokens < 0 || heads < 0 || d <= 0 || axes < 1) return fail(ADDRMS_ERR_INVALID_ARG, "sizes must not be negative");
    return tokens * (2ll * heads * d * x_bytes(dtype) + 8ll * axes);
}

}  // extern "C"
