// Penalties, biases and masks on logits, and the best token of each row (include/logits.h).
//
// A workgroup has a chunk of the vocabulary and some of a sequence's rows.  What the sequence's lists say of the chunk's tokens is
// gathered in LDS once, a word a token; then the rows pass by, each logit read once and written once.  Few tokens are named by a list:
// the others stay what they are but for the mask, without arithmetic, and the named ones are taken one by one by the thread that has them.
// Bound by memory where rows are many: 8 x 24 x 131072 bf16 without lists 20.6 us a call, with out alone 15.7 (6.6 TB/s); lists of up to 16384
// tokens take 12 more, most of it the named tokens (some hundreds of a chunk's), whose places and division are some 60 instructions a turn.
// Small calls are bound by fetching code: 1 x 32000 bf16 took 11.4 us with 24 KB of it and takes 7.8 with 8.
#include <algorithm>

#include "logits.h"
#include "serving_internal.h"

using namespace addrms_host;
using namespace serving;

namespace {

constexpr int kThreads = 256, kLongThreads = 512, kManyThreads = 1024;
constexpr int32_t kLongHistory = 8192;        // tokens
constexpr uint32_t kEach = 32;                // tokens of a thread: a bit each
// A token's word: whether the prompt has it, the first bias that names it (counted down from 1023), how often it was made.
constexpr uint32_t kMet = 1u << 31, kMade = (1u << 21) - 1, kBias = LOGITS_MAX_BIASES << 21;
static_assert(LOGITS_MAX_HISTORY + TREE_MAX_NODES <= kMade, "a count fits its bits");

struct LogitsArgs {
    addr_t logits, out, best, history, history_lens, prompt_lens, penalties, bias_tokens, bias_values, allowed, tree_tokens, tree_masks, partial;
    int64_t logits_stride, out_stride, history_stride, allowed_stride;
    uint32_t vocab, nodes, chunks, parts, part_rows, biases, history_width, rows, partials;        // of a row
};

// 16 bytes at any element's address.
template <int DT> struct Vec {
    typedef typename elem<DT>::type T;
    static constexpr int N = 16 / sizeof(T);
    typedef T type __attribute__((ext_vector_type(N)));
    typedef T loose __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

// Numbers in their order as whole numbers above 0, -0 as 0, NaN the largest.
__device__ __forceinline__ uint32_t order_of(float z)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, z + 0.0f);
    return z != z ? ~0u : u ^ (u >> 31 ? ~0u : 1u << 31);
}
// The largest of a wave's lanes, in all of them.
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t x) { return static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(x), CTRL, 0xf, 0xf, true)); }
__device__ __forceinline__ uint32_t most_of_wave(uint32_t x)
{
    x = max(x, moved<0xB1>(x));                                 // quad_perm 1,0,3,2
    x = max(x, moved<0x4E>(x));                                 // quad_perm 2,3,0,1
    x = max(x, moved<0x141>(x));                                // row_half_mirror
    x = max(x, moved<0x140>(x));                                // row_mirror
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    const uint32_t a = r[0], b = r[1];
    x = max(a, b);
    const auto h = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    const uint32_t c = h[0], d = h[1];
    return max(c, d);
}
// A number's order and its token, counted down: of equal numbers the lower token is more.
struct Best {
    uint32_t order, down;
    __device__ __forceinline__ void take(uint32_t o, uint32_t d)
    {
        const bool more = o > order || (o == order && d > down);
        order = more ? o : order;
        down = more ? d : down;
    }
    __device__ __forceinline__ Best of_wave() const
    {
        const uint32_t o = most_of_wave(order);
        return Best{o, most_of_wave(order == o ? down : 0)};
    }
};

// A bit as 32 of them.
__device__ __forceinline__ uint32_t spread(uint32_t bits, uint32_t at) { return static_cast<uint32_t>(static_cast<int32_t>(bits << (31 - at)) >> 31); }

// LISTS: there are penalties or biases.  Thread i's tokens are the pieces of N tokens i, i + THREADS, ... of the chunk; 32 bits, in
// that order, say something of each.  Code is kept short by loops: a small call's time is that of fetching it.
template <int DT, bool LISTS, int THREADS>
__global__ __launch_bounds__(THREADS) void logits_kernel(LogitsArgs a)
{
    typedef Vec<DT> V;
    typedef typename V::T T;
    constexpr uint32_t N = V::N, CHUNK = kEach * THREADS, PIECES = kEach / N, NAMED = (LOGITS_MAX_BIASES + THREADS - 1) / THREADS, BATCH = THREADS < kManyThreads ? 16 : 4, WAVES = THREADS / 64;
    constexpr uint32_t kPiece = (1u << N) - 1;
    // Which tokens are named is seen from their words where a workgroup takes in long lists (8 x 24 x 131072 34.6 us, so 33.6), else noted
    // with each (1 x 32000 8.6 us, so 8.0).
    constexpr bool BUILD = THREADS < kManyThreads;
    constexpr bool AHEAD = DT != DT_FP32;                       // the next row is under way; two of fp32 would leave fewer waves on a CU
    __shared__ __attribute__((aligned(16))) uint32_t words[LISTS ? CHUNK : 4];
    __shared__ float sums[LISTS ? LOGITS_MAX_BIASES : 1];
    __shared__ uint32_t named_in[LISTS ? THREADS : 1];          // of each thread's tokens those that a list names
    __shared__ uint32_t twice;
    __shared__ Best most[WAVES];
    const uint32_t tid = threadIdx.x, chunk = blockIdx.x % a.chunks, rest = blockIdx.x / a.chunks, part = rest % a.parts, seq = rest / a.parts;
    const uint32_t v0 = chunk * CHUNK, n = min(CHUNK, a.vocab - v0);
    const uint32_t first = part * a.part_rows, last = min(first + a.part_rows, a.nodes);
    // this thread's tokens in whole pieces, and those of a last piece that is not whole, which are taken one by one
    uint32_t have = 0, edge = 0;
#pragma unroll
    for (uint32_t k = 0; k < PIECES; ++k) {
        const uint32_t e = N * (tid + k * THREADS);
        have |= e + N <= n ? kPiece << (N * k) : 0;
        edge |= e < n && e + N > n ? ((1u << (n - e)) - 1) << (N * k) : 0;
    }
    const auto token_of = [&](uint32_t bit) { return N * (tid + bit / N * THREADS) + bit % N; };

    struct Row {
        typename V::type x[PIECES];
        uint32_t word[PIECES];                                  // the mask's, of each piece
    };
    // Nothing here looks at what it loads: it may be under way for long.
    const auto load = [&](Row& to, uint32_t i) {
        const uint32_t row = seq * a.nodes + i;
        if (n >= N) {
            const T* x = at_global<const T>(a.logits) + row * a.logits_stride + v0;
#pragma unroll
            for (uint32_t k = 0; k < PIECES; ++k) {
                const uint32_t e = N * (tid + k * THREADS);
                to.x[k] = *reinterpret_cast<const typename V::loose*>(x + (e + N <= n ? e : 0));
            }
        }
        if (a.allowed) {
            const uint32_t* allowed = at_global<const uint32_t>(a.allowed) + row * a.allowed_stride + v0 / 32;
#pragma unroll
            for (uint32_t k = 0; k < PIECES; ++k) to.word[k] = allowed[min(N * (tid + k * THREADS), n - 1) / 32];
        }
    };

    Row now, next;
    if constexpr (!LISTS) load(now, first);
    float r = 1.0f, f = 0.0f, p = 0.0f;
    int32_t node_token = -1;
    const bool tree = LISTS && a.tree_masks && a.penalties;
    const auto name = [&](uint32_t t) { atomicOr(named_in + t / N % THREADS, 1u << (t / (N * THREADS) * N + t % N)); };
    if constexpr (LISTS) {
        // What the lists say is asked for at once, then taken in: a history's first tokens before its length is known.
        const int32_t* const h = at_global<const int32_t>(a.history) + seq * a.history_stride;
        int32_t batch[BATCH], len = 0, prompt = 0, named[NAMED];
        float values[NAMED];
        const auto ask = [&](uint32_t from) {
#pragma unroll
            for (uint32_t k = 0; k < BATCH; ++k) batch[k] = h[min(from + tid + k * THREADS, a.history_width - 1)];
        };
        if (a.history) {
            ask(0);
            len = at_global<const int32_t>(a.history_lens)[seq];
            if (a.prompt_lens) prompt = at_global<const int32_t>(a.prompt_lens)[seq];
        }
#pragma unroll
        for (uint32_t k = 0; k < NAMED; ++k) {
            const uint32_t i = tid + k * THREADS;
            named[k] = -1;
            if (i < a.biases) {
                named[k] = at_global<const int32_t>(a.bias_tokens)[static_cast<int64_t>(seq) * a.biases + i];
                values[k] = at_global<const float>(a.bias_values)[static_cast<int64_t>(seq) * a.biases + i];
            }
        }
        if (a.penalties) {
            const float* pen = at_global<const float>(a.penalties) + 3 * static_cast<int64_t>(seq);
            r = pen[0], f = pen[1], p = pen[2];
        }
        if (a.tree_masks && tid < a.nodes) node_token = at_global<const int32_t>(a.tree_tokens)[seq * a.nodes + tid];
        load(now, first);                                       // loads come back in their order: while these do, the lists are taken in
#pragma unroll
        for (uint32_t i = 4 * tid; i < CHUNK; i += 4 * THREADS) *reinterpret_cast<u32x4*>(words + i) = u32x4{0, 0, 0, 0};
        if constexpr (!BUILD) named_in[tid] = 0;
        if (tid == 0) twice = 0;
        __syncthreads();
        if (a.history) {
            len = min(max(len, 0), static_cast<int32_t>(a.history_width));
            prompt = min(max(prompt, 0), len);
            const auto take = [&](int32_t from) {               // the batch from here on, while the next one is under way
                int32_t here[BATCH];
#pragma unroll
                for (uint32_t k = 0; k < BATCH; ++k) here[k] = batch[k];
                if (from + static_cast<int32_t>(BATCH * THREADS) < len) ask(static_cast<uint32_t>(from) + BATCH * THREADS);
#pragma unroll
                for (uint32_t k = 0; k < BATCH; ++k) {
                    const int32_t i = from + static_cast<int32_t>(tid + k * THREADS);
                    const uint32_t t = static_cast<uint32_t>(here[k]) - v0;
                    if (t < n && i < len) {
                        if (i < prompt) atomicOr(words + t, kMet);
                        else atomicAdd(words + t, 1u);
                        if constexpr (!BUILD) name(t);
                    }
                }
            };
            take(0);                                            // apart, so that it waits for its own loads and not for the row's behind them
#pragma unroll 1
            for (int32_t from = BATCH * THREADS; from < len; from += BATCH * THREADS) take(from);
        }
        if (a.biases) {
            __syncthreads();
            const auto mark = [&](uint32_t k) { return (LOGITS_MAX_BIASES - (tid + k * THREADS)) << 21; };
#pragma unroll
            for (uint32_t k = 0; k < NAMED; ++k) {
                const uint32_t t = static_cast<uint32_t>(named[k]) - v0;
                // the word's other bits do not change here
                if (t < n) {
                    atomicMax(words + t, (words[t] & ~kBias) | mark(k));
                    if constexpr (!BUILD) name(t);
                }
            }
            __syncthreads();
#pragma unroll
            for (uint32_t k = 0; k < NAMED; ++k) {
                const uint32_t t = static_cast<uint32_t>(named[k]) - v0;
                if (t < n) {
                    if ((words[t] & kBias) == mark(k)) sums[tid + k * THREADS] = values[k];
                    else twice = 1;
                }
            }
            __syncthreads();
            if (twice) {                                        // sums in the list's order, by the first that names a token
                const int32_t* tokens = at_global<const int32_t>(a.bias_tokens) + static_cast<int64_t>(seq) * a.biases;
#pragma unroll 1
                for (uint32_t k = 0; k < NAMED; ++k) {
                    const uint32_t i = tid + k * THREADS, t = i < a.biases ? static_cast<uint32_t>(tokens[i]) - v0 : n;
                    if (t >= n || (words[t] & kBias) != mark(k)) continue;
                    float sum = sums[i];
                    for (uint32_t j = i + 1; j < a.biases; ++j)
                        if (tokens[j] == tokens[i]) sum += at_global<const float>(a.bias_values)[static_cast<int64_t>(seq) * a.biases + j];
                    sums[i] = sum;
                }
            }
        }
        __syncthreads();
        if constexpr (BUILD) {
            uint32_t named_here = 0;
#pragma unroll
            for (uint32_t k = 0; k < PIECES; ++k)
#pragma unroll
                for (uint32_t j = 0; j < N; ++j) named_here |= words[N * (tid + k * THREADS) + j] ? 1u << (N * k + j) : 0;
            named_in[tid] = named_here;
            if (tree) __syncthreads();                          // paths name more
        }
    }
    // Of a tree's row the path's tokens are counted in, and those of the row before that are not on it, out: a thread has a node.
    uint64_t on_path = 0, path = tree ? at_global<const uint64_t>(a.tree_masks)[seq * a.nodes + first] : 0;
#pragma unroll 1
    for (uint32_t i = first; i < last; ++i) {
        const uint32_t row = seq * a.nodes + i;
        uint32_t bits = ~0u;                                    // tokens that the grammar allows
        if (a.allowed) {
            bits = 0;
#pragma unroll
            for (uint32_t k = 0; k < PIECES; ++k) bits |= __builtin_amdgcn_ubfe(now.word[k], N * tid % 32, N) << (N * k);        // N * THREADS is a multiple of 32
        }
        if constexpr (LISTS)
            if (tree) {
                const uint32_t t = static_cast<uint32_t>(node_token) - v0;
                if (tid < a.nodes && t < n && ((path ^ on_path) >> tid & 1)) {
                    atomicAdd(words + t, path >> tid & 1 ? 1u : ~0u);
                    name(t);
                }
                __syncthreads();
                on_path = path;
            }
        if (AHEAD && i + 1 < last) load(next, i + 1);
        if (tree && i + 1 < last) path = at_global<const uint64_t>(a.tree_masks)[row + 1];
        T* const y = at_global<T>(a.out) + row * a.out_stride + v0;
        uint32_t left = edge;                                   // tokens that are taken one by one
        if constexpr (LISTS) left |= named_in[tid] & bits & have;
        const uint32_t same = bits & have & ~left;          // tokens that stay what they are
        float top = -__builtin_huge_valf();
        uint32_t piece = 0;                                     // that the best so far is in
#pragma unroll
        for (uint32_t k = 0; k < PIECES; ++k) {
            const uint32_t e = N * (tid + k * THREADS);
            if (a.best) {
                float most_here = -__builtin_huge_valf();
#pragma unroll
                for (uint32_t j = 0; j < N; ++j) {
                    const uint32_t in = spread(same, N * k + j);
                    const uint32_t z = (__builtin_bit_cast(uint32_t, static_cast<float>(now.x[k][j])) & in) | (0xff800000u & ~in);
                    most_here = __builtin_elementwise_maximum(most_here, __builtin_bit_cast(float, z));
                }
                if (!(most_here <= top) && top == top) top = most_here, piece = k;
            }
            if (a.out && e + N <= n) {
                u32x4 kept = __builtin_bit_cast(u32x4, now.x[k]);
                if (a.allowed)
#pragma unroll
                    for (uint32_t w = 0; w < 4; ++w) {
                        // -infinity in the place of what is ruled out
                        const uint32_t in = N == 4 ? spread(bits, N * k + w)
                                                   : (spread(bits, N * k + 2 * w) & 0xffffu) | (spread(bits, N * k + 2 * w + 1) & 0xffff0000u);
                        constexpr uint32_t low = DT == DT_FP32 ? 0xff800000u : DT == DT_BF16 ? 0xff80ff80u : 0xfc00fc00u;
                        kept[w] = (kept[w] & in) | (low & ~in);
                    }
                *reinterpret_cast<typename V::loose*>(y + e) = __builtin_bit_cast(typename V::type, kept);
            }
        }
        const auto piece_of = [&](uint32_t which) {
            u32x4 x = __builtin_bit_cast(u32x4, now.x[0]);
#pragma unroll
            for (uint32_t k = 1; k < PIECES; ++k)
#pragma unroll
                for (uint32_t w = 0; w < 4; ++w) x[w] = which == k ? __builtin_bit_cast(u32x4, now.x[k])[w] : x[w];
            return x;
        };
        // The best of those that stay: only in the lanes that have the wave's.
        Best mine = {0, 0};
        if (a.best) {
            mine.order = have ? order_of(top) : 0;
            if (mine.order == most_of_wave(mine.order)) {
                const typename V::type x = __builtin_bit_cast(typename V::type, piece_of(piece));
                uint32_t e = 0;
#pragma unroll
                for (uint32_t j = N; j-- > 0;)
                    if ((same >> (N * piece + j) & 1) && order_of(static_cast<float>(x[j])) == mine.order) e = j;
                if (top == -__builtin_huge_valf()) e = 0;       // nothing is above what is ruled out: the first, also where it is that
                mine.down = ~(v0 + N * (tid + piece * THREADS) + e);
            }
        }
        // A wave takes as many turns as one of its lanes has tokens, few of 32.
#pragma unroll 1
        for (; left; left &= left - 1) {
            const uint32_t b = static_cast<uint32_t>(__builtin_ctz(left)), e = token_of(b), j = b % N;
            const u32x4 x = piece_of(b / N);
            const uint32_t at = N == 4 ? j : j / 2, lo = at & 1 ? x[1] : x[0], hi = at & 1 ? x[3] : x[2], word = at & 2 ? hi : lo;
            float z;
            if constexpr (DT == DT_FP32) z = __builtin_bit_cast(float, word);
            else z = static_cast<float>(__builtin_bit_cast(T, static_cast<uint16_t>(j & 1 ? word >> 16 : word)));
            if (edge >> b & 1) z = bits >> b & 1 ? static_cast<float>((at_global<const T>(a.logits) + row * a.logits_stride + v0)[e]) : -__builtin_huge_valf();
            if constexpr (LISTS) {
                const uint32_t w = words[e];
                if (w & (kMet | kMade)) z = z > 0.0f ? z / r : z * r;
                if (w & kMade) {
                    z = z - f * static_cast<float>(w & kMade);
                    z = z - p;
                }
                if (w & kBias) z = z + sums[LOGITS_MAX_BIASES - ((w & kBias) >> 21)];
                if (!(bits >> b & 1)) z = -__builtin_huge_valf();
            }
            mine.take(order_of(z), ~(v0 + e));
            if (a.out) y[e] = static_cast<T>(z);
        }
        if (a.best) {
            const Best wave = mine.of_wave();
            if (a.chunks > 1) {
                if (tid % 64 == 0) at_global<Best>(a.partial)[static_cast<int64_t>(row) * a.partials + chunk * WAVES + tid / 64] = wave;
            } else {
                if (tid % 64 == 0) most[tid / 64] = wave;
                __syncthreads();
                if (tid < 64) {
                    const Best all = (tid < WAVES ? most[tid] : Best{0, 0}).of_wave();
                    if (tid == 0) at_global<uint32_t>(a.best)[row] = ~all.down;
                }
                __syncthreads();
            }
        }
        if (tree) __syncthreads();
        if constexpr (AHEAD) now = next;
        else if (i + 1 < last) load(now, i + 1);
    }
}

// The best of a row's chunks: a wave a row.
__global__ __launch_bounds__(kThreads) void best_kernel(LogitsArgs a)
{
    const uint32_t row = blockIdx.x * (kThreads / 64) + threadIdx.x / 64, lane = threadIdx.x % 64;
    if (row >= a.rows) return;
    Best mine = {0, 0};
    for (uint32_t c = lane; c < a.partials; c += 64) {
        const Best o = at_global<const Best>(a.partial)[static_cast<int64_t>(row) * a.partials + c];
        mine.take(o.order, o.down);
    }
    mine = mine.of_wave();
    if (lane == 0) at_global<uint32_t>(a.best)[row] = ~mine.down;
}

int check(int64_t batch, int32_t nodes, int64_t vocab, int dtype)
{
    if (dtype != ADDRMS_BF16 && dtype != ADDRMS_FP16 && dtype != ADDRMS_FP32) return fail(ADDRMS_ERR_UNSUPPORTED_DTYPE, "unsupported dtype %d for logits", dtype);
    if (batch < 0 || nodes < 0 || vocab <= 0) return fail(ADDRMS_ERR_INVALID_ARG, "batch and nodes must be >= 0, vocab > 0");
    if (batch >= (1 << 24) || nodes > 65536 || batch * nodes >= (1 << 24) || vocab > (1 << 24))
        return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "%lld sequences of %d rows, or %lld tokens, are beyond the limits (2^24 rows, 2^24 tokens)", (long long)batch, nodes,
                    (long long)vocab);
    return ADDRMS_OK;
}
// Threads of a workgroup, and so its tokens: all of a row where 1024 threads can have them, which then need no second launch for the best
// (1 x 32000 bf16 7.8 us, with 256 threads 8.8; 256 x 32000 10.9 and 14.4; 32 x 16 nodes x 32000 18.4 and 20.1).  Of longer rows they have
// a quarter as many lists to go over, but come one a CU: 8 x 24 nodes x 131072 with histories of up to 16384 31.3 us in place of 33.3, but 8
// x 40000 10.0 in place of 9.1, 256 x 50001 23.7 in place of 22.5, 8 x 24 x 100000 fp32 38.2 in place of 33.4, 16 x 8 x 152000 22.9 and 19.5.
// Of the others, long histories are gone over half as often by 512 threads (8 x 24 x 131072 with up to 16384 32.4 us in place of 33.3, 1 x 64 nodes x
// 50001 with 30000 18.4 and 23.1), short ones are not worth it (256 x 50001 24.9 in place of 22.4).
// Rows of up to 16384 tokens have threads enough in 512 or 256, of which more come on a CU: 58 x 11 x 8000 bf16 9.3 us with 256, 13.2 with 512, 15.8 with
// 1024, 100 x 3 x 2900 9.3, 10.7 and 14.8, 58 x 11 x 16000 15.1 with 512 and 17.4 with 1024, 54 x 8000 with histories of up to 19500 19.0, 14.4 and 14.9,
// 1 x 8000 8.1, 7.3 and 8.1.  Where 1024 for each row find room at once, short rows are no faster with fewer (1 x 2900 7.9, 7.7 and 6.9).
int threads_of(int64_t rows, int64_t vocab, int32_t history)
{
    const bool many = rows > 256;
    if (vocab <= kEach * kThreads && many && history < kLongHistory) return kThreads;
    if (vocab <= kEach * kLongThreads && (vocab > 4096 || many)) return kLongThreads;
    return vocab <= kEach * kManyThreads ? kManyThreads : history >= kLongHistory ? kLongThreads : kThreads;
}
int64_t chunks_of(int64_t vocab, int threads) { return (vocab + kEach * threads - 1) / (kEach * threads); }
// Partial results of a row: one of each wave, none where one workgroup has the row.
int64_t partials_of(int64_t vocab, int threads) { return chunks_of(vocab, threads) > 1 ? chunks_of(vocab, threads) * (threads / 64) : 0; }

}  // namespace

extern "C" {

int64_t logits_workspace_bytes(int64_t batch, int32_t nodes, int64_t vocab, int dtype)
{
    if (const int st = check(batch, nodes, vocab, dtype)) return st;
    return vocab <= kEach * kManyThreads ? 0 : 8 * batch * nodes * std::max(partials_of(vocab, kThreads), partials_of(vocab, kLongThreads));
}

int64_t logits_algorithmic_bytes(int64_t batch, int32_t nodes, int64_t vocab, int dtype, int64_t tokens, int32_t biases, int masked, int write)
{
    if (const int st = check(batch, nodes, vocab, dtype)) return st;
    if (tokens < 0 || biases < 0) return fail(ADDRMS_ERR_INVALID_ARG, "tokens and biases must be >= 0");
    const int64_t rows = batch * nodes;
    return rows * vocab * (dtype == ADDRMS_FP32 ? 4 : 2) * (write ? 2 : 1) + (masked ? rows * ((vocab + 31) / 32) * 4 : 0) + 4 * tokens + batch * biases * 8ll + 4 * rows;
}

int logits_run(const void* logits, int64_t logits_stride, void* out, int64_t out_stride, int32_t* best, int64_t batch, int32_t nodes, int64_t vocab, int dtype,
               const logits_lists* lists, void* workspace, int64_t workspace_bytes, void* stream)
{
    if (const int st = check(batch, nodes, vocab, dtype)) return st;
    if (!lists) return fail(ADDRMS_ERR_INVALID_ARG, "lists is NULL");
    const logits_lists& l = *lists;
    if (l.history_width < 0 || l.history_width > LOGITS_MAX_HISTORY || l.biases < 0 || l.biases > LOGITS_MAX_BIASES)
        return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "histories of %d tokens or %d biases are beyond the limits (%d, %d)", l.history_width, l.biases, LOGITS_MAX_HISTORY,
                    LOGITS_MAX_BIASES);
    if (l.tree_masks && nodes > TREE_MAX_NODES) return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "a tree of %d nodes is beyond the limit (%d)", nodes, TREE_MAX_NODES);
    if (batch == 0 || nodes == 0) return ADDRMS_OK;
    const int64_t need = best ? logits_workspace_bytes(batch, nodes, vocab, dtype) : 0;
    if (!logits || (l.history && l.history_width && !l.history_lens) || (l.biases && (!l.bias_tokens || !l.bias_values)) || (need && !workspace))
        return fail(ADDRMS_ERR_INVALID_ARG, "no pointer may be NULL");
    if ((l.tree_tokens == nullptr) != (l.tree_masks == nullptr)) return fail(ADDRMS_ERR_INVALID_ARG, "tree_tokens and tree_masks are given together");
    if (workspace_bytes < need)
        return fail(ADDRMS_ERR_INVALID_ARG, "the workspace has %lld bytes, the call needs %lld", (long long)workspace_bytes, (long long)need);
    const uintptr_t es = dtype == ADDRMS_FP32 ? 4 : 2;
    if (!aligned_to(logits, es) || !aligned_to(out, es) || !aligned_to(best, 4) || !aligned_to(l.history, 4) || !aligned_to(l.history_lens, 4) ||
        !aligned_to(l.prompt_lens, 4) || !aligned_to(l.penalties, 4) || !aligned_to(l.bias_tokens, 4) || !aligned_to(l.bias_values, 4) ||
        !aligned_to(l.allowed, 4) || !aligned_to(l.tree_tokens, 4) || !aligned_to(l.tree_masks, 8) || !aligned_to(workspace, 8))
        return fail(ADDRMS_ERR_MISALIGNED, "arrays must be aligned to their elements, the workspace to 8 bytes");
    if (out && out_stride < vocab && batch * nodes > 1) return fail(ADDRMS_ERR_INVALID_ARG, "rows of out overlap: %lld elements apart", (long long)out_stride);
    if (out == logits && out_stride != logits_stride && batch * nodes > 1)
        return fail(ADDRMS_ERR_INVALID_ARG, "out is logits with another stride");
    if (!out && !best) return ADDRMS_OK;
    LogitsArgs a = {};
    a.logits = addr(logits), a.out = addr(out), a.best = addr(best), a.penalties = addr(l.penalties);
    a.history = l.penalties && l.history_width ? addr(l.history) : 0, a.history_lens = addr(l.history_lens), a.prompt_lens = addr(l.prompt_lens);
    a.bias_tokens = addr(l.bias_tokens), a.bias_values = addr(l.bias_values), a.allowed = addr(l.allowed);
    a.tree_tokens = addr(l.tree_tokens), a.tree_masks = addr(l.tree_masks), a.partial = addr(workspace);
    a.logits_stride = logits_stride, a.out_stride = out_stride, a.history_stride = l.history_stride, a.allowed_stride = l.allowed_stride;
    a.vocab = static_cast<uint32_t>(vocab), a.nodes = static_cast<uint32_t>(nodes), a.rows = static_cast<uint32_t>(batch * nodes);
    a.biases = static_cast<uint32_t>(l.biases), a.history_width = static_cast<uint32_t>(l.history_width);
    const int threads = threads_of(batch * nodes, vocab, a.history ? l.history_width : 0);
    a.chunks = static_cast<uint32_t>(chunks_of(vocab, threads));
    a.partials = static_cast<uint32_t>(partials_of(vocab, threads));
    const bool used = l.biases || (l.penalties && (a.history || l.tree_masks));
    // A tree's rows are shared out until the chip is full twice over, or with one workgroup a CU full; each share takes in the lists anew (8
    // x 24 nodes x 131072 with 256 threads: 52.6 us with 256 workgroups, 35.8 with 512, 33.3 with 1024, 36.7 with 2048).
    const int64_t wanted = threads == kThreads ? 1024 : threads == kLongThreads ? 512 : 256, units = a.chunks * batch;
    int64_t parts = used ? std::max<int64_t>(1, wanted / units) : nodes;
    if (parts > nodes) parts = nodes;
    a.part_rows = static_cast<uint32_t>((nodes + parts - 1) / parts);
    a.parts = static_cast<uint32_t>((nodes + a.part_rows - 1) / a.part_rows);
    if (!launchable(units * a.parts, threads)) return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "the call is too large: %lld workgroups", (long long)(units * a.parts));
    const dim3 grid(static_cast<unsigned>(units * a.parts));
    const hipStream_t s = static_cast<hipStream_t>(stream);
#define AS(DT, T) launch_kernel(used ? logits_kernel<DT, true, T> : logits_kernel<DT, false, T>, grid, dim3(threads), s, a)
#define GO(DT) (threads == kThreads ? AS(DT, kThreads) : threads == kLongThreads ? AS(DT, kLongThreads) : AS(DT, kManyThreads))
    SERVING_HIP_TRY(dtype == ADDRMS_BF16 ? GO(DT_BF16) : dtype == ADDRMS_FP16 ? GO(DT_FP16) : GO(DT_FP32));
#undef GO
#undef AS
    if (best && a.chunks > 1)
        SERVING_HIP_TRY(launch_kernel(best_kernel, dim3(static_cast<unsigned>((a.rows + kThreads / 64 - 1) / (kThreads / 64))), dim3(kThreads), s, a));
    return ADDRMS_OK;
}

}  // extern "C"
