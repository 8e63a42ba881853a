// Penalties, biases and masks on logits, and the best token of each row (include/logits.h).
//
// A workgroup has a chunk of the vocabulary and some of a sequence's rows.  What the sequence's lists say of the chunk's tokens is
// gathered in LDS once, a word a token; then the rows pass by, each logit read once and written once.
#include "logits.h"
#include "serving_internal.h"

using namespace addrms_host;
using namespace serving;

namespace {

constexpr int kThreads = 256;
constexpr uint32_t kChunk = 8192;
// A token's word: whether the prompt has it, the first bias that names it (counted down from 1023), how often it was made.
constexpr uint32_t kMet = 1u << 31, kMade = (1u << 21) - 1, kBias = LOGITS_MAX_BIASES << 21;
static_assert(LOGITS_MAX_HISTORY + TREE_MAX_NODES <= kMade, "a count fits its bits");

struct LogitsArgs {
    addr_t logits, out, best, history, history_lens, prompt_lens, penalties, bias_tokens, bias_values, allowed, tree_tokens, tree_masks, partial;
    int64_t logits_stride, out_stride, history_stride, allowed_stride;
    uint32_t vocab, nodes, chunks, parts, part_rows, biases, history_width, rows;
};

// 16 bytes at any element's address.
template <int DT> struct Vec {
    typedef typename elem<DT>::type T;
    static constexpr int N = 16 / sizeof(T);
    typedef T type __attribute__((ext_vector_type(N)));
    typedef T loose __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

// Larger numbers have larger keys, NaN the largest; of equal ones the lower token.
__device__ __forceinline__ uint64_t key_of(float z, uint32_t token)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, z + 0.0f);               // -0 counts as 0
    const uint32_t order = z != z ? ~0u : u ^ (u >> 31 ? ~0u : 1u << 31);
    return static_cast<uint64_t>(order) << 32 | ~token;
}
__device__ __forceinline__ uint64_t most_of_wave(uint64_t k)
{
#pragma unroll
    for (int x = 32; x; x >>= 1) {
        const uint64_t o = __shfl_xor(static_cast<unsigned long long>(k), x);
        k = o > k ? o : k;
    }
    return k;
}

// LISTS: there are penalties or biases.
template <int DT, bool LISTS>
__global__ __launch_bounds__(kThreads) void logits_kernel(LogitsArgs a)
{
    typedef Vec<DT> V;
    typedef typename V::T T;
    constexpr uint32_t N = V::N;
    __shared__ __attribute__((aligned(16))) uint32_t words[LISTS ? kChunk : 4];
    __shared__ float sums[LISTS ? LOGITS_MAX_BIASES : 1];
    __shared__ uint32_t twice;
    __shared__ uint64_t most[kThreads / 64];
    const uint32_t tid = threadIdx.x, chunk = blockIdx.x % a.chunks, rest = blockIdx.x / a.chunks, part = rest % a.parts, seq = rest / a.parts;
    const uint32_t v0 = chunk * kChunk, n = min(kChunk, a.vocab - v0);
    float r = 1.0f, f = 0.0f, p = 0.0f;
    if constexpr (LISTS) {
        for (uint32_t i = 4 * tid; i < kChunk; i += 4 * kThreads) *reinterpret_cast<u32x4*>(words + i) = u32x4{0, 0, 0, 0};
        if (tid == 0) twice = 0;
        __syncthreads();
        if (a.penalties) {
            const float* pen = at_global<const float>(a.penalties) + 3 * static_cast<int64_t>(seq);
            r = pen[0], f = pen[1], p = pen[2];
            if (a.history) {
                const int32_t len = min(max(at_global<const int32_t>(a.history_lens)[seq], 0), static_cast<int32_t>(a.history_width));
                const int32_t prompt = a.prompt_lens ? min(max(at_global<const int32_t>(a.prompt_lens)[seq], 0), len) : 0;
                const int32_t* h = at_global<const int32_t>(a.history) + seq * a.history_stride;
#pragma unroll 8
                for (int32_t i = static_cast<int32_t>(tid); i < len; i += kThreads) {
                    const uint32_t t = static_cast<uint32_t>(h[i]) - v0;
                    if (t < n) {
                        if (i < prompt) atomicOr(words + t, kMet);
                        else atomicAdd(words + t, 1u);
                    }
                }
            }
        }
        if (a.biases) {
            __syncthreads();
            const int32_t* tokens = at_global<const int32_t>(a.bias_tokens) + static_cast<int64_t>(seq) * a.biases;
            const float* values = at_global<const float>(a.bias_values) + static_cast<int64_t>(seq) * a.biases;
            for (uint32_t i = tid; i < a.biases; i += kThreads) {
                const uint32_t t = static_cast<uint32_t>(tokens[i]) - v0;
                // the word's other bits do not change here
                if (t < n) atomicMax(words + t, (words[t] & ~kBias) | (LOGITS_MAX_BIASES - i) << 21);
            }
            __syncthreads();
            for (uint32_t i = tid; i < a.biases; i += kThreads) {
                const uint32_t t = static_cast<uint32_t>(tokens[i]) - v0;
                if (t < n && (words[t] & kBias) >> 21 != LOGITS_MAX_BIASES - i) twice = 1;
            }
            __syncthreads();
            for (uint32_t i = tid; i < a.biases; i += kThreads) {
                const int32_t token = tokens[i];
                const uint32_t t = static_cast<uint32_t>(token) - v0;
                if (t >= n || (words[t] & kBias) >> 21 != LOGITS_MAX_BIASES - i) continue;
                float sum = values[i];
                if (twice)
                    for (uint32_t j = i + 1; j < a.biases; ++j)
                        if (tokens[j] == token) sum += values[j];
                sums[i] = sum;
            }
        }
        __syncthreads();
    }
    const auto adjusted = [&](float z, uint32_t w) {
        if (w & (kMet | kMade)) {
            z = z > 0.0f ? z / r : z * r;
            if (w & kMade) {
                z = z - f * static_cast<float>(w & kMade);
                z = z - p;
            }
        }
        if (w & kBias) z = z + sums[LOGITS_MAX_BIASES - ((w & kBias) >> 21)];
        return z;
    };
    // the path's tokens, counted in before a row and out again behind it
    const auto path = [&](uint32_t row, uint32_t by) {
        const uint64_t mask = at_global<const uint64_t>(a.tree_masks)[row];
        if (tid < a.nodes && (mask >> tid & 1)) {
            const uint32_t t = static_cast<uint32_t>(at_global<const int32_t>(a.tree_tokens)[seq * a.nodes + tid]) - v0;
            if (t < n) atomicAdd(words + t, by);
        }
        __syncthreads();
    };
    const bool tree = LISTS && a.tree_masks && a.penalties;
    for (uint32_t i = part * a.part_rows; i < min((part + 1) * a.part_rows, a.nodes); ++i) {
        const uint32_t row = seq * a.nodes + i;
        if constexpr (LISTS)
            if (tree) path(row, 1u);
        const T* x = at_global<const T>(a.logits) + row * a.logits_stride + v0;
        T* y = at_global<T>(a.out) + row * a.out_stride + v0;
        const uint32_t* allowed = at_global<const uint32_t>(a.allowed) + row * a.allowed_stride + v0 / 32;
        float top = -__builtin_huge_valf();
        uint32_t at = N * tid;                                  // of the best so far, at first the first of this thread's
        for (uint32_t e = N * tid; e < n; e += N * kThreads) {
            const bool whole = e + N <= n;
            typename V::type raw = {};
            if (whole) raw = *reinterpret_cast<const typename V::loose*>(x + e);
            else
#pragma unroll
                for (uint32_t j = 0; j < N; ++j)
                    if (e + j < n) raw[j] = x[e + j];
            const uint32_t bits = a.allowed ? allowed[e / 32] >> (e % 32) : ~0u;
            float z[N];
#pragma unroll
            for (uint32_t j = 0; j < N; ++j) z[j] = static_cast<float>(raw[j]);
            if constexpr (LISTS) {
                uint32_t w[N], any = 0;
#pragma unroll
                for (uint32_t j = 0; j < N; ++j) any |= w[j] = words[e + j];
                if (any)
#pragma unroll
                    for (uint32_t j = 0; j < N; ++j) z[j] = adjusted(z[j], w[j]);
            }
#pragma unroll
            for (uint32_t j = 0; j < N; ++j)
                if (!(bits >> j & 1) || e + j >= n) z[j] = -__builtin_huge_valf();
            float most_here = z[0];
#pragma unroll
            for (uint32_t j = 1; j < N; ++j) most_here = __builtin_elementwise_maximum(most_here, z[j]);
            if (!(most_here <= top) && top == top) {
#pragma unroll
                for (uint32_t j = 0; j < N; ++j)
                    if (!(z[j] <= top) && top == top) top = z[j], at = e + j;
            }
            if (a.out) {
                typename V::type rounded;
#pragma unroll
                for (uint32_t j = 0; j < N; ++j) rounded[j] = static_cast<T>(z[j]);
                if (whole) *reinterpret_cast<typename V::loose*>(y + e) = rounded;
                else
#pragma unroll
                    for (uint32_t j = 0; j < N; ++j)
                        if (e + j < n) y[e + j] = rounded[j];
            }
        }
        if (a.best) {
            const uint64_t k = most_of_wave(at < n ? key_of(top, v0 + at) : 0);
            if (tid % 64 == 0) most[tid / 64] = k;
            __syncthreads();
            if (tid == 0) {
                uint64_t all = most[0];
#pragma unroll
                for (int w = 1; w < kThreads / 64; ++w) all = most[w] > all ? most[w] : all;
                if (a.chunks == 1) at_global<uint32_t>(a.best)[row] = ~static_cast<uint32_t>(all);
                else at_global<uint64_t>(a.partial)[static_cast<int64_t>(row) * a.chunks + chunk] = all;
            }
            __syncthreads();
        }
        if constexpr (LISTS)
            if (tree) {
                __syncthreads();
                path(row, ~0u);
            }
    }
}

// The best of a row's chunks: a wave a row.
__global__ __launch_bounds__(kThreads) void best_kernel(LogitsArgs a)
{
    const uint32_t row = blockIdx.x * (kThreads / 64) + threadIdx.x / 64, lane = threadIdx.x % 64;
    if (row >= a.rows) return;
    uint64_t k = 0;
    for (uint32_t c = lane; c < a.chunks; c += 64) {
        const uint64_t o = at_global<const uint64_t>(a.partial)[static_cast<int64_t>(row) * a.chunks + c];
        k = o > k ? o : k;
    }
    k = most_of_wave(k);
    if (lane == 0) at_global<uint32_t>(a.best)[row] = ~static_cast<uint32_t>(k);
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
int64_t chunks_of(int64_t vocab) { return (vocab + kChunk - 1) / kChunk; }

}  // namespace

extern "C" {

int64_t logits_workspace_bytes(int64_t batch, int32_t nodes, int64_t vocab, int dtype)
{
    if (const int st = check(batch, nodes, vocab, dtype)) return st;
    return chunks_of(vocab) > 1 ? 8 * batch * nodes * chunks_of(vocab) : 0;
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
    a.history = l.history_width ? addr(l.history) : 0, a.history_lens = addr(l.history_lens), a.prompt_lens = addr(l.prompt_lens);
    a.bias_tokens = addr(l.bias_tokens), a.bias_values = addr(l.bias_values), a.allowed = addr(l.allowed);
    a.tree_tokens = addr(l.tree_tokens), a.tree_masks = addr(l.tree_masks), a.partial = addr(workspace);
    a.logits_stride = logits_stride, a.out_stride = out_stride, a.history_stride = l.history_stride, a.allowed_stride = l.allowed_stride;
    a.vocab = static_cast<uint32_t>(vocab), a.nodes = static_cast<uint32_t>(nodes), a.rows = static_cast<uint32_t>(batch * nodes);
    a.biases = static_cast<uint32_t>(l.biases), a.history_width = static_cast<uint32_t>(l.history_width);
    a.chunks = static_cast<uint32_t>(chunks_of(vocab));
    const bool used = l.biases || (l.penalties && (a.history || l.tree_masks));
    const int64_t wanted = 1024, units = a.chunks * batch;
    int64_t parts = used ? (wanted + units - 1) / units : nodes;
    if (parts > nodes) parts = nodes;
    a.part_rows = static_cast<uint32_t>((nodes + parts - 1) / parts);
    a.parts = static_cast<uint32_t>((nodes + a.part_rows - 1) / a.part_rows);
    if (!launchable(units * a.parts, kThreads)) return fail(ADDRMS_ERR_UNSUPPORTED_SHAPE, "the call is too large: %lld workgroups", (long long)(units * a.parts));
    const dim3 grid(static_cast<unsigned>(units * a.parts));
    const hipStream_t s = static_cast<hipStream_t>(stream);
#define GO(DT) launch_kernel(used ? logits_kernel<DT, true> : logits_kernel<DT, false>, grid, dim3(kThreads), s, a)
    SERVING_HIP_TRY(dtype == ADDRMS_BF16 ? GO(DT_BF16) : dtype == ADDRMS_FP16 ? GO(DT_FP16) : GO(DT_FP32));
#undef GO
    if (best && a.chunks > 1)
        SERVING_HIP_TRY(launch_kernel(best_kernel, dim3(static_cast<unsigned>((a.rows + kThreads / 64 - 1) / (kThreads / 64))), dim3(kThreads), s, a));
    return ADDRMS_OK;
}

}  // extern "C"
