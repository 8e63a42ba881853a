// How the keys of sequences of different lengths are cut into pieces of one length, as even shares of the work (device code).
//
// Lengths are known on the device alone.  Sequence b has k_b keys, its nodes' among them; a piece has as many as all together have for
// each of `cut_parts`, cut_least at least, in steps of 64, and sequence b has n_b = ceil(k_b / piece): together no more than cut_parts
// and one for each sequence.  Every wave works this out by itself, a sequence a lane.
#pragma once
#include "prefixattn_args.h"
#include "serving_internal.h"

namespace serving {

constexpr int32_t kCutStep = 64;

// Keys that sequence b has, 0 beyond the batch.
__device__ __forceinline__ int32_t keys_of(const AttnArgs& a, int32_t b)
{
    const int32_t room = a.suffix_width << a.page_shift;
    if (b >= a.batch) return 0;
    return min(min(max(at_global<const int32_t>(a.suffix_lens)[b], 0), room) + a.q_len, room);
}
__device__ __forceinline__ float sum_of_wave(float x)
{
    x += dpp<0xB1>(x);                                          // quad_perm 1,0,3,2
    x += dpp<0x4E>(x);                                          // quad_perm 2,3,0,1
    x += dpp<0x141>(x);                                         // row_half_mirror
    x += dpp<0x140>(x);                                         // row_mirror
    const pair r = with_row(x);
    const pair h = with_half(r.a + r.b);
    return h.a + h.b;
}
// Keys of a piece.  In fp32, where sums are off by less than 2^-18, and a little more than the share.
__device__ __forceinline__ int32_t piece_of(const AttnArgs& a, int32_t mine)
{
    float all = sum_of_wave(static_cast<float>(mine));
    for (int32_t b = 64; b < a.batch; b += 64) all += sum_of_wave(static_cast<float>(keys_of(a, b + (threadIdx.x & 63))));
    const float share = fminf(all / static_cast<float>(a.cut_parts) * 1.0001f, 0x1p30f);
    const int32_t keys = max(static_cast<int32_t>(share) + 1, a.cut_least);
    return (keys + kCutStep - 1) / kCutStep * kCutStep;
}
__device__ __forceinline__ int32_t pieces_of(int32_t keys, int32_t piece) { return static_cast<int32_t>((static_cast<uint32_t>(keys) + piece - 1) / static_cast<uint32_t>(piece)); }

// Of a sequence: the pieces of those before it, and its own.
struct Cut {
    int32_t before, pieces;
};
__device__ __forceinline__ Cut cut_of(const AttnArgs& a, int32_t seq)
{
    const int32_t lane = threadIdx.x & 63, mine = keys_of(a, lane), piece = piece_of(a, mine);
    int32_t before = 0;
    for (int32_t b = 0; b < seq; b += 64) {
        int32_t n = b + lane < seq ? pieces_of(b ? keys_of(a, b + lane) : mine, piece) : 0;
#pragma unroll
        for (int x = 32; x; x >>= 1) n += __shfl_xor(n, x);
        before += n;
    }
    return Cut{before, pieces_of(keys_of(a, seq), piece)};
}
// The sequence that a piece is of, by the piece's number among all (-1: there are fewer), its number there, and its length.
struct Piece {
    int32_t seq, number, keys;
};
__device__ __forceinline__ Piece piece_at(const AttnArgs& a, int32_t at)
{
    const int32_t lane = threadIdx.x & 63, mine = keys_of(a, lane), piece = piece_of(a, mine);
    for (int32_t b = 0; b < a.batch; b += 64) {
        int32_t n = pieces_of(b ? keys_of(a, b + lane) : mine, piece), end = n;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) {
            const int32_t o = __shfl_up(end, x);
            end += lane >= x ? o : 0;
        }
        const uint64_t has = __ballot(at < end);
        if (has) {
            const int32_t l = __builtin_ctzll(has);
            return Piece{b + l, at - (__shfl(end, l) - __shfl(n, l)), piece};
        }
        at -= __shfl(end, 63);
    }
    return Piece{-1, 0, piece};
}
// The sequence with the r-th most keys (of up to 64; of equals the first).
__device__ __forceinline__ int32_t by_length(const AttnArgs& a, int32_t r)
{
    const int32_t lane = threadIdx.x & 63, mine = lane < a.batch ? keys_of(a, lane) : -1;
    int32_t rank = 0;
    for (int32_t b = 0; b < a.batch; ++b) {
        const int32_t o = __builtin_amdgcn_readlane(mine, b);
        rank += o > mine || (o == mine && b < lane) ? 1 : 0;
    }
    return __builtin_ctzll(__ballot(lane < a.batch && rank == r));
}

}  // namespace serving
