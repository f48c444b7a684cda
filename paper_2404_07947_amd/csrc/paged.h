// Looking things up in a batch of new tokens over a paged cache.
#pragma once
#include "common.h"

namespace exe {

// The block table of a batch, [n_seqs, max_blocks]; blocks of 2^shift positions.
struct PagedTable {
    const int32_t* entry;
    int max_blocks, shift, n_blocks;
    // The block with position `pos` of sequence b; -1 where the table has none or names one outside of the pool.
    __device__ __forceinline__ int block(int b, int pos) const
    {
        int i = pos >> shift;
        if (pos < 0 || i >= max_blocks) return -1;
        int blk = entry[(int64_t)b * max_blocks + i];
        return (unsigned)blk < (unsigned)n_blocks ? blk : -1;
    }
};

// A sequence's new tokens among the packed ones: t0 .. t0 + n - 1 of sequence b (-1: none).
struct ChunkSeq { int b, t0, n; };

// The last of the positions lo .. hi - 1 at which `before` holds (it holds up to some position and not behind it; lo - 1: nowhere),
// by a whole wave, 64 probes at a time.
template <typename F> __device__ __forceinline__ int wave_search(int lo, int hi, int lane, F before)
{
    while (lo < hi) {
        int step = (int)(((int64_t)hi - lo + 63) / 64);
        int64_t i = lo + (int64_t)lane * step;
        int n = __popcll(__builtin_amdgcn_ballot_w64(i < hi && before((int)i)));
        if (n == 0) return lo - 1;
        lo += (n - 1) * step;
        if (step == 1) return lo;
        hi = lo + step < hi ? lo + step : hi;
    }
    return lo - 1;
}

// The sequence of token t.
__device__ __forceinline__ ChunkSeq seq_of_token(const int32_t* __restrict__ cu, int n_seqs, int t, int lane)
{
    int b = wave_search(0, n_seqs, lane, [&](int i) { return cu[i] <= t; });
    if (b < 0) return ChunkSeq{-1, 0, 0};
    int t0 = cu[b], end = cu[b + 1];
    return t < end ? ChunkSeq{b, t0, end - t0} : ChunkSeq{-1, 0, 0};
}

}  // namespace exe
