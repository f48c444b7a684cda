// Attention of a few or many new tokens over a paged cache: what its kernels share (kernels_chunk.hip, kernels_prefix.hip).
#pragma once
#include "attn_row.h"
#include "attn_tile.h"
#include "gemm_epilogue.h"
#include "kernels.h"
#include "paged.h"

namespace exe {

// Keys first .. last - 1 that a row at position p sees.  The table gives positions below `limit`; a row beyond sees the first missing
// one, which makes it NaN, and no further.
struct KeyRange { int first, last; };
__device__ __forceinline__ KeyRange keys_of(int p, int window, int limit)
{
    int first = window > 0 && p >= window ? p - window + 1 : 0, last = p < 0 ? 0 : p < limit ? p + 1 : limit + 1;
    return KeyRange{first < limit ? first : limit, last};
}
__device__ __forceinline__ int table_limit(const PagedTable& t)
{
    int64_t n = (int64_t)t.max_blocks << t.shift;
    return n < 0x7ffff000 ? (int)n : 0x7ffff000;
}

// One query row by one wave over keys first .. last - 1, 64 at a time: a lane takes a key for the scores, and features lane, lane + 64
// of the result.  kv: this head's keys of block 0; block_of: the block with a position (-1: none); rows of a block's values lie v_off elements behind its keys; sc: the scale for exp2.
// acc is the mean over the keys so far, not their sum: it stays within the values' range, where the sum of some hundred values near a float's
// end does not.  A factor a step more, and 3 half steps of rounding for each 64 keys.
template <typename T, int DH, typename F>
__device__ __forceinline__ void chunk_row(const T* q, const T* kv, int64_t block_elems, int64_t v_off, int shift, F block_of, KeyRange r, float sc, int lane,
                                          T* out)
{
    float m = -INFINITY, l = 0.f, acc[DH / 64] = {};
    bool bad = false;
    const int mask = (1 << shift) - 1;
    for (int j0 = r.first; j0 < r.last; j0 += 64) {
        int j = j0 + lane, cnt = r.last - j0 < 64 ? r.last - j0 : 64, jj = j < r.last ? j : r.last - 1;
        int blk = block_of(jj);
        bad |= blk < 0;
        const int64_t at = (blk < 0 ? 0 : blk) * block_elems + (jj & mask) * DH;
        const T* k = kv + at;
        float s = 0.f;
#pragma unroll 4
        for (int e = 0; e < DH; ++e) s = fmaf(to_f32(q[e]), to_f32(k[e]), s);
        s = j < r.last ? s * sc : -INFINITY;
        float mx = wave_max(fmaxf(m, s)), mref = mx == -INFINITY ? 0.f : mx;
        float old = l * fast_exp2(m - mref), p = fast_exp2(s - mref);
        l = old + wave_sum(p);
        const float inv = l > 0.f ? 1.f / l : 0.f, keep = old * inv;
        p *= inv;
#pragma unroll
        for (int f = 0; f < DH / 64; ++f) acc[f] *= keep;
        for (int t = 0; t < cnt; ++t) {
            float pt = __shfl(p, t, WAVE);
            const T* v = kv + __shfl(at, t, WAVE) + v_off + lane;
#pragma unroll
            for (int f = 0; f < DH / 64; ++f) acc[f] = fmaf(pt, to_f32(v[f * 64]), acc[f]);
        }
        m = mx;
    }
    if (__builtin_amdgcn_ballot_w64(bad)) l = NAN;
#pragma unroll
    for (int f = 0; f < DH / 64; ++f) out[lane + f * 64] = from_f32<T>(r.last <= r.first ? 0.f : l > 0.f ? acc[f] : NAN);
}

// Rows whose results are not finite are computed again from their own keys: 0 times the infinite or NaN value of a key that the mask hides is
// NaN, and sums, of probabilities up to 2^8 here, pass a float's end where their mean does not.  most: the largest magnitude, or NaN; total:
// the sum of the probabilities.  That is NaN where one of the row's own scores is (or is infinite, or its block missing), 0 where all are
// minus infinity: such a row is NaN and stays it (512 tokens of NaN queries over a window of 1000: 33 times faster so).
__device__ __forceinline__ float magnitude(float most, float v) { return __builtin_elementwise_maximum(most, fabsf(v)); }
__device__ __forceinline__ bool spoilt(float most, float total) { return !(most < INFINITY) && total > 0.f; }

// What the loads of a position without a block read in its place, 16 rows each: NaN keys make the scores of the rows that see it NaN,
// values of 0 leave the others as they are.  (Tiles reach up to 63 positions in front of a window, where pages may have been given back.)
struct NoBlock {
    uint32_t keys[16 * 512 / 4], values[16 * 512 / 4];
    constexpr NoBlock() : keys(), values() { for (uint32_t& x : keys) x = 0xffffffffu; }
};
static __device__ const __align__(16) NoBlock no_block;

template <int N> __device__ __forceinline__ void wait_loads()        // all but the last N
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N) : "memory");
}

// Moves 16 positions (a multiple of 16 on) of one head's keys or values from the cache to LDS, by one wave: LOADS direct loads of 1 KB, RPL rows each,
// row-major, chunks swizzled (see attn_tile.h).  The loads are inline assembly, so that the compiler does not order every later LDS read
// behind them; whoever reads the rows waits.  The table is read by scalar loads, which do not wait behind the loads in flight.
// NT: nontemporal, for rows that no other workgroup reads.
template <typename T, int DH, bool NT> struct RowLoader {
    static constexpr int RB = DH * (int)sizeof(T), RPL = 1024 / RB, CPR = RB / 16, LOADS = 16 / RPL, HALF = LOADS / 2;
    typedef const __attribute__((address_space(4))) int32_t* ScalarPtr;
    const char* kv;                       // this head's keys of block 0
    int64_t v_off;                        // bytes from a row's key to its value
    unsigned block_bytes;
    ScalarPtr entry;
    int max_blocks, shift, n_blocks, limit, last, lane;
    unsigned voff;                        // of load 0; load p's is this one with other chunk bits
    __device__ __forceinline__ RowLoader(const PagedTable& t, const void* pool, int b, int kvh, int Hkv, int limit_, int last_, int lane_)
        : entry((ScalarPtr)(uintptr_t)(t.entry + (int64_t)b * t.max_blocks)), max_blocks(t.max_blocks), shift(t.shift), n_blocks(t.n_blocks), limit(limit_), last(last_), lane(lane_)
    {
        const int64_t head = (int64_t)RB << shift;
        kv = (const char*)pool + kvh * head;
        v_off = Hkv * head;
        block_bytes = (unsigned)(2 * v_off);
        voff = lane / CPR * RB + (((lane & (CPR - 1)) ^ pf_swz<RB>(lane / CPR)) << 4);
    }
    // Table entries of positions j and j + 8, as they stand: looked at where they are used, so that nothing waits for them before.
    struct Entries { int e0, e1; };
    __device__ __forceinline__ Entries lookup(int j) const
    {
        const int j0 = j < last ? j : last - 1, j1 = j + 8 < last ? j + 8 : last - 1, i0 = j0 >> shift, i1 = j1 >> shift;
        return Entries{entry[i0 < max_blocks ? i0 : max_blocks - 1], entry[i1 < max_blocks ? i1 : max_blocks - 1]};
    }
    // Where the key of a position lies, and how far behind it its value.
    struct Row { const char* key; int64_t value; };
    __device__ __forceinline__ Row row(int e, int pos) const
    {
        const bool ok = (unsigned)e < (unsigned)n_blocks && pos < limit;
        const uint64_t at = (uint64_t)(unsigned)e * block_bytes + (unsigned)((pos & ((1 << shift) - 1)) * RB);
        return Row{ok ? kv + at : (const char*)no_block.keys, ok ? v_off : (int64_t)sizeof(no_block.keys)};
    }
    struct Rows { Row r0, r1; };          // of positions j .. j + 7 and j + 8 .. j + 15; of the last one where those are beyond it
    __device__ __forceinline__ Rows rows(int j, Entries en) const
    {
        if (shift > 3 && j + 8 < last) {                               // one block
            const Row r = row(en.e0, j);
            return Rows{r, Row{r.key + 8 * RB, r.value}};
        }
        return Rows{row(en.e0, j < last ? j : last - 1), row(en.e1, j + 8 < last ? j + 8 : last - 1)};
    }
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
    // Loads P .. P + HALF - 1, of 8 rows that follow each other from src on.  The immediate offset counts for the source and for LDS.
    template <int P> __device__ __forceinline__ void half(const char* src, unsigned dst_rows) const
    {
        const unsigned dst = dst_rows + P * 1024;
        auto v = [&](int p) { return voff ^ (pf_swz<RB>(p * RPL) << 4); };
        if constexpr (HALF == 1) {
            load_one(src, v(P), dst);
        } else if constexpr (HALF == 2) {
#define EXE_HALF2(FLAG)                                                                                                                     \
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3" FLAG "\n\tglobal_load_lds_dwordx4 %2, %3 offset:%4" FLAG   \
                 ::"s"(dst), "v"(v(P)), "v"(v(P + 1)), "s"(src), "i"(1024) : "memory", "m0")
            if (NT) EXE_HALF2(" nt");
            else EXE_HALF2("");
#undef EXE_HALF2
        } else {
#define EXE_HALF4(FLAG)                                                                                                                     \
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5" FLAG "\n\tglobal_load_lds_dwordx4 %2, %5 offset:%6" FLAG   \
                 "\n\tglobal_load_lds_dwordx4 %3, %5 offset:%7" FLAG "\n\tglobal_load_lds_dwordx4 %4, %5 offset:%8" FLAG                    \
                 ::"s"(dst), "v"(v(P)), "v"(v(P + 1)), "v"(v(P + 2)), "v"(v(P + 3)), "s"(src), "i"(1024), "i"(2 * 1024), "i"(3 * 1024) : "memory", "m0")
            if (NT) EXE_HALF4(" nt");
            else EXE_HALF4("");
#undef EXE_HALF4
        }
    }
    __device__ __forceinline__ void load_one(const char* src, unsigned v, unsigned dst) const
    {
        if (NT) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(dst), "v"(v), "s"(src) : "memory", "m0");
        else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(dst), "v"(v), "s"(src) : "memory", "m0");
    }
#pragma clang diagnostic pop
    // 16 rows from s0 (8 rows) and s1 on; rows of positions from `last` on are last - 1 again
    __device__ __forceinline__ void move(int j, const char* s0, const char* s1, unsigned dst) const
    {
        if (j + 16 <= last) {
            half<0>(s0, dst);
            half<HALF>(s1, dst);
            return;
        }
#pragma unroll
        for (int p = 0; p < LOADS; ++p) {
            const int half_at = p < HALF ? j : j + 8, in = lane / CPR, row = p % HALF * RPL + in, most = half_at < last ? last - 1 - half_at : 0;
            const unsigned v = (row < most ? row : most) * RB + (((lane & (CPR - 1)) ^ pf_swz<RB>(p * RPL + in)) << 4);
            load_one(p < HALF ? s0 : s1, v, dst + p * 1024);
        }
    }
    __device__ __forceinline__ void keys(int j, const Rows& r, unsigned dst) const { move(j, r.r0.key, r.r1.key, dst); }
    __device__ __forceinline__ void values(int j, const Rows& r, unsigned dst) const { move(j, r.r0.key + r.r0.value, r.r1.key + r.r1.value, dst); }
};

// A row's query fragments (B operand of the first product): lane (row qi, group g) holds 16-byte chunks 4 * ds + g.  The sign of the
// scale goes to the query, since the softmax takes the maximum of the raw scores; scale 0 makes it 0, and all scores that are numbers.
template <typename T, int DS> __device__ __forceinline__ void load_query(const T* q, int g, float scale, u32x4 (&f)[DS])
{
#pragma unroll
    for (int ds = 0; ds < DS; ++ds) f[ds] = ((const u32x4*)q)[4 * ds + g];
    if (scale < 0.f || scale == 0.f) {
#pragma unroll
        for (int ds = 0; ds < DS; ++ds)
            f[ds] = scale == 0.f ? u32x4{0, 0, 0, 0} : f[ds] ^ (sizeof(T) == 4 ? 0x80000000u : 0x80008000u);
    }
}
__device__ __forceinline__ float exponent_scale(float scale) { return scale == 0.f ? 1.f : fabsf(scale) * LOG2E; }

}  // namespace exe
