// Log probabilities of given tokens, entropy and the largest probabilities, of rows of logits.  Rows of 50272, a call: 1 float 7.0 us, of which loads and
// sums of 200 KB by one CU are 2.8 (by the difference to a row of 12000), 256 float 12.4 (4.1 TB/s), 2048 bf16 41.5 (5.0 TB/s; vector instructions four fifths
// of the time, of which 13 a logit, 8 in the sums).  One pass over the registers for the maximum and the sums, about a number that follows the lane's largest logit,
// has a tenth fewer of them and is slower (43), since it waits chunk by chunk.
//
// With the largest logit M and c = scale * log2 e: z = (x - M) * c, S = sum of 2^z, Y = sum of 2^z z; then log p = (z - log2 S) ln 2 and the
// entropy is (log2 S - Y / S) ln 2.
//  * logprob_part_kernel: a workgroup takes 256 * C chunks of 16 bytes of a row into registers, in one round of loads, and makes the sums and the sorted
//    list of its k best from there: the logits are read once.
//  * logprob_join_kernel: where a row has several parts, adds up their sums and merges their lists, 64 parts at a time.
#include <type_traits>

#include "attn_row.h"
#include "kernels.h"

namespace exe {

typedef unsigned long long u64;
constexpr int LP_JOIN_THREADS = 256, LP_CAP = 512, LP_JOIN = 64;      // LP_CAP: all logits of a part in which fewer than 64 threads have some
constexpr float LN2 = 0.69314718055994530942f;

struct LogprobKernelArgs {
    const void* logits; int64_t row_stride;
    unsigned n;
    float c, scale;                        // scale * log2 e
    const int32_t* tokens; int n_tokens;
    float *logprobs, *entropy;
    int k;
    int32_t* top_ids; float* top_logprobs;
    unsigned parts, span;                  // of a row, that this launch writes; logits of each
    float* sums; u64* lists;               // where they go: [rows * parts][M, S, Y, -], [rows * parts][k]; parts 1: the results themselves
    unsigned from_parts;                   // joining: of a row, that it reads
    const float* from_sums; const u64* from_lists;
};

// A logit and its place as one number, larger for the larger logit and, of equal ones (0 and -0 are), for the lower place; never 0.
__device__ __forceinline__ unsigned logit_order(float x)
{
    const unsigned u = __float_as_uint(x + 0.f);
    return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ u64 logit_key(unsigned order, unsigned i) { return (u64)order << 32 | ~i; }
__device__ __forceinline__ float order_logit(unsigned o) { return __uint_as_float(o ^ (o >> 31 ? 0x80000000u : 0xffffffffu)); }
__device__ __forceinline__ float key_logit(u64 key) { return order_logit((unsigned)(key >> 32)); }

// The largest over the wave, of numbers (a NaN is never taken)
__device__ __forceinline__ float lanes_max(float v)
{
    v = fmaxf(v, dpp_move<0xB1>(v));
    v = fmaxf(v, dpp_move<0x4E>(v));
    v = fmaxf(v, dpp_move<0x141>(v));
    v = fmaxf(v, dpp_move<0x140>(v));
    return rows_max(v);
}

struct Sums { float M, S, Y; };
// A part's sums to the largest logit M of several.  Where a part has no number but -inf its M is -inf, and its sums are 0, or NaN.
__device__ __forceinline__ void sums_to(Sums& p, float M, float c)
{
    if (p.M == -INFINITY) return;
    // halves, whose difference is never infinite where the scale makes it small
    const float d = fmaxf((0.5f * p.M - 0.5f * M) * c * 2.f, -1e30f), w = fast_exp2(d);
    p.Y = w * fmaf(p.S, d, p.Y);
    p.S *= w;
    p.M = M;
}

// The given token of this thread, asked for early, and its logit, which is on its way while others are sorted: two trips to memory.
__device__ __forceinline__ unsigned given_token(const LogprobKernelArgs& a, int64_t row)
{
    return a.parts == 1 && (int)threadIdx.x < a.n_tokens ? (unsigned)a.tokens[row * a.n_tokens + threadIdx.x] : 0xffffffffu;
}
template <typename T> __device__ __forceinline__ float given_logit(const LogprobKernelArgs& a, int64_t row, unsigned token)
{
    return token < a.n ? to_f32(((const T*)a.logits + row * a.row_stride)[token]) : NAN;
}
// The results of a row, by a workgroup: sums, and the k best keys in LDS (0: there are fewer).
template <typename T, int THREADS> __device__ __forceinline__ void logprob_finish(const LogprobKernelArgs& a, int64_t row, Sums t, const u64* top, float given)
{
    // The largest logit's own term is 1, but comes out as 1 - 2^-24 where the rounding of its sums' reference is taken out again: no probability above 1,
    // no entropy below 0.  (Comparisons: a NaN stays one.)
    if (t.S > 0.f && t.S < 1.f) t.S = 1.f;
    const float L = log2f(t.S) * LN2;
    // in 64 bits: the logits may lie further apart than the largest float
    auto logprob = [&](float x) { return (float)(((double)x - (double)t.M) * (double)a.scale - (double)L); };
    if ((int)threadIdx.x < a.n_tokens) a.logprobs[row * a.n_tokens + threadIdx.x] = logprob(given);
    for (int i = threadIdx.x + THREADS; i < a.n_tokens; i += THREADS)
        a.logprobs[row * a.n_tokens + i] = logprob(given_logit<T>(a, row, (unsigned)a.tokens[row * a.n_tokens + i]));
    if (a.entropy && threadIdx.x == 0) {
        const float h = L - t.Y / t.S * LN2;
        a.entropy[row] = h < 0.f ? 0.f : h;
    }
    if ((int)threadIdx.x < a.k) {
        const u64 key = top[threadIdx.x];
        a.top_ids[row * a.k + threadIdx.x] = key ? (int)~(unsigned)key : -1;
        a.top_logprobs[row * a.k + threadIdx.x] = key ? logprob(key_logit(key)) : -INFINITY;
    }
}

// f of 0 .. C - 1 as constants, as far as `chunks` goes (SOME; else all): one branch around all that follow, where the compiler makes of a loop with a
// condition one for each, which it then moves together (bf16 rows 45 us, so 59), and of a longer one with a break no constants.
template <int C, bool SOME, int I = 0, typename F> __device__ __forceinline__ void each_chunk(int chunks, F f)
{
    if constexpr (I < C) {
        if (SOME && I >= chunks) return;
        f(std::integral_constant<int, I>{});
        each_chunk<C, SOME, I + 1>(chunks, f);
    }
}

template <typename T, int THREADS, int C> struct LogitPart {
    // Few chunks: all are in use.  Many, in float: a wave that has all of them, or all but one, of a row that begins on 16 bytes makes the sums of the first ones
    // while the others are on their way (a row a CU of 256 of 50272 13.4 -> 12.5 us a call, one row 7.3 -> 7.0; in thirds the same).
    static constexpr bool SOME = THREADS > 256, HALVES = THREADS > 256 && sizeof(T) == 4;
    static constexpr int V = 16 / (int)sizeof(T), N = C * V, SPAN = THREADS * N;
    uint4 raw[C];
    __device__ __forceinline__ float at(int i) const       // i: a constant after unrolling
    {
        const uint4 u = raw[i / V];
        const int w = sizeof(T) == 4 ? i % V : i % V / 2;
        const unsigned d = w == 0 ? u.x : w == 1 ? u.y : w == 2 ? u.z : u.w;
        return sizeof(T) == 4 ? __uint_as_float(d) : i & 1 ? bf16hi(d) : bf16lo(d);
    }
    // place of element i among the part's
    static __device__ __forceinline__ unsigned place(int i) { return (i / V * THREADS + threadIdx.x) * V + i % V; }
    // New values to the compiler, which would keep what it made of all of them in registers from one use to the next.
    __device__ __forceinline__ void renew()
    {
#pragma unroll
        for (int c = 0; c < C; ++c) asm volatile("" : "+v"(raw[c].x), "+v"(raw[c].y), "+v"(raw[c].z), "+v"(raw[c].w));
    }
    // Logits first .. end - 1 of the row, the first on 16 bytes: up to V - 1 before the row's first one.  What is not of them is -inf.  All loads go
    // out before anything waits: those of chunks that are not there, or only in part, from the nearest whole one.
    // Of the C chunks the first `chunks` are in use (SOME), or all; LONG: there is a whole one for sure.  `fill`
    // looks after those of chunks I .. J - 1 that are there in part or not at all: none, where the first `whole` are so in all lanes of the wave.
    template <bool SOME, bool LONG> __device__ __forceinline__ void load(const T* x, unsigned first, unsigned n, int chunks)
    {
        // whole chunks of the row: from its first or second one on, up to `high`, both counted from `first`
        const int lead = (int)((uintptr_t)x & 15) / (int)sizeof(T), low = first > n && lead ? V : 0;
        const int64_t at = first > n ? -(int64_t)lead : (int64_t)first, high = at + ((int64_t)n - at) / V * V - V - at;
        if (LONG || high >= low) {
            const char* base = (const char*)(x + at);
            const int most = high < SPAN ? (int)high : SPAN;
            each_chunk<C, SOME>(chunks, [&](auto c) {
                int i = (int)place(c * V);
                i = i < low ? low : i < most ? i : most;
                raw[c] = load_chunk<true>((const uint4*)(base + (unsigned)(i * (int)sizeof(T))));
            });
        }
    }
    template <bool SOME, int I, int J> __device__ __forceinline__ void fill(const T* x, unsigned first, unsigned end, int chunks, int whole)
    {
        if (whole >= (SOME ? chunks : C)) return;
        each_chunk<J, SOME, I>(chunks, [&](auto c) {
            const unsigned i = first + place(c * V);
            if (i < end && end - i >= V) return;
            if ((int)(end - i) <= 0) {                         // nothing of it
                const unsigned none = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
                raw[c] = uint4{none, none, none, none};
                return;
            }
            unsigned w[4];
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                if constexpr (sizeof(T) == 4) {
                    w[d] = i + d < end ? __float_as_uint(x[i + d]) : 0xff800000u;
                } else {
                    const unsigned lo = i + 2 * d < end ? ((const uint16_t*)x)[i + 2 * d] : 0xff80u, hi = i + 2 * d + 1 < end ? ((const uint16_t*)x)[i + 2 * d + 1] : 0xff80u;
                    w[d] = lo | hi << 16;
                }
            }
            raw[c] = uint4{w[0], w[1], w[2], w[3]};
        });
    }
};
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// The k best of `count` keys, at most LP_CAP, sorted by counting, for each, those above it; 0 where there are fewer.
template <int THREADS> __device__ __forceinline__ void sort_keys(const u64* keys, int count, u64* top, int k)
{
    const int tid = threadIdx.x;
    auto sort = [&](int i) {
        if (i >= count) return;
        const u64 mine = keys[i];
        int above = 0;
        for (int j = 0; j < count; ++j) above += keys[j] > mine;
        if (above < k) top[above] = mine;
    };
    sort(tid);
    if (LP_CAP > THREADS && count > THREADS) sort(tid + THREADS);
    if (tid >= count && tid < k) top[tid] = 0;
}

template <typename T, int THREADS, int C> __global__ __launch_bounds__(THREADS, THREADS == 1024 && sizeof(T) == 2 ? 8 : 1) void logprob_part_kernel(LogprobKernelArgs a)
{
    typedef LogitPart<T, THREADS, C> Part;
    constexpr int WAVES = THREADS / WAVE, V = Part::V;
    __shared__ u64 s_keys[LP_CAP], s_top[WAVE];
    __shared__ Sums s_sums[WAVES], s_row;
    __shared__ float s_given[THREADS];
    __shared__ __align__(16) float s_best[THREADS];
    __shared__ int s_count, s_digit, s_counts[256];
    static_assert(THREADS % 256 == 0 && WAVES <= WAVE && Part::SPAN <= 1 << 16, "a count for each digit; a lane for each wave; 16 bits of a place");
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = blockIdx.x / a.parts;
    const unsigned part = blockIdx.x - (unsigned)row * a.parts;
    const T* x = (const T*)a.logits + row * a.row_stride;
    const unsigned first = part * a.span - (unsigned)((uintptr_t)x & 15) / sizeof(T), end = first + a.span < a.n ? first + a.span : a.n;
    Part p;
    // chunks of which this wave has something
    const int there = (int)(end - first) - __builtin_amdgcn_readfirstlane(wave) * (WAVE * V), chunks = there > 0 ? (there + THREADS * V - 1) / (THREADS * V) : 0;
    // those that are whole in all of its lanes; none where the first ones begin in front of the row
    const int whole = first > end || there < WAVE * V ? 0 : (there - WAVE * V) / (THREADS * V) + 1;
    const unsigned token = given_token(a, row);
    if (tid == 0) s_count = 0;

    float tops[C], best = -INFINITY;                           // of a chunk; of all
#pragma unroll
    for (int c = 0; c < C; ++c) tops[c] = -INFINITY;
    // Sums of chunks I .. J - 1, about the wave's largest of them, or (HALVES) this lane's
    auto sum_chunks = [&](auto some, auto from, auto to) {
        constexpr bool SOME = some;
        constexpr int I = from, J = to;
        if constexpr (SOME == Part::SOME) {
            p.template fill<SOME, I, J>(x, first, end, chunks, whole);
        } else if constexpr (J == C) {
            p.template fill<SOME, C - 2, C>(x, first, end, chunks, whole);
        }
        each_chunk<J, SOME, I>(chunks, [&](auto c) {
            const int i = c * V;
            tops[c] = max3(p.at(i), p.at(i + 1), p.at(i + 2));
            if constexpr (V == 8) tops[c] = max3(max3(tops[c], p.at(i + 3), p.at(i + 4)), p.at(i + 5), p.at(i + 6));
            tops[c] = max3(tops[c], tops[c], p.at(i + V - 1));
        });
        float most = -INFINITY;
#pragma unroll
        for (int c = I; c < J; ++c) most = fmaxf(most, tops[c]);
        best = fmaxf(best, most);
        if constexpr (!Part::HALVES) most = lanes_max(most);
        if constexpr ((J - I) * V > 32) p.renew();
        const float R = most == -INFINITY ? 0.f : most * a.c;
        float S = 0.f, Y = 0.f;
        auto add = [&](float z) {
            const float e = fast_exp2(z);
            S += e;
            Y = fmaf(e, fmaxf(z, -1e30f), Y);                  // 0 times minus infinity is 0 here; what is NaN is so in e
        };
        if (!__builtin_amdgcn_ballot_w64(!(fabsf(R) < 0x1p20f))) {
            // One operation a logit: z + off = c * x - R, where off = c * M - R, what R was rounded by, is 1/16 at most, and taken out of the sums.
            each_chunk<J, SOME, I>(chunks, [&](auto c) {
#pragma unroll
                for (int i = c * V; i < (c + 1) * V; ++i) add(fmaf(p.at(i), a.c, -R));
            });
            const float off = most == -INFINITY ? 0.f : fmaf(most, a.c, -R), w = fast_exp2(-off);
            Y = (Y - off * S) * w;
            S *= w;
        } else {
            each_chunk<J, SOME, I>(chunks, [&](auto c) {
#pragma unroll
                for (int i = c * V; i < (c + 1) * V; ++i) add((p.at(i) - (most == -INFINITY ? 0.f : most)) * a.c);
            });
        }
        if (S != S) {
            // A NaN (or plus infinity).  Of a signalling NaN and a number the instruction makes a quiet NaN, and of that and the next number the latter: the first is
            // lost.  So by comparisons, for the alternatives' sake: the sums are NaN, about whatever maximum.
            each_chunk<J, SOME, I>(chunks, [&](auto c) {
                tops[c] = -INFINITY;
#pragma unroll
                for (int i = c * V; i < (c + 1) * V; ++i) tops[c] = p.at(i) > tops[c] ? p.at(i) : tops[c];
                best = fmaxf(best, tops[c]);
            });
        }
        return Sums{most, S, Y};
    };
    constexpr auto zero = std::integral_constant<int, 0>{};
    constexpr auto all = std::integral_constant<int, C>{};
    float S, Y, most;
    auto join_lanes = [&](Sums q) {
        if constexpr (Part::HALVES) sums_to(q, most, a.c);
        S += q.S;
        Y += q.Y;
    };
    S = Y = 0.f;
    if (Part::HALVES && chunks >= C - 1 && first == 0) {
        constexpr auto half = std::integral_constant<int, C / 2>{};
        p.template load<false, true>(x, first, a.n, chunks);
        const Sums q = sum_chunks(std::false_type{}, zero, half), r = sum_chunks(std::false_type{}, half, all);
        most = lanes_max(best);
        join_lanes(q);
        join_lanes(r);
    } else {
        p.template load<Part::SOME, false>(x, first, a.n, chunks);
        const Sums q = sum_chunks(std::bool_constant<Part::SOME>{}, zero, all);
        most = Part::HALVES ? lanes_max(best) : q.M;
        join_lanes(q);
    }
    S = wave_sum(S);
    Y = wave_sum(Y);
    if (lane == 0) s_sums[wave] = Sums{most, S, Y};
    s_best[tid] = best;
    __syncthreads();
    const float given = given_logit<T>(a, row, token);
    auto join_waves = [&]() {                                  // by the last one, which has no part in the sorting
        if (wave != WAVES - 1) return;
        Sums p = lane < WAVES ? s_sums[lane] : Sums{-INFINITY, 0.f, 0.f};
        const float M = lanes_max(p.M);
        sums_to(p, M, a.c);
        const float S = wave_sum(p.S), Y = wave_sum(p.Y);
        if (lane == 0) {
            if (a.parts > 1) *(f32x4*)(a.sums + (int64_t)blockIdx.x * 4) = f32x4{M, S, Y, 0.f};
            else s_row = Sums{M, S, Y};
        }
    };
    if (a.k) {
        // k logits or more are no smaller than the k-th largest of the threads' best ones, of which the largest of each 64th of them will do where k is small and so many
        // 64ths have one: these take part in a search for its upper 16 bits, a number no larger.  (Short parts of 256 threads may have fewer, which leaves all their
        // logits: 64 rows of 300 floats, k 20, 62 us with them sorted in memory, 5.2 by the threads' best.)
        f32x4 b4;
        if (a.k > 1) {
            b4 = *(const f32x4*)(s_best + 4 * lane);
#pragma unroll
            for (int i = 1; i < THREADS / 256; ++i) {
                const f32x4 more = *(const f32x4*)(s_best + 256 * i + 4 * lane);
#pragma unroll
                for (int e = 0; e < 4; ++e) b4[e] = fmaxf(b4[e], more[e]);
            }
        }
        unsigned kth = 0;
        if (a.k == 1) {
            kth = logit_order(lanes_max(s_sums[lane % WAVES].M));            // the largest of all, at hand (2048 bf16 rows of 50272 41.4 -> 40.5 us)
        } else if (const float of4 = fmaxf(fmaxf(b4[0], b4[1]), fmaxf(b4[2], b4[3])); a.k <= 32 && (THREADS > 256 || __popcll(__builtin_amdgcn_ballot_w64(of4 > -INFINITY)) >= a.k)) {
            const unsigned o = logit_order(of4);
            for (unsigned bit = 1u << 31; bit >= 1u << 16; bit >>= 1)          // (two bits a step, by three counts: 0.3 us more)
                if (__popcll(__builtin_amdgcn_ballot_w64(o >= (kth | bit))) >= a.k) kth |= bit;
        } else {
            const unsigned o[4] = {logit_order(b4[0]), logit_order(b4[1]), logit_order(b4[2]), logit_order(b4[3])};
            for (unsigned bit = 1u << 31; bit >= 1u << 16; bit >>= 1) {
                int n = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) n += __popcll(__builtin_amdgcn_ballot_w64(o[i] >= (kth | bit)));
                if (n >= a.k) kth |= bit;
            }
        }
        s_given[tid] = given;                                  // (a register to spare)
        p.renew();
        float least = order_logit(kth);
        least = least >= -3.4028235e38f ? least : -3.4028235e38f;              // those of -inf are ruled out; not a number: fewer than k
        // One of each lane that has some at a time, in any order: they are sorted.
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if (!__builtin_amdgcn_ballot_w64(tops[c] >= least)) continue;
            unsigned have = 0;                                 // a bit for each
#pragma unroll
            for (int e = 0; e < V; ++e) have |= p.at(c * V + e) >= least ? 1u << e : 0u;
            for (u64 some; (some = __builtin_amdgcn_ballot_w64(have != 0)); have &= have - 1) {
                int at = 0;
                if (lane == 0) at = atomicAdd(&s_count, __popcll(some));
                at = __builtin_amdgcn_readfirstlane(at) + __builtin_amdgcn_mbcnt_hi((unsigned)(some >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)some, 0));
                if (have && at < LP_CAP) {
                    const int e = __builtin_ctz(have);
                    float v = p.at(c * V);
#pragma unroll
                    for (int o = 1; o < V; ++o) v = e == o ? p.at(c * V + o) : v;
                    s_keys[at] = logit_key(logit_order(v), first + Part::place(c * V) + e);
                }
            }
        }
        __syncthreads();
        int count = s_count;
        if (count > LP_CAP) {
            // Many equal ones, or most of a wave's ruled out: the k-th largest of (logit, place), 8 bits a round, from memory again; then those from it on.
            auto key_at = [&](unsigned i, unsigned place) {
                const float v = to_f32(x[i]);
                return v > -INFINITY ? (u64)logit_order(v) << 16 | (0xffff - place) : 0ull;
            };
            u64 kth = 0;
            int need = a.k;
            for (int shift = 40; shift >= 0; shift -= 8) {
                if (tid < 256) s_counts[tid] = 0;
                __syncthreads();
                for (unsigned i = tid; i < a.span; i += THREADS) {
                    const u64 key = first + i < end ? key_at(first + i, i) : 0;
                    if (key && key >> shift >> 8 == kth >> shift >> 8) atomicAdd(&s_counts[key >> shift & 255], 1);
                }
                __syncthreads();
                int above = 0;
                for (int j = tid + 1; j < 256; ++j) above += s_counts[j];
                if (tid < 256 && above < need && above + s_counts[tid] >= need) {
                    s_count = above;
                    s_digit = tid;
                }
                __syncthreads();
                need -= s_count;
                kth |= (u64)s_digit << shift;
                __syncthreads();
            }
            if (tid == 0) s_count = 0;
            __syncthreads();
            for (unsigned i = tid; i < a.span; i += THREADS) {
                const u64 key = first + i < end ? key_at(first + i, i) : 0;
                if (key >= kth) s_keys[atomicAdd(&s_count, 1)] = logit_key((unsigned)(key >> 16), first + i);
            }
            __syncthreads();
            count = a.k;
        }
        join_waves();
        if (a.parts > 1) {
            sort_keys<THREADS>(s_keys, count, a.lists + (int64_t)blockIdx.x * a.k, a.k);
        } else {
            sort_keys<THREADS>(s_keys, count, s_top, a.k);
            __syncthreads();
        }
    }
    if (!a.k) {
        s_given[tid] = given;
        join_waves();
        __syncthreads();
    }
    if (a.parts > 1) return;
    logprob_finish<T, THREADS>(a, row, s_row, s_top, s_given[tid]);
}

// Lists i of up to 64, sorted, each of k keys: the k best of them all.  What the m-th of every list (k of them or more together) and the k-th of
// one are not below is left out, the rest sorted by counting; if that leaves too many, one wave takes the largest of the lists' heads k times.
template <typename T> __global__ __launch_bounds__(LP_JOIN_THREADS) void logprob_join_kernel(LogprobKernelArgs a)
{
    extern __shared__ __align__(16) unsigned char lp_smem[];
    u64* s_all = (u64*)lp_smem;                                // [lists][k]
    __shared__ u64 s_keys[LP_CAP], s_top[WAVE];
    __shared__ int s_count;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = blockIdx.x / a.parts;
    const unsigned part = blockIdx.x - (unsigned)row * a.parts;
    const int lists = a.from_parts - part * LP_JOIN < LP_JOIN ? a.from_parts - part * LP_JOIN : LP_JOIN;
    const int64_t from = row * a.from_parts + part * LP_JOIN;
    const float given = given_logit<T>(a, row, given_token(a, row));
    f32x4 s = {-INFINITY, 0.f, 0.f, 0.f};
    if (lane < lists) s = *(const f32x4*)(a.from_sums + (from + lane) * 4);
    if (a.k) {
        const u64* in = a.from_lists + from * a.k;
        const int m = (a.k + lists - 1) / lists;
        u64 low = ~0ull, high = 0;
        if (lane < lists) {
            low = in[lane * a.k + m - 1];
            high = in[lane * a.k + a.k - 1];
        }
        if (tid == 0) s_count = 0;
        for (int i = tid; i < lists * a.k; i += LP_JOIN_THREADS) s_all[i] = in[i];
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const u64 l = __shfl_xor(low, o, WAVE), h = __shfl_xor(high, o, WAVE);
            low = l < low ? l : low;
            high = h > high ? h : high;
        }
        u64 least = low > high ? low : high;
        if (!least) least = 1;                                 // 0 is no key
        __syncthreads();
        for (int i = tid; i < lists * a.k; i += LP_JOIN_THREADS)
            if (s_all[i] >= least) {
                const int at = atomicAdd(&s_count, 1);
                if (at < LP_CAP) s_keys[at] = s_all[i];
            }
        __syncthreads();
        u64* top = a.parts > 1 ? a.lists + (int64_t)blockIdx.x * a.k : s_top;
        if (s_count <= LP_CAP) {
            sort_keys<LP_JOIN_THREADS>(s_keys, s_count, top, a.k);
        } else if (wave == 0) {
            int next = 0;
            for (int i = 0; i < a.k; ++i) {
                const u64 head = lane < lists && next < a.k ? s_all[lane * a.k + next] : 0;
                u64 best = head;
#pragma unroll
                for (int o = 32; o > 0; o >>= 1) {
                    const u64 other = __shfl_xor(best, o, WAVE);
                    best = other > best ? other : best;
                }
                if (head == best) ++next;                      // keys differ, but where there is none
                if (lane == 0) top[i] = best;
            }
        }
        __syncthreads();
    }
    Sums t{lanes_max(s[0]), s[1], s[2]}, mine{s[0], s[1], s[2]};
    sums_to(mine, t.M, a.c);
    t.S = wave_sum(mine.S);
    t.Y = wave_sum(mine.Y);
    if (a.parts > 1) {
        if (tid == 0) *(f32x4*)(a.sums + (int64_t)blockIdx.x * 4) = f32x4{t.M, t.S, t.Y, 0.f};
    } else {
        logprob_finish<T, LP_JOIN_THREADS>(a, row, t, s_top, given);
    }
}

// ---------------------------------------------------------------- launches
struct LogprobPlan { int threads, chunks; unsigned parts, span; };
static unsigned parts_of(int64_t n, int span) { return (unsigned)((n + span - 1) / span); }
static LogprobPlan logprob_plan(const LogprobArgs& a)
{
    const int v = a.dtype == DT_F32 ? 4 : 8;
    const bool aligned = ((uintptr_t)a.logits & 15) == 0 && a.row_stride % v == 0;
    const int64_t n = (int64_t)a.n + (aligned ? 0 : v - 1);
    // 256 threads, up to 32 logits each: as many parts as that makes, or, where they would not fill the chip, more of fewer logits.
    LogprobPlan p{256, 1, parts_of(n, 256 * v), 0};
    const int most = 32 / v;
    while (p.chunks < most && p.parts > 1 && (p.parts > LP_JOIN || (int64_t)p.parts * a.rows > 256)) p.parts = parts_of(n, 256 * v * (p.chunks *= 2));
    // Rows of several such parts: more threads save the second launch.  us of a call by such parts / with more threads, k 20: bf16, 2048 rows of 50272 64.2 / 47.6, 256 rows
    // 16.2 / 10.7, 1 row 9.6 / 8.2, 700 of 128256 (two parts) 53.1 / 43.0, 1000 of 12000 17.4 / 11.5; float, a row a CU at most: 1 row of 50272 9.5 / 7.9, 64 rows 12.5 / 9.4,
    // 256 rows 18.7 / 12.9, but 300 rows 20.4 / 20.1, 512 27.1 / 24.0, 1000 43.5 / 43.9, 2000 78.5 / 81.3, 256 of 64000 (two parts) 20.6 / 22.5.
    if (n > 256 * 32) {
        const int chunks = a.dtype == DT_F32 ? 13 : 8, threads = a.dtype == DT_BF16 && n <= 512 * v * chunks ? 512 : 1024;
        const unsigned parts = parts_of(n, threads * v * chunks);
        if (a.dtype == DT_F32 ? parts == 1 && a.rows <= 256 : parts == 1 || (int64_t)parts * a.rows >= 192) p = LogprobPlan{threads, chunks, parts, 0};
    }
    p.span = (unsigned)((n + p.parts - 1) / p.parts + 64 * v - 1) / (64 * v) * (64 * v);       // equal ones, of whole KB
    p.parts = parts_of(n, p.span);
    return p;
}
static size_t level_bytes(int64_t rows, unsigned parts, int k) { return (size_t)rows * parts * (16 + 8 * (size_t)k); }

size_t logprobs_workspace(const LogprobArgs& a)
{
    // whatever the alignment turns out to be
    LogprobArgs worst = a;
    worst.logits = (const void*)1;
    size_t bytes = 0;
    for (const LogprobArgs& b : {a, worst}) {
        size_t need = 0;
        for (unsigned parts = logprob_plan(b).parts; parts > 1; parts = parts_of(parts, LP_JOIN)) need += level_bytes(a.rows, parts, a.k);
        bytes = need > bytes ? need : bytes;
    }
    return bytes;
}

template <typename T> static hipError_t launch_logprobs_t(const LogprobArgs& a, hipStream_t s)
{
    const LogprobPlan p = logprob_plan(a);
    // a launch has fewer than 2^32 threads
    const int64_t fit = MAX_LAUNCH_THREADS / p.threads / p.parts;
    for (int64_t r0 = 0; r0 < a.rows; r0 += fit) {
        const int64_t rows = a.rows - r0 < fit ? a.rows - r0 : fit;
        LogprobKernelArgs k{};
        k.logits = (const T*)a.logits + r0 * a.row_stride;
        k.row_stride = a.row_stride;
        k.n = (unsigned)a.n;
        k.c = (float)((double)a.scale * 1.4426950408889634);
        k.scale = a.scale;
        k.n_tokens = a.n_tokens;
        if (a.n_tokens) {
            k.tokens = a.tokens + r0 * a.n_tokens;
            k.logprobs = a.logprobs + r0 * a.n_tokens;
        }
        k.entropy = a.entropy ? a.entropy + r0 : nullptr;
        k.k = a.k;
        if (a.k) {
            k.top_ids = a.top_ids + r0 * a.k;
            k.top_logprobs = a.top_logprobs + r0 * a.k;
        }
        unsigned char* w = (unsigned char*)a.workspace;
        auto level = [&](unsigned parts) {
            k.parts = parts;
            if (parts <= 1) return;
            k.sums = (float*)w;
            k.lists = (u64*)(w + (size_t)rows * parts * 16);
            w += level_bytes(rows, parts, a.k);
        };
        k.span = p.span;
        level(p.parts);
        const unsigned wgs = (unsigned)(rows * p.parts);
        constexpr int V = 16 / (int)sizeof(T);
        if (p.threads == 1024) logprob_part_kernel<T, 1024, (V == 4 ? 13 : 8)><<<wgs, 1024, 0, s>>>(k);
        else if (p.threads == 512) {
            if constexpr (V == 8) logprob_part_kernel<T, 512, 8><<<wgs, 512, 0, s>>>(k);
        } else if (p.chunks == 1) logprob_part_kernel<T, 256, 1><<<wgs, 256, 0, s>>>(k);
        else if (p.chunks == 2) logprob_part_kernel<T, 256, 2><<<wgs, 256, 0, s>>>(k);
        else if (p.chunks == 4) logprob_part_kernel<T, 256, 4><<<wgs, 256, 0, s>>>(k);
        else if constexpr (V == 4) logprob_part_kernel<T, 256, 8><<<wgs, 256, 0, s>>>(k);
        hipError_t e = hipGetLastError();
        for (unsigned parts = p.parts; e == hipSuccess && parts > 1; parts = k.parts) {
            k.from_parts = parts;
            k.from_sums = k.sums;
            k.from_lists = k.lists;
            level(parts_of(parts, LP_JOIN));
            const unsigned lists = parts < LP_JOIN ? parts : LP_JOIN;
            logprob_join_kernel<T><<<(unsigned)(rows * k.parts), LP_JOIN_THREADS, lists * a.k * sizeof(u64), s>>>(k);
            e = hipGetLastError();
        }
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
hipError_t launch_logprobs(const LogprobArgs& a, hipStream_t s)
{
    if (a.rows <= 0) return hipSuccess;
    return a.dtype == DT_F32 ? launch_logprobs_t<float>(a, s) : launch_logprobs_t<bf16_t>(a, s);
}

}  // namespace exe
