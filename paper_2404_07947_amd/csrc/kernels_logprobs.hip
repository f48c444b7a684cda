// Log probabilities of given tokens, entropy and the largest probabilities, of rows of logits.
//
// With the largest logit M and c = scale * log2 e: z = (x - M) * c, S = sum of 2^z, Y = sum of 2^z z; then log p = (z - log2 S) ln 2 and the
// entropy is (log2 S - Y / S) ln 2.
//  * logprob_part_kernel: a workgroup takes 256 * C chunks of 16 bytes of a row into registers, in one round of loads, and makes the sums and the sorted
//    list of its k best from there: the logits are read once.
//  * logprob_join_kernel: where a row has several parts, adds up their sums and merges their lists, 64 parts at a time.
#include "attn_row.h"
#include "kernels.h"

namespace exe {

typedef unsigned long long u64;
constexpr int LP_THREADS = 256, LP_WAVES = LP_THREADS / WAVE, LP_CAP = LP_THREADS, LP_JOIN = 64;
constexpr float LN2 = 0.69314718055994530942f;

struct LogprobKernelArgs {
    const void* logits; int64_t row_stride;
    unsigned n;
    float c, scale;                        // scale * log2 e
    const int32_t* tokens; int n_tokens;
    float *logprobs, *entropy;
    int k;
    int32_t* top_ids; float* top_logprobs;
    unsigned parts;                        // of a row, that this launch writes
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
__device__ __forceinline__ float key_logit(u64 key)
{
    const unsigned o = (unsigned)(key >> 32);
    return __uint_as_float(o ^ (o >> 31 ? 0x80000000u : 0xffffffffu));
}

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
// Of up to 64 parts, a lane each (the others hold M = -inf, S = Y = 0).  Where a part has no number but -inf its M is -inf, and its sums are 0, or NaN.
__device__ __forceinline__ Sums join_sums(Sums p, float c)
{
    const float M = lanes_max(p.M);
    const bool none = p.M == -INFINITY;
    const float d = fmaxf((p.M - M) * c, -1e30f), w = fast_exp2(d);
    return Sums{M, wave_sum(none ? p.S : p.S * w), wave_sum(none ? p.Y : w * fmaf(p.S, d, p.Y))};
}

// The results of a row, by a workgroup: sums, and the k best keys in LDS (0: there are fewer).
template <typename T> __device__ __forceinline__ void logprob_finish(const LogprobKernelArgs& a, int64_t row, Sums t, const u64* top)
{
    const float L = log2f(t.S) * LN2;
    // in 64 bits: the logits may lie further apart than the largest float
    auto logprob = [&](float x) { return (float)(((double)x - (double)t.M) * (double)a.scale - (double)L); };
    const T* x = (const T*)a.logits + row * a.row_stride;
    for (int i = threadIdx.x; i < a.n_tokens; i += LP_THREADS) {
        const unsigned tok = (unsigned)a.tokens[row * a.n_tokens + i];
        a.logprobs[row * a.n_tokens + i] = tok < a.n ? logprob(to_f32(x[tok])) : NAN;
    }
    if (a.entropy && threadIdx.x == 0) a.entropy[row] = L - t.Y / t.S * LN2;
    if ((int)threadIdx.x < a.k) {
        const u64 key = top[threadIdx.x];
        a.top_ids[row * a.k + threadIdx.x] = key ? (int)~(unsigned)key : -1;
        a.top_logprobs[row * a.k + threadIdx.x] = key ? logprob(key_logit(key)) : -INFINITY;
    }
}

template <typename T, int C> struct LogitPart {
    static constexpr int V = 16 / (int)sizeof(T), N = C * V, SPAN = LP_THREADS * N;
    uint4 raw[C];
    __device__ __forceinline__ float at(int i) const       // i: a constant after unrolling
    {
        const uint4 u = raw[i / V];
        const int w = sizeof(T) == 4 ? i % V : i % V / 2;
        const unsigned d = w == 0 ? u.x : w == 1 ? u.y : w == 2 ? u.z : u.w;
        return sizeof(T) == 4 ? __uint_as_float(d) : i & 1 ? bf16hi(d) : bf16lo(d);
    }
    // place of element i among the part's
    static __device__ __forceinline__ unsigned place(int i) { return (i / V * LP_THREADS + threadIdx.x) * V + i % V; }
    // first: the logit with which the part begins, on 16 bytes; up to V - 1 before the row's first one.  What is not of the row is -inf.
    __device__ __forceinline__ void load(const T* x, unsigned first, unsigned n)
    {
        if (first < n && n - first >= SPAN) {
#pragma unroll
            for (int c = 0; c < C; ++c) raw[c] = load_chunk<true>(x + first + place(c * V));
            return;
        }
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const unsigned i = first + place(c * V);
            if (i < n && n - i >= V) {
                raw[c] = load_chunk<true>(x + i);
            } else {
                unsigned w[4];
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    if constexpr (sizeof(T) == 4) {
                        w[d] = i + d < n ? __float_as_uint(x[i + d]) : 0xff800000u;
                    } else {
                        const unsigned lo = i + 2 * d < n ? ((const uint16_t*)x)[i + 2 * d] : 0xff80u, hi = i + 2 * d + 1 < n ? ((const uint16_t*)x)[i + 2 * d + 1] : 0xff80u;
                        w[d] = lo | hi << 16;
                    }
                }
                raw[c] = uint4{w[0], w[1], w[2], w[3]};
            }
        }
    }
};

// The best keys among those of the part that `take` lets through, at most LP_CAP: sorted by counting, for each, those above it.
__device__ __forceinline__ void sort_keys(const u64* keys, int count, u64* top, int k)
{
    const int tid = threadIdx.x;
    if (tid < count) {
        const u64 mine = keys[tid];
        int above = 0;
        for (int j = 0; j < count; ++j) above += keys[j] > mine;
        if (above < k) top[above] = mine;
    }
    if (tid >= count && tid < k) top[tid] = 0;
}

template <typename T, int C> __global__ __launch_bounds__(LP_THREADS) void logprob_part_kernel(LogprobKernelArgs a)
{
    typedef LogitPart<T, C> Part;
    constexpr int N = Part::N;
    __shared__ u64 s_keys[LP_CAP], s_top[WAVE];
    __shared__ Sums s_sums[LP_WAVES];
    __shared__ float s_least[LP_WAVES];
    __shared__ int s_count, s_counts[48];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = blockIdx.x / a.parts;
    const unsigned part = blockIdx.x - (unsigned)row * a.parts;
    const T* x = (const T*)a.logits + row * a.row_stride;
    const unsigned first = part * Part::SPAN - (unsigned)((uintptr_t)x & 15) / sizeof(T);
    Part p;
    p.load(x, first, a.n);
    if (tid == 0) s_count = 0;
    if (tid < 48) s_counts[tid] = 0;

    float best = p.at(0);
#pragma unroll
    for (int i = 1; i < N; ++i) best = fmaxf(best, p.at(i));
    if (!(best >= -INFINITY)) best = -INFINITY;                // all of them NaN
    const float most = lanes_max(best), R = most == -INFINITY ? 0.f : most * a.c;
    float S = 0.f, Y = 0.f;
    auto add = [&](float z) {
        const float e = fast_exp2(z);
        S += e;
        Y = fmaf(e, fmaxf(z, -1e30f), Y);                      // 0 times minus infinity is 0 here; what is NaN is so in e
    };
    if (fabsf(R) < 0x1p20f) {
        // One operation a logit: z + off = c * x - R, where off = c * M - R, what R was rounded by, is 1/16 at most, and taken out of the sums.
#pragma unroll
        for (int i = 0; i < N; ++i) add(fmaf(p.at(i), a.c, -R));
        const float off = most == -INFINITY ? 0.f : fmaf(most, a.c, -R), w = fast_exp2(-off);
        Y = (Y - off * S) * w;
        S *= w;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) add((p.at(i) - most) * a.c);
    }
    S = wave_sum(S);
    Y = wave_sum(Y);
    if (lane == 0) s_sums[wave] = Sums{most, S, Y};
    if (a.k) {
        // The waves' (k / 4)-th largest of their lanes' best: k logits or more are no smaller than the least of these.
        float b = best, least = most;
        for (int i = 1; i < (a.k + LP_WAVES - 1) / LP_WAVES; ++i) {
            if (lane == __builtin_ctzll(__builtin_amdgcn_ballot_w64(b == least))) b = -INFINITY;
            least = lanes_max(b);
        }
        if (lane == 0) s_least[wave] = least;
    }
    __syncthreads();
    const Sums t = join_sums(lane < LP_WAVES ? s_sums[lane] : Sums{-INFINITY, 0.f, 0.f}, a.c);
    if (a.k) {
        float least = s_least[0];
#pragma unroll
        for (int w = 1; w < LP_WAVES; ++w) least = fminf(least, s_least[w]);
        if (best >= least) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float v = p.at(i);
                if (v >= least && v > -INFINITY) {
                    const int at = atomicAdd(&s_count, 1);     // in any order: they are sorted
                    if (at < LP_CAP) s_keys[at] = logit_key(logit_order(v), first + Part::place(i));
                }
            }
        }
        __syncthreads();
        int count = s_count;
        if (count > LP_CAP) {
            // Many equal ones, or most of a wave's ruled out: the k-th largest, bit by bit, and of those that equal it the lowest places.
            auto count_of = [&](int slot, auto take) {
                int n = 0;
                // a new value to the compiler: it would keep orders and masks of all elements over the loops
#pragma unroll
                for (int c = 0; c < C; ++c) asm volatile("" : "+v"(p.raw[c].x), "+v"(p.raw[c].y), "+v"(p.raw[c].z), "+v"(p.raw[c].w));
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float v = p.at(i);
                    n += v > -INFINITY && take(logit_order(v), Part::place(i));
                }
                if (n) atomicAdd(&s_counts[slot], n);
                __syncthreads();
                return s_counts[slot];
            };
            unsigned kth = 0, last = 0;
            for (int bit = 31; bit >= 0; --bit) {
                const unsigned from = kth | 1u << bit;
                if (count_of(bit, [&](unsigned o, unsigned) { return o >= from; }) >= a.k) kth = from;
            }
            const int equal = a.k - count_of(32, [&](unsigned o, unsigned) { return o > kth; });
            static_assert(Part::SPAN <= 1 << 15, "a count for each bit of a place");
            for (int bit = 14; bit >= 0; --bit) {
                const unsigned below = last | 1u << bit;
                if (count_of(33 + bit, [&](unsigned o, unsigned i) { return o == kth && i < below; }) < equal) last = below;
            }
            if (tid == 0) s_count = 0;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float v = p.at(i);
                const unsigned o = logit_order(v);
                if (v > -INFINITY && (o > kth || (o == kth && Part::place(i) <= last))) s_keys[atomicAdd(&s_count, 1)] = logit_key(o, first + Part::place(i));
            }
            __syncthreads();
            count = a.k;
        }
        if (a.parts > 1) {
            sort_keys(s_keys, count, a.lists + (int64_t)blockIdx.x * a.k, a.k);
        } else {
            sort_keys(s_keys, count, s_top, a.k);
            __syncthreads();
        }
    }
    if (a.parts > 1) {
        if (tid == 0) *(f32x4*)(a.sums + (int64_t)blockIdx.x * 4) = f32x4{t.M, t.S, t.Y, 0.f};
    } else {
        logprob_finish<T>(a, row, t, s_top);
    }
}

// Lists i of up to 64, sorted, each of k keys: the k best of them all.  What the m-th of every list (k of them or more together) and the k-th of
// one are not below is left out, the rest sorted by counting; if that leaves too many, one wave takes the largest of the lists' heads k times.
template <typename T> __global__ __launch_bounds__(LP_THREADS) void logprob_join_kernel(LogprobKernelArgs a)
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
        for (int i = tid; i < lists * a.k; i += LP_THREADS) s_all[i] = in[i];
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const u64 l = __shfl_xor(low, o, WAVE), h = __shfl_xor(high, o, WAVE);
            low = l < low ? l : low;
            high = h > high ? h : high;
        }
        u64 least = low > high ? low : high;
        if (!least) least = 1;                                 // 0 is no key
        __syncthreads();
        for (int i = tid; i < lists * a.k; i += LP_THREADS)
            if (s_all[i] >= least) {
                const int at = atomicAdd(&s_count, 1);
                if (at < LP_CAP) s_keys[at] = s_all[i];
            }
        __syncthreads();
        u64* top = a.parts > 1 ? a.lists + (int64_t)blockIdx.x * a.k : s_top;
        if (s_count <= LP_CAP) {
            sort_keys(s_keys, s_count, top, a.k);
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
    const Sums t = join_sums(Sums{s[0], s[1], s[2]}, a.c);
    if (a.parts > 1) {
        if (tid == 0) *(f32x4*)(a.sums + (int64_t)blockIdx.x * 4) = f32x4{t.M, t.S, t.Y, 0.f};
    } else {
        logprob_finish<T>(a, row, t, s_top);
    }
}

// ---------------------------------------------------------------- launches
struct LogprobPlan { int chunks; unsigned parts; };
static unsigned parts_of(int64_t n, int span) { return (unsigned)((n + span - 1) / span); }
static LogprobPlan logprob_plan(const LogprobArgs& a)
{
    const int v = a.dtype == DT_F32 ? 4 : 8, most = a.dtype == DT_F32 ? 8 : 4;
    const bool aligned = ((uintptr_t)a.logits & 15) == 0 && a.row_stride % v == 0;
    const int64_t n = (int64_t)a.n + (aligned ? 0 : v - 1);
    LogprobPlan p{1, parts_of(n, LP_THREADS * v)};
    while (p.chunks < most && p.parts > 1 && (p.parts > LP_JOIN || (int64_t)p.parts * a.rows > 256)) p.parts = parts_of(n, LP_THREADS * v * (p.chunks *= 2));
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
    const int64_t fit = MAX_LAUNCH_THREADS / LP_THREADS / p.parts;
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
        level(p.parts);
        const unsigned wgs = (unsigned)(rows * p.parts);
        if (p.chunks == 1) logprob_part_kernel<T, 1><<<wgs, LP_THREADS, 0, s>>>(k);
        else if (p.chunks == 2) logprob_part_kernel<T, 2><<<wgs, LP_THREADS, 0, s>>>(k);
        else if (p.chunks == 4) logprob_part_kernel<T, 4><<<wgs, LP_THREADS, 0, s>>>(k);
        else if constexpr (sizeof(T) == 4) logprob_part_kernel<T, 8><<<wgs, LP_THREADS, 0, s>>>(k);
        hipError_t e = hipGetLastError();
        for (unsigned parts = p.parts; e == hipSuccess && parts > 1; parts = k.parts) {
            k.from_parts = parts;
            k.from_sums = k.sums;
            k.from_lists = k.lists;
            level(parts_of(parts, LP_JOIN));
            const unsigned lists = parts < LP_JOIN ? parts : LP_JOIN;
            logprob_join_kernel<T><<<(unsigned)(rows * k.parts), LP_THREADS, lists * a.k * sizeof(u64), s>>>(k);
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
