// Norms of the heads of queries and keys, with their rotary positions in the same pass: of rows alone, and of a chunk of new tokens on
// their way to a paged cache.
#include "kernels.h"
#include "paged.h"
#include "rotary.h"

namespace exe {

// A head x of dh elements becomes y = gain * (x - mean) / sqrt(mean of (x - mean)^2 + eps), or without the mean, and pair p of its first
// rot elements is then turned by pos * inv_freq[p], as rotary_kernel does it.  DH / (2 * EPL) lanes hold a head, two chunks of EPL elements
// each, which are those of its turned pairs: statistics, gain and turn are made in registers, in float, and rounded once.  Since
// a wave's 64 lanes are whole heads, a lane has the same place in each of its heads, and keeps its sines and cosines.
//
// Bound by memory where tokens are many: every element is read once and written once.  4000 tokens of OPT-13B's 120 heads x 128 in chunks 54 us, 4.3 TB/s
// (rotary_append_kernel 50, a large copy 46); two slots in flight a lane, as there, 59, and three 65, for their registers take away waves; ordinary
// loads and, into the cache, stores (nontemporal ones 56 and 57).  4099 x 20 x 64 in float 11 us.  Few tokens: the call, of which the
// kernel takes 2.8 us (one token) or 4.4 (64 sequences; their place in the cache is found while the rows are on their way).
template <int P> __device__ __forceinline__ float head_sum(float d)
{
    if constexpr (P == 64) return wave_sum(d);
    else if constexpr (P == 4) return d += dpp_move<0xB1>(d), d + dpp_move<0x4E>(d);
    else return row_sum<P>(d);
}

// The N elements of this lane, at(0) .. at(N - 1), of a head of DH on DH / N lanes, without gain.
template <int DH, int N, typename F> __device__ __forceinline__ void head_norm(F at, float (&v)[N], bool rms, float eps)
{
    constexpr int P = DH / N;
    auto sum = [&](auto f) {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < N; ++e) s += f(v[e]);
        return head_sum<P>(s);
    };
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = at(e);
    auto center = [&]() {
        // a second round takes away what the first mean's rounding left: it may be large beside the deviations
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float mean = sum([](float a) { return a; }) * (1.f / DH);
#pragma unroll
            for (int e = 0; e < N; ++e) v[e] -= mean;
        }
    };
    if (!rms) center();
    const float var = sum([](float a) { return a * a; }) * (1.f / DH) + eps;
    float r = rsqrtf(var);
    if (!(var > 1e-30f && var < INFINITY)) {
        // squares that pass a float's ends (rows of 2^64 and more, or of 2^-50 and less beside an eps as small): all of it again, times a power of
        // two that takes the largest of them to 1.  An infinite one makes the others 0 and itself NaN.
        float most = sqrtf(eps);
#pragma unroll
        for (int e = 0; e < N; ++e) most = fmaxf(most, fabsf(at(e)));
#pragma unroll
        for (int o = P / 2; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o, WAVE));
        const int ex = __builtin_amdgcn_frexp_expf(most);
        const float s = __builtin_amdgcn_ldexpf(1.f, ex < -126 ? 126 : -ex);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = at(e) * s;
        if (!rms) center();
        // Equal elements have no deviations, and are 0 by an eps that the scale takes below a float (a deviation that is one is 2^-25 of the largest element or more)
        const float scaled = sum([](float a) { return a * a; }) * (1.f / DH) + eps * s * s;
        r = eps > 0.f && scaled < 0x1p-100f ? 0.f : rsqrtf(scaled);
    }
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] *= r;
}

template <typename T, int DH, int EPL, bool INTERLEAVED, bool APPEND>
__global__ __launch_bounds__(ROT_WAVES * 64) void head_norm_kernel(HeadNormArgs a, int parts)
{
    typedef Elems<T, EPL> E;
    constexpr int PER = DH / (2 * EPL), HEADS = 64 / PER, N = 2 * EPL;
    __shared__ float2 s_cs[ROT_WAVES][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t unit = (int64_t)blockIdx.x * ROT_WAVES + wave;
    const int t = (int)(unit / parts), part = (int)(unit - (int64_t)t * parts);
    if (t >= a.tokens) return;                     // a whole wave; nothing below waits for another one
    const T* xr = (const T*)a.x + t * a.x_stride;
    const int half = a.rot / 2, pair = lane % PER * EPL;
    const bool turn = pair < half;
    const int c0 = INTERLEAVED || !turn ? 2 * pair : pair, c1 = INTERLEAVED || !turn ? 2 * pair + EPL : pair + half;
    const int normed = a.H + a.Hkv, step = parts * HEADS;
    int heads = a.H + 2 * a.Hkv, h0 = (APPEND && !a.out ? a.H : 0) + part * HEADS + lane / PER;

    E x[2], gain[2];
    auto load = [&](int h) {
        if (h >= heads) return;
        x[0] = *(const E*)(xr + (int64_t)h * DH + c0);
        x[1] = *(const E*)(xr + (int64_t)h * DH + c1);
        const T* g = (const T*)(h < a.H ? a.q_gain : a.k_gain);
        if (!g || h >= normed) return;
        g += a.gain_per_head ? (int64_t)(h < a.H ? h : h - a.H) * DH : 0;
        gain[0] = *(const E*)(g + c0);
        gain[1] = *(const E*)(g + c1);
    };
    load(h0);                                      // on its way while the token's place is found
    int at = 0, blk = 0;
    if constexpr (APPEND) {
        const ChunkSeq sq = seq_of_token(a.cu, a.n_seqs, t, lane);
        if (sq.b < 0) return;
        at = a.len[sq.b] - sq.n + (t - sq.t0);     // position in the cache
        blk = a.table.block(sq.b, at);
        if (blk < 0) heads = a.H;                  // the table gives no row
    }
    float2 cs[EPL];
    if (a.rot) {
        float2* all = s_cs[wave];
        if (lane < half) all[lane] = rotary_cs(a.pos ? a.pos[t] : at, a.inv_freq[lane], a.amplitude);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int e = 0; e < EPL; ++e) cs[e] = all[pair + e < half ? pair + e : 0];
    }
    T* qr = (T*)a.out + t * a.out_stride;
    const int rows = APPEND ? 1 << a.table.shift : 0;
    T* kd = APPEND ? (T*)a.kv_blocks + ((int64_t)blk * 2 * a.Hkv * rows + (at & (rows - 1))) * DH : nullptr;   // head g's key at kd + g * rows * DH
    while (h0 < heads) {
        if (!APPEND || h0 < normed) {              // (asked without need, float rows' stores came out with an address over their data)
            float v[N];
            head_norm<DH, N>([&](int e) { return to_f32(x[e / EPL].v[e % EPL]); }, v, a.rms, a.eps);
            if (h0 < a.H ? a.q_gain : a.k_gain) {
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] *= to_f32(gain[e / EPL].v[e % EPL]);
            }
            if (turn) {
#pragma unroll
                for (int e = 0; e < EPL; ++e) {
                    if (INTERLEAVED && pair + e >= half) continue;               // rot ends inside the chunks
                    float &p = v[INTERLEAVED ? 2 * e : e], &q = v[INTERLEAVED ? 2 * e + 1 : EPL + e];
                    const float b = p, c = q;
                    p = b * cs[e].x - c * cs[e].y;
                    q = c * cs[e].x + b * cs[e].y;
                }
            }
#pragma unroll
            for (int e = 0; e < N; ++e) x[e / EPL].v[e % EPL] = from_f32<T>(v[e]);
        }
        T* to = !APPEND || h0 < a.H ? qr + (int64_t)h0 * DH : kd + (int64_t)(h0 - a.H) * rows * DH;
        if constexpr (!APPEND && sizeof(E) == 16) {
            typedef unsigned v4u __attribute__((ext_vector_type(4)));
            __builtin_nontemporal_store(__builtin_bit_cast(v4u, x[0]), (v4u*)(to + c0));
            __builtin_nontemporal_store(__builtin_bit_cast(v4u, x[1]), (v4u*)(to + c1));
        } else {
            *(E*)(to + c0) = x[0];
            *(E*)(to + c1) = x[1];
        }
        h0 += step;
        load(h0);
    }
}

template <typename T, int DH, bool APPEND> static hipError_t launch_head_norm_t(const HeadNormArgs& a, hipStream_t s)
{
    constexpr int W = 16 / (int)sizeof(T);
    const bool wide = rotary_wide<T>(a.rot, a.interleaved) && aligned_rows(a.x, a.x_stride, sizeof(T)) && aligned_rows(a.out, a.out_stride, sizeof(T)) &&
                      aligned_rows(a.q_gain, 0, 1) && aligned_rows(a.k_gain, 0, 1);
    const int64_t heads = (APPEND && !a.out ? 0 : a.H) + 2 * (int64_t)a.Hkv;
    const int parts = rotary_parts(a.tokens, heads * DH / (wide ? 2 * W : 2));
    const int64_t wgs = ((int64_t)a.tokens * parts + ROT_WAVES - 1) / ROT_WAVES;
    if (wgs * ROT_WAVES * 64 > MAX_LAUNCH_THREADS) return hipErrorInvalidValue;
#define EXE_HEAD_NORM(EPL, IL) head_norm_kernel<T, DH, EPL, IL, APPEND><<<(unsigned)wgs, ROT_WAVES * 64, 0, s>>>(a, parts)
    if (wide) { if (a.interleaved) EXE_HEAD_NORM(W, true); else EXE_HEAD_NORM(W, false); }
    else { if (a.interleaved) EXE_HEAD_NORM(1, true); else EXE_HEAD_NORM(1, false); }
#undef EXE_HEAD_NORM
    return hipGetLastError();
}
template <bool APPEND> static hipError_t launch_head_norm_of(const HeadNormArgs& a, hipStream_t s)
{
    if (a.dtype == DT_F32) return a.dh == 64 ? launch_head_norm_t<float, 64, APPEND>(a, s) : launch_head_norm_t<float, 128, APPEND>(a, s);
    return a.dh == 64 ? launch_head_norm_t<bf16_t, 64, APPEND>(a, s) : launch_head_norm_t<bf16_t, 128, APPEND>(a, s);
}
hipError_t launch_head_norm(const HeadNormArgs& a, hipStream_t s)
{
    if (a.tokens <= 0 || (a.kv_blocks && a.n_seqs <= 0)) return hipSuccess;
    return a.kv_blocks ? launch_head_norm_of<true>(a, s) : launch_head_norm_of<false>(a, s);
}

}  // namespace exe
