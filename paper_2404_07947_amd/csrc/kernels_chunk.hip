// Attention of a chunk of new tokens over a paged cache.
#include "attn_row.h"
#include "kernels.h"

namespace exe {

// Keys first .. last - 1 that a row at position p sees.
struct KeyRange { int first, last; };
__device__ __forceinline__ KeyRange keys_of(int p, int window) { return KeyRange{window > 0 && p >= window ? p - window + 1 : 0, p + 1 > 0 ? p + 1 : 0}; }

// One query row by one wave over keys first .. last - 1, 64 at a time: a lane takes a key for the scores, and features lane, lane + 64
// of the result.  kv: this head's keys of block 0; rows of a block's values lie v_off elements behind its keys; sc: the scale for exp2.
template <typename T, int DH>
__device__ __forceinline__ void chunk_row(const T* q, const T* kv, int64_t block_elems, int64_t v_off, const PagedTable& tbl, int b, KeyRange r, float sc,
                                          int lane, T* out)
{
    float m = -INFINITY, l = 0.f, acc[DH / 64] = {};
    bool bad = false;
    const int mask = (1 << tbl.shift) - 1;
    for (int j0 = r.first; j0 < r.last; j0 += 64) {
        int j = j0 + lane, cnt = r.last - j0 < 64 ? r.last - j0 : 64, jj = j < r.last ? j : r.last - 1;
        int blk = tbl.block(b, jj);
        bad |= blk < 0;
        const int64_t at = (blk < 0 ? 0 : blk) * block_elems + (jj & mask) * DH;
        const T* k = kv + at;
        float s = 0.f;
#pragma unroll 4
        for (int e = 0; e < DH; ++e) s = fmaf(to_f32(q[e]), to_f32(k[e]), s);
        s = j < r.last ? s * sc : -INFINITY;
        float mx = wave_max(fmaxf(m, s)), mref = mx == -INFINITY ? 0.f : mx;
        float alpha = fast_exp2(m - mref), p = fast_exp2(s - mref);
        l = l * alpha + wave_sum(p);
#pragma unroll
        for (int f = 0; f < DH / 64; ++f) acc[f] *= alpha;
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
    for (int f = 0; f < DH / 64; ++f) out[lane + f * 64] = from_f32<T>(r.last > r.first ? acc[f] / l : 0.f);
}

template <typename T, int DH>
__global__ __launch_bounds__(256) void chunk_row_kernel(const int32_t* __restrict__ cu, int n_seqs, int tokens, const T* __restrict__ q, int64_t q_stride,
                                                        const T* __restrict__ kv_blocks, PagedTable tbl, const int32_t* __restrict__ len, int H, int Hkv,
                                                        float scale, int window, T* __restrict__ out, int64_t out_stride)
{
    int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t unit = (int64_t)blockIdx.x * 4 + wave;
    int t = (int)(unit / H), h = (int)(unit - (int64_t)t * H);
    if (t >= tokens) return;
    ChunkSeq sq = seq_of_token(cu, n_seqs, t, lane);
    if (sq.b < 0) return;
    int p = len[sq.b] - sq.n + (t - sq.t0);
    const int64_t head = (int64_t)DH << tbl.shift;
    chunk_row<T, DH>(q + t * q_stride + h * DH, kv_blocks + h / (H / Hkv) * head, 2 * Hkv * head, Hkv * head, tbl, sq.b, keys_of(p, window), scale * LOG2E, lane,
                     out + t * out_stride + h * DH);
}

template <typename T, int DH> static hipError_t launch_chunk(const ChunkAttnArgs& a, hipStream_t s)
{
    int64_t wgs = ((int64_t)a.tokens * a.H + 3) / 4;
    if (wgs * 256 > MAX_LAUNCH_THREADS) return hipErrorInvalidValue;
    chunk_row_kernel<T, DH><<<(unsigned)wgs, 256, 0, s>>>(a.cu, a.n_seqs, a.tokens, (const T*)a.q, a.q_stride, (const T*)a.kv_blocks, a.table, a.len, a.H, a.Hkv,
                                                         a.scale, a.window, (T*)a.out, a.out_stride);
    return hipGetLastError();
}

size_t chunk_attn_workspace(const ChunkAttnArgs&) { return 0; }

hipError_t launch_chunk_attn(const ChunkAttnArgs& a, hipStream_t s)
{
    if (a.dtype == DT_F32) return a.dh == 64 ? launch_chunk<float, 64>(a, s) : launch_chunk<float, 128>(a, s);
    return a.dh == 64 ? launch_chunk<bf16_t, 64>(a, s) : launch_chunk<bf16_t, 128>(a, s);
}

}  // namespace exe
