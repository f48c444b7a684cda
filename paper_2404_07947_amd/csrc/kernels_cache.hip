// What is done to a paged cache beside attention: rotary positions and the append of a chunk's keys and values, copies of pages.
#include "kernels.h"
#include "paged.h"

namespace exe {

// ---------------------------------------------------------------- rotary positions
// Pair p of a head is turned by the angle pos * inv_freq[p]: (a, b) -> amplitude * (a cos - b sin, b cos + a sin).  The pair's two
// elements are 2p, 2p + 1 (interleaved) or p, p + rot / 2; elements from rot on pass through, bit by bit.
//
// Every head of a token is turned by the same rot / 2 <= 64 angles, so a wave takes one token (or a part of its heads), makes an angle a
// lane, and goes over its heads with the sines and cosines in LDS: per 32 bytes moved a lane then spends its time on memory alone.
// Angles are made in turns, in 64 bits with the products' rounding errors carried along (a position of 2^31 keeps its angle to 1e-15), cut
// to an eighth of a turn either side of a quarter, and only then rounded to float: wherever the position is, that moves the angle by
// 2 pi 2^-28 = 2.3e-8 at most, to which the sine and cosine add their own rounding (2^-25 and more; together 6.7e-8 at most over 2^22 angles).
// (A float angle is 0.06 off at position 10^6.)
__device__ __forceinline__ float2 rotary_cs(int pos, double freq, float amplitude)
{
    constexpr double INV = 0.15915494309189535, INV_LO = -9.839338337591474e-18;       // 1 / 2 pi
    double p = (double)pos * freq, pe = fma((double)pos, freq, -p);
    double t = p * INV, te = fma(p, INV, -t) + fma(p, INV_LO, pe * INV);
    double f = (t - rint(t)) + te;                  // turns, half a turn either side of 0
    double quarter = rint(4.0 * f);
    float r = (float)(f - 0.25 * quarter), s, c;
    sincospif(2.f * r, &s, &c);
    int k = (int)quarter & 3;
    float cs = k & 1 ? -s : c, sn = k & 1 ? c : s;
    if (k & 2) { cs = -cs; sn = -sn; }
    return float2{cs * amplitude, sn * amplitude};
}

constexpr int ROT_WAVES = 4, ROT_U = 2;   // waves of a workgroup, each with a token (or part of one) of its own; slots in flight per lane
template <typename T, int N> struct __align__(sizeof(T) * N) Elems { T v[N]; };

// Slot s of a head: 2 * EPL elements, either EPL pairs or EPL x 2 elements that pass through, loaded and stored as two chunks.  Both
// chunks are the same thread's, so out may be x itself.
template <typename T, int EPL, bool INTERLEAVED> struct RotarySlot {
    typedef Elems<T, EPL> E;
    E a, b;
    int pair, c0, c1;                     // first pair; the chunks' places
    bool turn;
    __device__ __forceinline__ void load(const T* x, int slot, int rot)
    {
        pair = slot * EPL;
        turn = pair < rot / 2;
        c0 = INTERLEAVED || !turn ? 2 * pair : pair;
        c1 = INTERLEAVED || !turn ? 2 * pair + EPL : pair + rot / 2;
        a = *(const E*)(x + c0);
        b = *(const E*)(x + c1);
    }
    // NT: nontemporal
    template <bool NT> __device__ __forceinline__ void store(T* out, int rot, const float2* cs)
    {
        if (turn) {
#pragma unroll
            for (int e = 0; e < EPL; ++e) {
                if (INTERLEAVED && pair + e >= rot / 2) continue;                // rot ends inside the slot
                float2 w = cs[pair + e];
                T& u = INTERLEAVED ? (2 * e < EPL ? a.v[2 * e < EPL ? 2 * e : 0] : b.v[2 * e >= EPL ? 2 * e - EPL : 0]) : a.v[e];
                T& v = INTERLEAVED ? (2 * e + 1 < EPL ? a.v[2 * e + 1 < EPL ? 2 * e + 1 : 0] : b.v[2 * e + 1 >= EPL ? 2 * e + 1 - EPL : 0]) : b.v[e];
                float p = to_f32(u), q = to_f32(v);
                u = from_f32<T>(p * w.x - q * w.y);
                v = from_f32<T>(q * w.x + p * w.y);
            }
        }
        if constexpr (NT && sizeof(E) == 16) {
            typedef unsigned v4u __attribute__((ext_vector_type(4)));
            __builtin_nontemporal_store(__builtin_bit_cast(v4u, a), (v4u*)(out + c0));
            __builtin_nontemporal_store(__builtin_bit_cast(v4u, b), (v4u*)(out + c1));
        } else {
            *(E*)(out + c0) = a;
            *(E*)(out + c1) = b;
        }
    }
};

template <typename T, int EPL, bool INTERLEAVED>
__global__ __launch_bounds__(ROT_WAVES * 64) void rotary_kernel(const T* x, int64_t x_stride, int tokens, int parts, int heads, int dh, int rot,
                                                                const int32_t* __restrict__ pos, const double* __restrict__ inv_freq,
                                                                float amplitude, T* out, int64_t out_stride)
{
    __shared__ float2 s_cs[ROT_WAVES][64];
    int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t unit = (int64_t)blockIdx.x * ROT_WAVES + wave;
    int t = (int)(unit / parts), part = (int)(unit - (int64_t)t * parts);
    if (t >= tokens) return;                       // a whole wave; nothing below waits for another one
    float2* cs = s_cs[wave];
    if (lane < rot / 2) cs[lane] = rotary_cs(pos[t], inv_freq[lane], amplitude);
    __builtin_amdgcn_wave_barrier();
    const T* xr = x + t * x_stride;
    T* yr = out + t * out_stride;
    int per_head = dh / (2 * EPL), shift = 31 - __builtin_clz(per_head);
    const int end = heads << shift;
    for (int i0 = part * 64 + lane; i0 < end; i0 += parts * 64 * ROT_U) {
        RotarySlot<T, EPL, INTERLEAVED> s[ROT_U];
#pragma unroll
        for (int u = 0; u < ROT_U; ++u) {
            int i = i0 + u * parts * 64;
            if (i < end) s[u].load(xr + (i >> shift) * dh, i & (per_head - 1), rot);
        }
#pragma unroll
        for (int u = 0; u < ROT_U; ++u) {
            int i = i0 + u * parts * 64;
            if (i < end) s[u].template store<true>(yr + (i >> shift) * dh, rot, cs);
        }
    }
}

// The same for a chunk of new tokens over a paged cache: queries to q_out, keys turned and values as they are to the row of their
// position's block.  Rows behind the last sequence are left alone, and so is a row of the cache that the table does not give (a position
// before 0 or past the table, a block outside of the pool).
template <typename T, int EPL, bool INTERLEAVED>
__global__ __launch_bounds__(ROT_WAVES * 64) void rotary_append_kernel(
    const int32_t* __restrict__ cu, int n_seqs, int tokens, int parts, const T* qkv, int64_t row_stride, int H, int Hkv, int dh, int rot,
    const int32_t* __restrict__ pos, const double* __restrict__ inv_freq, float amplitude, T* __restrict__ kv_blocks, PagedTable tbl,
    const int32_t* __restrict__ len, T* q_out, int64_t q_out_stride)
{
    __shared__ float2 s_cs[ROT_WAVES][64];
    int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t unit = (int64_t)blockIdx.x * ROT_WAVES + wave;
    int t = (int)(unit / parts), part = (int)(unit - (int64_t)t * parts);
    if (t >= tokens) return;
    ChunkSeq sq = seq_of_token(cu, n_seqs, t, lane);
    if (sq.b < 0) return;
    int at = len[sq.b] - sq.n + (t - sq.t0);        // position in the cache
    int blk = tbl.block(sq.b, at);
    float2* cs = s_cs[wave];
    if (lane < rot / 2) cs[lane] = rotary_cs(pos ? pos[t] : at, inv_freq[lane], amplitude);
    __builtin_amdgcn_wave_barrier();
    const T* xr = qkv + t * row_stride;
    T* qr = q_out + t * q_out_stride;
    const int rows = 1 << tbl.shift;
    T* kd = kv_blocks + ((int64_t)blk * 2 * Hkv * rows + (at & (rows - 1))) * dh;      // head g's key at kd + g * rows * dh
    int per_head = dh / (2 * EPL), shift = 31 - __builtin_clz(per_head);
    int first = q_out ? 0 : H, last = blk >= 0 ? H + 2 * Hkv : H;
    const int end = last << shift;
    for (int i0 = (first << shift) + part * 64 + lane; i0 < end; i0 += parts * 64 * ROT_U) {
        RotarySlot<T, EPL, INTERLEAVED> s[ROT_U];
#pragma unroll
        for (int u = 0; u < ROT_U; ++u) {
            int i = i0 + u * parts * 64, h = i >> shift;
            if (i < end) s[u].load(xr + h * dh, i & (per_head - 1), h < H + Hkv ? rot : 0);
        }
#pragma unroll
        for (int u = 0; u < ROT_U; ++u) {
            int i = i0 + u * parts * 64, h = i >> shift;
            if (i < end) s[u].template store<false>(h < H ? qr + h * dh : kd + (int64_t)(h - H) * rows * dh, h < H + Hkv ? rot : 0, cs);
        }
    }
}

// Parts of a token: 16384 waves, two for each that the chip holds, where tokens are few; up to one per 64 slots.
static int rotary_parts(int tokens, int64_t slots)
{
    int64_t most = (slots + 63) / 64, want = (16384 + tokens - 1) / tokens;
    return (int)(most < want ? most : want);
}
static bool aligned_rows(const void* p, int64_t stride, int esz) { return !p || (((uintptr_t)p & 15) == 0 && stride * esz % 16 == 0); }

// Chunks of 16 bytes where rows and (half layout) both halves of the turned part begin on 16 bytes, else single elements.
template <typename T> static bool rotary_wide(int rot, int interleaved) { return interleaved || rot % (32 / (int)sizeof(T)) == 0; }

template <typename T> static hipError_t launch_rotary_t(const RotaryArgs& a, hipStream_t s)
{
    constexpr int W = 16 / (int)sizeof(T);
    bool wide = rotary_wide<T>(a.rot, a.interleaved) && aligned_rows(a.x, a.x_stride, sizeof(T)) && aligned_rows(a.out, a.out_stride, sizeof(T));
    int parts = rotary_parts(a.tokens, (int64_t)a.heads * a.dh / (wide ? 2 * W : 2));
    int64_t wgs = ((int64_t)a.tokens * parts + ROT_WAVES - 1) / ROT_WAVES;
    if (wgs * ROT_WAVES * 64 > MAX_LAUNCH_THREADS) return hipErrorInvalidValue;
#define EXE_ROTARY(EPL, IL)                                                                                                              \
    rotary_kernel<T, EPL, IL><<<(unsigned)wgs, ROT_WAVES * 64, 0, s>>>((const T*)a.x, a.x_stride, a.tokens, parts, a.heads, a.dh, a.rot, a.pos, \
                                                                       a.inv_freq, a.amplitude, (T*)a.out, a.out_stride)
    if (wide) { if (a.interleaved) EXE_ROTARY(W, true); else EXE_ROTARY(W, false); }
    else { if (a.interleaved) EXE_ROTARY(1, true); else EXE_ROTARY(1, false); }
#undef EXE_ROTARY
    return hipGetLastError();
}
hipError_t launch_rotary(const RotaryArgs& a, hipStream_t s)
{
    if (a.tokens <= 0 || a.heads <= 0) return hipSuccess;
    return a.dtype == DT_F32 ? launch_rotary_t<float>(a, s) : launch_rotary_t<bf16_t>(a, s);
}

template <typename T> static hipError_t launch_rotary_append_t(const RotaryAppendArgs& a, hipStream_t s)
{
    constexpr int W = 16 / (int)sizeof(T);
    bool wide = rotary_wide<T>(a.rot, a.interleaved) && aligned_rows(a.qkv, a.row_stride, sizeof(T)) && aligned_rows(a.q_out, a.q_out_stride, sizeof(T));
    int heads = (a.q_out ? a.H : 0) + 2 * a.Hkv, parts = rotary_parts(a.tokens, (int64_t)heads * a.dh / (wide ? 2 * W : 2));
    int64_t wgs = ((int64_t)a.tokens * parts + ROT_WAVES - 1) / ROT_WAVES;
    if (wgs * ROT_WAVES * 64 > MAX_LAUNCH_THREADS) return hipErrorInvalidValue;
#define EXE_APPEND(EPL, IL)                                                                                                                  \
    rotary_append_kernel<T, EPL, IL><<<(unsigned)wgs, ROT_WAVES * 64, 0, s>>>(a.cu, a.n_seqs, a.tokens, parts, (const T*)a.qkv, a.row_stride, a.H, a.Hkv, \
                                                                              a.dh, a.rot, a.pos, a.inv_freq, a.amplitude, (T*)a.kv_blocks, a.table, a.len, \
                                                                              (T*)a.q_out, a.q_out_stride)
    if (wide) { if (a.interleaved) EXE_APPEND(W, true); else EXE_APPEND(W, false); }
    else { if (a.interleaved) EXE_APPEND(1, true); else EXE_APPEND(1, false); }
#undef EXE_APPEND
    return hipGetLastError();
}
hipError_t launch_rotary_append(const RotaryAppendArgs& a, hipStream_t s)
{
    if (a.tokens <= 0 || a.n_seqs <= 0) return hipSuccess;
    return a.dtype == DT_F32 ? launch_rotary_append_t<float>(a, s) : launch_rotary_append_t<bf16_t>(a, s);
}

// ---------------------------------------------------------------- copies of pages
// Positions 0 .. rows - 1 of every head's keys and values, of every layer.  The list travels in the kernel's arguments: nothing is
// allocated or staged, and a captured launch keeps its own.  A workgroup moves COPY_PIECE bytes of one (copy, layer), in which the runs
// of the heads (rows * row_bytes each; one run where whole blocks are copied) follow each other.  Stores are nontemporal, loads are not: a
// fork reads one source for every copy.  90 blocks of 1.3 MB in 8 layers, 1.9 GB moved: 362 us (5.2 TB/s; a plain copy of 2 GiB 4.9), with
// ordinary stores 369; 37 of 64 positions of a block to 8 others, 40 layers, 273 MB: 57 and 79 us.
constexpr int COPY_MAX = 256, COPY_THREADS = 256, COPY_U = 16, COPY_PIECE = COPY_THREADS * COPY_U * 16;
struct CopyList { BlockCopy c[COPY_MAX]; };

__global__ __launch_bounds__(COPY_THREADS) void copy_blocks_kernel(CopyList list, unsigned char* pool, int64_t layer_bytes, int64_t block_bytes, int layers,
                                                                   int block_rows, int row_bytes, int runs, unsigned pieces)
{
    typedef unsigned v4u __attribute__((ext_vector_type(4)));
    unsigned piece = blockIdx.x % pieces, rest = blockIdx.x / pieces, layer = rest % layers;
    // straight from the arguments in memory, of which the list is the first: an array that is indexed there would go to registers
    const auto* entry = (const __attribute__((address_space(4))) int32_t*)__builtin_amdgcn_kernarg_segment_ptr() + 3 * (rest / layers);
    const int c_src = entry[0], c_dst = entry[1], c_rows = entry[2];
    const unsigned run16 = (unsigned)c_rows * row_bytes / 16, total = run16 * runs;       // 16-byte chunks of a run, of the copy
    const unsigned skip = (unsigned)(block_rows - c_rows) * row_bytes / 16;               // between the end of a run and the next one
    const unsigned first = piece * (COPY_THREADS * COPY_U) + threadIdx.x;
    if (piece * (COPY_THREADS * COPY_U) >= total) return;
    const v4u* src = (const v4u*)(pool + layer * layer_bytes + c_src * block_bytes);
    v4u* dst = (v4u*)(pool + layer * layer_bytes + c_dst * block_bytes);
    auto place = [&](unsigned i) { return i + (skip ? i / run16 * skip : 0); };
    if (piece * (COPY_THREADS * COPY_U) + COPY_THREADS * COPY_U <= total) {
        v4u v[COPY_U];
        unsigned at[COPY_U];
#pragma unroll
        for (int u = 0; u < COPY_U; ++u) v[u] = src[at[u] = place(first + u * COPY_THREADS)];
#pragma unroll
        for (int u = 0; u < COPY_U; ++u) __builtin_nontemporal_store(v[u], dst + at[u]);
    } else {
        for (unsigned i = first; i < total; i += COPY_THREADS) dst[place(i)] = src[place(i)];
    }
}

hipError_t launch_copy_blocks(const BlockCopyArgs& a, hipStream_t s)
{
    const int64_t block_bytes = (int64_t)a.runs * a.block_rows * a.row_bytes, layer_bytes = block_bytes * a.n_blocks;
    for (int i = 0; i < a.n; i += COPY_MAX) {
        const int n = a.n - i < COPY_MAX ? a.n - i : COPY_MAX;
        CopyList list;
        int most = 0;
        for (int k = 0; k < n; ++k) {
            list.c[k] = a.list[i + k];
            most = most < list.c[k].rows ? list.c[k].rows : most;
        }
        if (!most) continue;
        const int64_t pieces = ((int64_t)a.runs * most * a.row_bytes + COPY_PIECE - 1) / COPY_PIECE;
        // a launch has fewer than 2^32 threads: many layers of large blocks take several
        const int64_t per_layer = pieces * n, fit = MAX_LAUNCH_THREADS / COPY_THREADS / per_layer;
        if (fit < 1) return hipErrorInvalidValue;
        for (int l = 0; l < a.layers; l += (int)(fit < a.layers ? fit : a.layers)) {
            const int layers = a.layers - l < fit ? a.layers - l : (int)fit;
            copy_blocks_kernel<<<(unsigned)(per_layer * layers), COPY_THREADS, 0, s>>>(list, (unsigned char*)a.pool + l * layer_bytes, layer_bytes, block_bytes, layers,
                                                                                      a.block_rows, a.row_bytes, a.runs, (unsigned)pieces);
            hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

}  // namespace exe
