// Attention of a chunk of new tokens over a paged cache.
//
// The query rows of one sequence that share a key/value head are its new tokens times the H / Hkv heads of the group, row r = token
// r / G, head r % G: they read the same keys, so they are packed into one tile.
//  * chunk_stream_kernel: up to 16 rows a sequence (single tokens, a few drafted ones).  Bound by reading the cache once.
//  * chunk_tile_kernel: 64 to 256 rows a workgroup.  Bound by the MFMAs and by what feeds them.
//  * chunk_join_kernel: where the keys of a tile were cut into parts for several workgroups, adds the parts up.
// All hold scores and softmax in float, with the running maximum and sum of one pass over the keys.
#include <type_traits>

#include "attn_row.h"
#include "attn_tile.h"
#include "gemm_epilogue.h"
#include "kernels.h"

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
    return n < 0x7fffff00 ? (int)n : 0x7fffff00;
}

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

// ---------------------------------------------------------------- what the kernels share
struct ChunkKernelArgs {
    const int32_t* cu; const int32_t* len;
    int n_seqs, tokens;
    const void* q; int64_t q_stride;
    const void* kv_blocks;
    PagedTable table;
    int H, Hkv, G;
    float scale;
    int window;
    void* out; int64_t out_stride;
    // Keys go to workgroups in parts: `keys` of them each, at most `parts` (the last takes what is left), for the streaming and for the
    // tile kernel.  Part i of row (t, h) lies at acc[(i * tokens + t) * H + h][DH], ml[(i * tokens + t) * H + h][maximum, sum].
    struct Cut { int parts, keys; } stream, tile;
    int stream_rows;          // sequences of up to so many rows are the streaming kernel's, the others the tile kernel's
    int tile_rows;            // rows of a tile of the tile kernel
    float *acc, *ml;
};

constexpr int STREAM_ROWS = 16;
// Keys that the rows r0 .. r1 - 1 of a sequence see, the first one rounded down to a multiple of `align`; first >= last: none.
// p0: position of the first new token.
__device__ __forceinline__ KeyRange tile_keys(int p0, int G, int r0, int r1, int window, int limit, int align)
{
    KeyRange a = keys_of(p0 + r0 / G, window, limit), b = keys_of(p0 + (r1 - 1) / G, window, limit);
    return KeyRange{a.first & -align, b.last};
}
__device__ __forceinline__ int parts_of(KeyRange k, ChunkKernelArgs::Cut cut)
{
    if (k.last <= k.first) return 1;
    int n = (int)(((int64_t)k.last - k.first + cut.keys - 1) / cut.keys);
    return n < cut.parts ? n : cut.parts;
}
__device__ __forceinline__ KeyRange part_of(KeyRange k, ChunkKernelArgs::Cut cut, int part, int parts)
{
    int first = k.first + part * cut.keys;
    return KeyRange{first, part + 1 < parts ? first + cut.keys : k.last};
}

// What the loads of a position without a block read in its place: NaN keys make the scores of the rows that see it NaN.
static __device__ __align__(16) uint32_t no_block[256] = {
#define EXE_NAN4 0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu
#define EXE_NAN16 EXE_NAN4, EXE_NAN4, EXE_NAN4, EXE_NAN4
#define EXE_NAN64 EXE_NAN16, EXE_NAN16, EXE_NAN16, EXE_NAN16
    EXE_NAN64, EXE_NAN64, EXE_NAN64, EXE_NAN64
#undef EXE_NAN64
#undef EXE_NAN16
#undef EXE_NAN4
};

// 1 KB from global memory to LDS by one wave, 16 bytes a lane: from src + voff (per lane) to dst + 16 * lane.  Inline assembly, so that
// the compiler does not order every later LDS read behind it; whoever reads the tile waits.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds(const void* src, unsigned voff, unsigned dst)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(dst), "v"(voff), "s"(src) : "memory", "m0");
}
#pragma clang diagnostic pop
template <int N> __device__ __forceinline__ void wait_loads()        // all but the last N
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N) : "memory");
}

// The block table of one sequence, read by scalar loads: they do not wait behind the tile loads in flight.
struct SeqTable {
    const __attribute__((address_space(4))) int32_t* entry;
    int max_blocks, shift, n_blocks;
    __device__ __forceinline__ SeqTable(const PagedTable& t, int b)
        : entry((const __attribute__((address_space(4))) int32_t*)(uintptr_t)(t.entry + (int64_t)b * t.max_blocks)), max_blocks(t.max_blocks), shift(t.shift),
          n_blocks(t.n_blocks) {}
    // entry of the block with position pos >= 0; pos is the same in all lanes
    __device__ __forceinline__ int at(int pos) const
    {
        int i = pos >> shift;
        int e = entry[i < max_blocks ? i : max_blocks - 1];
        return i < max_blocks && (unsigned)e < (unsigned)n_blocks ? e : -1;
    }
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

// ---------------------------------------------------------------- few rows: the cache streams by
// A workgroup of 4 waves takes the 16 rows of one (sequence, key/value head) and a part of its keys.  Every wave takes steps of 16 keys of
// its own (wave w steps w, w + 4, ..), through a ring of stages in LDS that it fills itself by direct global-to-LDS loads, so no wave
// waits for another one before the end.  64 KB of stages a workgroup, two workgroups a CU, keep 64 KB a CU in flight (float x 128: 128 KB,
// one a CU).  Per step and wave: S^T = K . Q^T and O^T += V^T . P^T by MFMAs with the 16 rows as columns (see prefill_mfma_kernel); idle
// columns cost nothing that the loads do not hide.  Probabilities enter the second product as two bf16 parts, 2^-17 relative.
constexpr int ST_WAVES = 4, ST_STEP = 16;
template <typename T, int DH> struct Stream {
    static constexpr int RB = DH * (int)sizeof(T), TILE = ST_STEP * RB, STAGE = 2 * TILE;
    static constexpr int FIT = 65536 / (ST_WAVES * STAGE), STAGES = FIT < 2 ? 2 : FIT;
    static constexpr int LOADS = TILE / 1024;
    static constexpr int MERGE = ST_WAVES * 16 * (DH + 4) * 4;            // bytes of the waves' results, over the stages
    static constexpr int LDS = ST_WAVES * STAGES * STAGE > MERGE ? ST_WAVES * STAGES * STAGE : MERGE;
};

template <typename T, int DH>
__global__ __launch_bounds__(ST_WAVES * 64, 2) void chunk_stream_kernel(ChunkKernelArgs a)
{
    typedef Stream<T, DH> S;
    constexpr int RB = S::RB, DS = RB / 64, DT = DH / 16, RPL = 1024 / RB, CPR = RB / 16;
    extern __shared__ __align__(16) unsigned char st_smem[];
    __shared__ float s_ml[ST_WAVES][16][2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), qi = lane & 15, g = lane >> 4;
    const int b = blockIdx.x / a.Hkv, kvh = blockIdx.x - b * a.Hkv, part = blockIdx.y, G = a.G;
    const int t0 = a.cu[b], end = a.cu[b + 1], n = end - t0 < a.tokens ? end - t0 : a.tokens, rows = n * G, p0 = a.len[b] - n, limit = table_limit(a.table);
    if (n <= 0 || rows > a.stream_rows) return;
    const SeqTable tbl(a.table, b);
    const int64_t head = (int64_t)DH << a.table.shift, block_elems = 2 * a.Hkv * head;
    const T* kv = (const T*)a.kv_blocks + kvh * head;
    const int64_t v_off = a.Hkv * head;
    const unsigned lds = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)st_smem + wave * (S::STAGES * S::STAGE);
    const unsigned char* mine = st_smem + wave * (S::STAGES * S::STAGE);
    const float mul = exponent_scale(a.scale);

    for (int r0 = 0; r0 < rows; r0 += 16) {
        const int r1 = r0 + 16 < rows ? r0 + 16 : rows;
        const KeyRange all = tile_keys(p0, G, r0, r1, a.window, limit, ST_STEP);
        const int parts = parts_of(all, a.stream);
        if (part >= parts) continue;
        const KeyRange k = part_of(all, a.stream, part, parts);
        const int row = r0 + qi < r1 ? r0 + qi : r1 - 1, tok = row / G, t = t0 + tok;
        const KeyRange sees = keys_of(p0 + tok, a.window, limit);
        // a token beyond the packed ones is none of this call's
        const bool live = r0 + qi < r1 && t >= 0 && t < a.tokens;
        u32x4 qf[DS];
        load_query<T, DS>((const T*)a.q + (int64_t)(live ? t : 0) * a.q_stride + (kvh * G + row % G) * DH, g, a.scale, qf);

        const int steps = k.last > k.first ? (k.last - k.first + ST_STEP - 1) / ST_STEP : 0, own = steps > wave ? (steps - wave + ST_WAVES - 1) / ST_WAVES : 0;
        int e0 = 0, e1 = 0;
        auto first_of = [&](int i) { return k.first + (wave + i * ST_WAVES) * ST_STEP; };
        // a load takes RPL <= 8 rows of one block; rows from k.last on are row k.last - 1 again
        auto lookup = [&](int i) {
            int j = first_of(i), j1 = j + 8 < k.last ? j + 8 : j;
            e0 = tbl.at(j);
            e1 = tbl.at(j1);
        };
        auto issue = [&](int i) {
            const int j = first_of(i), block_mask = (1 << tbl.shift) - 1;
            const unsigned dst = lds + i % S::STAGES * S::STAGE;
#pragma unroll
            for (int p = 0; p < S::LOADS; ++p) {
                int key = p * RPL, at = j + key;                       // first row of this load in the step, its position
                at = at < k.last ? at : (k.last - 1) & -RPL;
                const int e = key < 8 || at < j + 8 ? e0 : e1;
                const T* src = e < 0 ? (const T*)no_block : kv + e * block_elems + (int64_t)(at & block_mask) * DH;
                int in = lane / CPR;
                const unsigned chunk = ((lane & (CPR - 1)) ^ pf_swz<RB>(key + in)) << 4;
                in = at + in < k.last ? in : k.last - 1 - at;
                const unsigned voff = in * RB + chunk;
                load_to_lds(src, voff, dst + key * RB);
                load_to_lds(e < 0 ? src : src + v_off, voff, dst + S::TILE + key * RB);
            }
        };

        float m = -INFINITY, l = 0.f;                                  // l: this lane's share of the sum
        f32x4 o[DT];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int ahead = S::STAGES - 1;
        for (int i = 0; i < ahead && i < own; ++i) {
            lookup(i);
            issue(i);
        }
        if (ahead < own) lookup(ahead);
        for (int i = 0; i < own; ++i) {
            if (i + ahead < own) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // step i - 1 has left its stage
                issue(i + ahead);
                if (i + ahead + 1 < own) lookup(i + ahead + 1);
                wait_loads<2 * S::LOADS * (S::STAGES - 1)>();
            } else {
                wait_loads<0>();
            }
            const unsigned char* sK = mine + i % S::STAGES * S::STAGE;
            f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int ds = 0; ds < DS; ++ds) {
                u32x4 fk = *(const u32x4*)(sK + qi * RB + (((ds * 4 + g) ^ pf_swz<RB>(qi)) << 4));
                s[ds & 1] = HalfUnit<T>::mma(fk, qf[ds], s[ds & 1]);
            }
            f32x4 sc = s[0] + s[1];
            const int key0 = first_of(i) + 4 * g;
#pragma unroll
            for (int r = 0; r < 4; ++r) sc[r] = key0 + r >= sees.first && key0 + r < sees.last ? sc[r] : -INFINITY;
            float mx = fmaxf(fmaxf(sc[0], sc[1]), fmaxf(sc[2], sc[3])) * mul;
            // the maximum follows only where it grew by more than 2^8: sums stay far from a float's ends
            if (__builtin_amdgcn_ballot_w64(mx > m + 8.f)) {
                float to = fmaxf(m, rows_max(mx)), ref = to == -INFINITY ? 0.f : to, alpha = fast_exp2(m - ref);
                l *= alpha;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[dt] *= alpha;
                m = to;
            }
            const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                sc[r] = fast_exp2(fmaf(sc[r], mul, -ref));
                l += sc[r];
            }
            const unsigned char* sV = sK + S::TILE;
            if constexpr (sizeof(T) == 2) {
                typedef __attribute__((ext_vector_type(4))) short v4s;
                bf16x4 hi, lo;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    hi[r] = (bf16_t)sc[r];
                    lo[r] = (bf16_t)(sc[r] - (float)hi[r]);
                }
                const int v_row = 4 * g + (qi >> 2), v_q = qi & 3;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    uint2 v = pf_read_tr(sV + v_row * RB + (((2 * dt + (v_q >> 1)) ^ pf_swz<RB>(v_row)) << 4) + (v_q & 1) * 8);
                    o[dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(v4s, v), __builtin_bit_cast(v4s, hi), o[dt], 0, 0, 0);
                    o[dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(v4s, v), __builtin_bit_cast(v4s, lo), o[dt], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    f32x4 c = {0.f, 0.f, 0.f, 0.f};                    // a sum per step, so that no chain of additions is as long as the cache
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float v = *(const float*)(sV + (4 * g + r) * RB + (((4 * dt + (qi >> 2)) ^ pf_swz<RB>(4 * g + r)) << 4) + (qi & 3) * 4);
                        c = __builtin_amdgcn_mfma_f32_16x16x4f32(v, sc[r], c, 0, 0, 0);
                    }
                    o[dt] += c;
                }
            }
        }

        // the waves' results, joined; lane (qi, g) holds features 16 * dt + 4 * g .. +3 of its row
        l = rows_sum(l);
        __syncthreads();                                               // no wave reads its stages any more
        float* s_o = (float*)st_smem;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) *(f32x4*)(s_o + (wave * 16 + qi) * (DH + 4) + dt * 16 + 4 * g) = o[dt];
        if (g == 0) {
            s_ml[wave][qi][0] = m;
            s_ml[wave][qi][1] = l;
        }
        __syncthreads();
        const int r = tid >> 4, c = tid & 15;                          // 16 threads a row, features 4 * c .. +3 of every 64
        const int wtok = (r0 + r) / G, wt = t0 + wtok, h = kvh * G + (r0 + r) % G;
        const bool write = r0 + r < r1 && wt >= 0 && wt < a.tokens;
        float M = -INFINITY, L = 0.f, w[ST_WAVES];
#pragma unroll
        for (int i = 0; i < ST_WAVES; ++i) M = fmaxf(M, s_ml[i][r][0]);
        const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (int i = 0; i < ST_WAVES; ++i) {
            w[i] = fast_exp2(s_ml[i][r][0] - ref);
            L += s_ml[i][r][1] * w[i];
        }
        f32x4 v[DH / 64];
#pragma unroll
        for (int f = 0; f < DH / 64; ++f) {
            v[f] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < ST_WAVES; ++i) v[f] += *(const f32x4*)(s_o + (i * 16 + r) * (DH + 4) + f * 64 + 4 * c) * w[i];
        }
        if (parts > 1) {
            if (write) {
                const int64_t at = ((int64_t)part * a.tokens + wt) * a.H + h;
#pragma unroll
                for (int f = 0; f < DH / 64; ++f) *(f32x4*)(a.acc + at * DH + f * 64 + 4 * c) = v[f];
                if (c == 0) *(float2*)(a.ml + at * 2) = float2{M, L};
            }
        } else {
            const KeyRange ks = keys_of(p0 + wtok, a.window, limit);
            const float inv = ks.last > ks.first ? 1.f / L : 0.f;
            T* op = (T*)a.out + (int64_t)wt * a.out_stride + h * DH;
            float most = 0.f;
#pragma unroll
            for (int f = 0; f < DH / 64; ++f)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    v[f][e] = ks.last > ks.first ? v[f][e] * inv : 0.f;
                    most = __builtin_elementwise_maximum(most, v[f][e]);
                }
            // 0 times the infinite or NaN value of a key that the mask hides is NaN: such a row is computed again from its own keys
            unsigned long long again = __builtin_amdgcn_ballot_w64(write && most != most);
            if (write && !(again >> (lane & 48) & 0xffff)) {
#pragma unroll
                for (int f = 0; f < DH / 64; ++f) {
                    typename Vec4<T>::type x;
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = from_f32<T>(v[f][e]);
                    *(typename Vec4<T>::type*)(op + f * 64 + 4 * c) = x;
                }
            }
            for (int i = 0; i < 4; ++i)
                if (again >> (16 * i) & 0xffff) {
                    const int rr = r0 + wave * 4 + i, tk = rr / G, hh = kvh * G + rr % G;
                    chunk_row<T, DH>((const T*)a.q + (int64_t)(t0 + tk) * a.q_stride + hh * DH, kv, block_elems, v_off, a.table, b, keys_of(p0 + tk, a.window, limit),
                                     a.scale * LOG2E, lane, (T*)a.out + (int64_t)(t0 + tk) * a.out_stride + hh * DH);
                }
        }
        __syncthreads();                                               // before the next tile's loads overwrite the results
    }
}

// ---------------------------------------------------------------- many rows: tiles
// A workgroup of 4 waves owns 64 * QB rows, 16 * QB a wave, and a part of their keys, which pass through LDS in tiles of 64: two buffers
// for keys, two for values, filled by direct global-to-LDS loads a tile ahead, one barrier a tile.  The products are those of
// prefill_mfma_kernel.  A wave computes the scores of tile kt + 1 before it needs those of tile kt's successor: the MFMAs of the one
// and the exponentials of the other do not depend on each other.
constexpr int CT_WAVES = 4, CT_KEYS = 64;
template <typename T, int DH> constexpr int ct_lds() { return 4 * CT_KEYS * DH * (int)sizeof(T); }
template <typename T, int DH, int QB> constexpr int ct_per_cu() { return QB == 4 ? 1 : sizeof(T) == 4 && DH == 128 ? 1 : QB == 2 || DH == 128 ? 2 : 3; }

template <typename T, int DH, int QB>
__global__ __launch_bounds__(CT_WAVES * 64, (ct_per_cu<T, DH, QB>())) void chunk_tile_kernel(ChunkKernelArgs a, int slots)
{
    constexpr int RB = DH * (int)sizeof(T), DS = RB / 64, DT = DH / 16, RPL = 1024 / RB, CPR = RB / 16, LOADS = 16 / RPL, TILE = CT_KEYS * RB;
    constexpr int ROWS = 16 * QB * CT_WAVES;
    extern __shared__ __align__(16) unsigned char ct_smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), qi = lane & 15, g = lane >> 4;
    const int G = a.G, part = blockIdx.y;
    // Workgroup -> (slot, head), see prefill_mfma_kernel: the tiles of one sequence and head run side by side on one XCD.  Last rows
    // (most keys) first.
    int slot, kvh;
    if ((a.Hkv & 7) == 0) {
        int hpx = a.Hkv >> 3, j = blockIdx.x >> 3;
        slot = j / hpx;
        kvh = (blockIdx.x & 7) + 8 * (j - slot * hpx);
    } else {
        slot = blockIdx.x / a.Hkv;
        kvh = blockIdx.x - slot * a.Hkv;
    }
    slot = slots - 1 - slot;
    // Slot -> tile: those of sequence b begin at slot floor(cu[b] * G / ROWS) + b, which leaves room for every sequence's last, partly
    // filled tile whatever the lengths are.
    const int b = __builtin_amdgcn_readfirstlane(wave_search(0, a.n_seqs, lane, [&](int i) { return (int)((int64_t)a.cu[i] * G / ROWS) + i <= slot; }));
    if (b < 0) return;
    const int t0 = a.cu[b], end = a.cu[b + 1], n = end - t0 < a.tokens ? end - t0 : a.tokens, rows = n * G, p0 = a.len[b] - n, limit = table_limit(a.table);
    const int r0 = (slot - ((int)((int64_t)t0 * G / ROWS) + b)) * ROWS;
    if (n <= 0 || r0 >= rows || rows <= a.stream_rows) return;
    const KeyRange all = tile_keys(p0, G, r0, r0 + ROWS < rows ? r0 + ROWS : rows, a.window, limit, CT_KEYS);
    const int parts = parts_of(all, a.tile);
    if (part >= parts) return;
    const KeyRange k = part_of(all, a.tile, part, parts);
    const SeqTable tbl(a.table, b);
    const int64_t head = (int64_t)DH << a.table.shift, block_elems = 2 * a.Hkv * head, v_off = a.Hkv * head;
    const T* kv = (const T*)a.kv_blocks + kvh * head;
    const float mul = exponent_scale(a.scale);
    const int w0 = r0 + wave * (16 * QB);                              // this wave's first row
    const int wl = w0 + 16 * QB < rows ? w0 + 16 * QB - 1 : rows - 1;  // and last one
    const bool active = w0 < rows;
    const int p_min = p0 + w0 / G, p_max = p0 + wl / G;
    const int n_tiles = k.last > k.first ? (k.last - k.first + CT_KEYS - 1) / CT_KEYS : 0;

    u32x4 qf[QB][DS];
    KeyRange sees[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        int row = w0 + qb * 16 + qi;
        row = row < rows ? row : rows - 1;
        int t = t0 + row / G;
        sees[qb] = keys_of(p0 + row / G, a.window, limit);
        load_query<T, DS>((const T*)a.q + (int64_t)(t >= 0 && t < a.tokens ? t : 0) * a.q_stride + (kvh * G + row % G) * DH, g, a.scale, qf[qb]);
    }

    // ---- loaders: wave w fills rows 16 * w .. +15 of a tile
    const unsigned lds = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)ct_smem;
    struct Entries { int e0, e1; };
    auto lookup = [&](int kt) {
        int j = k.first + kt * CT_KEYS + wave * 16;
        j = j < k.last ? j : k.last - 1;
        int j1 = j + 8 < k.last ? j + 8 : k.last - 1;
        return Entries{tbl.at(j), tbl.at(j1)};
    };
    auto load_tile = [&](int kt, Entries en, int64_t off, unsigned dst) {
        const int j = k.first + kt * CT_KEYS + wave * 16, block_mask = (1 << tbl.shift) - 1;
#pragma unroll
        for (int p = 0; p < LOADS; ++p) {
            int key = p * RPL, at = j + key;
            // rows from k.last on are row k.last - 1 again; the second entry is of row j + 8 or of the last one
            const int e = key < 8 ? en.e0 : en.e1;
            at = at < k.last ? at : (k.last - 1) & -RPL;
            const T* src = e < 0 ? (const T*)no_block : kv + e * block_elems + off + (int64_t)(at & block_mask) * DH;
            int in = lane / CPR;
            const unsigned chunk = ((lane & (CPR - 1)) ^ pf_swz<RB>(key + in)) << 4;
            in = at + in < k.last ? in : k.last - 1 - at;
            load_to_lds(src, in * RB + chunk, dst + (wave * 16 + key) * RB);
        }
    };
    auto load_k = [&](int kt, Entries en) { load_tile(kt, en, 0, lds + (kt & 1) * TILE); };
    auto load_v = [&](int kt, Entries en) { load_tile(kt, en, v_off, lds + (2 + (kt & 1)) * TILE); };

    f32x4 o[QB][DT];
    float m[QB], l[QB];                                                // l: this lane's share
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        m[qb] = -INFINITY;
        l[qb] = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[qb][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    typedef f32x4 Scores[QB][4];
    auto scores = [&](int kt, Scores& s) {
        const unsigned char* sK = ct_smem + (kt & 1) * TILE;
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) {
            f32x4 c[QB][2];
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) c[qb][0] = c[qb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ds = 0; ds < DS; ++ds) {
                u32x4 fk = *(const u32x4*)(sK + (kb * 16 + qi) * RB + (((ds * 4 + g) ^ pf_swz<RB>(qi)) << 4));
                constexpr bool TWO = sizeof(T) == 4;                   // float: two shorter chains of additions
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) c[qb][TWO ? ds & 1 : 0] = HalfUnit<T>::mma(fk, qf[qb][ds], c[qb][TWO ? ds & 1 : 0]);
            }
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) s[qb][kb] = sizeof(T) == 4 ? c[qb][0] + c[qb][1] : c[qb][0];
        }
    };
    // masks, and moves the running maxima where a score passes one by more than 2^8
    auto look = [&](int kt, Scores& s) {
        const int j = k.first + kt * CT_KEYS;
        if (j + CT_KEYS - 1 > p_min || j + CT_KEYS > k.last || (a.window && j <= p_max - a.window)) {
            int key0 = j + 4 * g;
            asm volatile("" : "+v"(key0));                             // keeps the mask arithmetic inside this branch
#pragma unroll
            for (int qb = 0; qb < QB; ++qb)
#pragma unroll
                for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        int key = key0 + kb * 16 + r;
                        s[qb][kb][r] = key >= sees[qb].first && key < sees[qb].last && key < k.last ? s[qb][kb][r] : -INFINITY;
                    }
        }
        float mx[QB];
        bool grew = false;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            mx[qb] = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                for (int r = 0; r < 4; ++r) mx[qb] = fmaxf(mx[qb], s[qb][kb][r]);
            mx[qb] *= mul;
            grew |= mx[qb] > m[qb] + 8.f;
        }
        if (__builtin_amdgcn_ballot_w64(grew)) {
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                float to = fmaxf(m[qb], rows_max(mx[qb])), ref = to == -INFINITY ? 0.f : to, alpha = fast_exp2(m[qb] - ref);
                l[qb] *= alpha;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[qb][dt] *= alpha;
                m[qb] = to;
            }
        }
    };
    auto exponentials = [&](Scores& s) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const float ref = m[qb] == -INFINITY ? 0.f : m[qb];
#pragma unroll
            for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[qb][kb][r] = fast_exp2(fmaf(s[qb][kb][r], mul, -ref));
                    l[qb] += s[qb][kb][r];
                }
        }
    };
    auto values = [&](int kt, Scores& s) {
        const unsigned char* tV = ct_smem + (2 + (kt & 1)) * TILE;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                f32x4 c[QB][2];
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) c[qb][0] = c[qb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kb = 0; kb < 4; ++kb)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float v = *(const float*)(tV + (kb * 16 + 4 * g + r) * RB + (((4 * dt + (qi >> 2)) ^ pf_swz<RB>(4 * g + r)) << 4) + (qi & 3) * 4);
#pragma unroll
                        for (int qb = 0; qb < QB; ++qb) c[qb][kb & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, s[qb][kb][r], c[qb][kb & 1], 0, 0, 0);
                    }
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) o[qb][dt] += c[qb][0] + c[qb][1];
            }
        } else {
            const int v_row = 4 * g + (qi >> 2), v_q = qi & 3;
            const unsigned char* sV = tV + v_row * RB + (v_q & 1) * 8;
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                // one rounding to bf16 per probability, half a step of the result's own type
                bf16x8 pf[QB];
#pragma unroll
                for (int qb = 0; qb < QB; ++qb)
#pragma unroll
                    for (int e = 0; e < 8; ++e) pf[qb][e] = (bf16_t)s[qb][2 * ks + (e >> 2)][e & 3];
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    const int at = ((2 * dt + (v_q >> 1)) ^ pf_swz<RB>(v_row)) << 4;
                    uint2 lo = pf_read_tr(sV + ks * 32 * RB + at), hi = pf_read_tr(sV + (ks * 32 + 16) * RB + at);
                    bf16x8 fv = __builtin_bit_cast(bf16x8, uint4{lo.x, lo.y, hi.x, hi.y});
#pragma unroll
                    for (int qb = 0; qb < QB; ++qb) o[qb][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fv, pf[qb], o[qb][dt], 0, 0, 0);
                }
            }
        }
    };

    if (n_tiles > 0) {
        // tile kt's values are loaded an iteration before its second product, its keys two before that
        Scores s[2];
        Entries ek = lookup(0), ev = ek;
        load_k(0, ek);
        wait_loads<0>();
        __syncthreads();
        load_v(0, ek);
        ek = lookup(n_tiles > 1 ? 1 : 0);
        if (n_tiles > 1) load_k(1, ek);
        ev = ek;
        ek = lookup(n_tiles > 2 ? 2 : 0);
        if (active) scores(0, s[0]);
        auto iteration = [&](int kt, Scores& now, Scores& next) {
            wait_loads<0>();                                           // values of tile kt, keys of kt + 1
            __syncthreads();
            if (kt + 1 < n_tiles) load_v(kt + 1, ev);
            if (kt + 2 < n_tiles) load_k(kt + 2, ek);
            ev = ek;
            ek = lookup(kt + 3 < n_tiles ? kt + 3 : 0);
            if (!active) return;
            look(kt, now);
            if (kt + 1 < n_tiles) scores(kt + 1, next);
            exponentials(now);
            values(kt, now);
        };
        for (int kt = 0; kt < n_tiles; kt += 2) {
            iteration(kt, s[0], s[1]);
            if (kt + 1 < n_tiles) iteration(kt + 1, s[1], s[0]);
        }
    }
    if (!active) return;

    // lane (qi, g) holds features 16 * dt + 4 * g .. +3 of its rows
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int row = w0 + qb * 16 + qi, t = t0 + row / G, h = kvh * G + row % G;
        const bool write = row < rows && t >= 0 && t < a.tokens;
        const float sum = rows_sum(l[qb]);
        if (parts > 1) {
            if (!write) continue;
            const int64_t at = ((int64_t)part * a.tokens + t) * a.H + h;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) *(f32x4*)(a.acc + at * DH + dt * 16 + 4 * g) = o[qb][dt];
            if (g == 0) *(float2*)(a.ml + at * 2) = float2{m[qb], sum};
            continue;
        }
        const bool any = sees[qb].last > sees[qb].first;
        const float inv = 1.f / sum;
        float most = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                o[qb][dt][e] = any ? o[qb][dt][e] * inv : 0.f;
                most = __builtin_elementwise_maximum(most, o[qb][dt][e]);
            }
        // 0 times the infinite or NaN value of a key that the mask hides is NaN: such a row is computed again from its own keys
        unsigned long long lanes = __builtin_amdgcn_ballot_w64(write && most != most);
        unsigned again = (unsigned)(lanes | lanes >> 32);
        again = (again | again >> 16) & 0xffff;                        // bit qi: row w0 + 16 * qb + qi
        if (write && !(again >> qi & 1)) {
            T* op = (T*)a.out + (int64_t)t * a.out_stride + h * DH + 4 * g;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                typename Vec4<T>::type x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = from_f32<T>(o[qb][dt][e]);
                *(typename Vec4<T>::type*)(op + dt * 16) = x;
            }
        }
        for (; again; again &= again - 1) {
            const int rr = w0 + qb * 16 + __builtin_ctz(again), tk = rr / G, hh = kvh * G + rr % G;
            chunk_row<T, DH>((const T*)a.q + (int64_t)(t0 + tk) * a.q_stride + hh * DH, kv, block_elems, v_off, a.table, b, keys_of(p0 + tk, a.window, limit), a.scale * LOG2E,
                             lane, (T*)a.out + (int64_t)(t0 + tk) * a.out_stride + hh * DH);
        }
    }
}

// ---------------------------------------------------------------- parts of the keys, joined
// A wave per row: sum over the parts of 2^(m_i - M) times their sums, in the order of the parts.  Rows of a single part are complete.
template <typename T, int DH> __global__ __launch_bounds__(256) void chunk_join_kernel(ChunkKernelArgs a)
{
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = (int)(unit / a.H), h = (int)(unit - (int64_t)t * a.H), G = a.G;
    if (t >= a.tokens) return;
    const ChunkSeq sq = seq_of_token(a.cu, a.n_seqs, t, lane);
    if (sq.b < 0) return;
    const int rows = sq.n * G, p0 = a.len[sq.b] - sq.n, limit = table_limit(a.table), row = (t - sq.t0) * G + h % G;
    const bool streamed = rows <= a.stream_rows;
    const ChunkKernelArgs::Cut cut = streamed ? a.stream : a.tile;
    const int tile = streamed ? STREAM_ROWS : a.tile_rows, r0 = row / tile * tile;
    const int parts = parts_of(tile_keys(p0, G, r0, r0 + tile < rows ? r0 + tile : rows, a.window, limit, streamed ? ST_STEP : CT_KEYS), cut);
    if (parts <= 1) return;
    const int64_t at = (int64_t)t * a.H + h, step = (int64_t)a.tokens * a.H;
    float M = -INFINITY;
    for (int i = lane; i < parts; i += 64) M = fmaxf(M, a.ml[(at + i * step) * 2]);
    M = wave_max(M);
    const float ref = M == -INFINITY ? 0.f : M;
    float L = 0.f, v[DH / 64] = {};
#pragma unroll 4
    for (int i = 0; i < parts; ++i) {
        const float2 ml = *(const float2*)(a.ml + (at + i * step) * 2);
        const float w = fast_exp2(ml.x - ref);
        L = fmaf(ml.y, w, L);
#pragma unroll
        for (int f = 0; f < DH / 64; ++f) v[f] = fmaf(a.acc[(at + i * step) * DH + f * 64 + lane], w, v[f]);
    }
    const KeyRange ks = keys_of(p0 + (t - sq.t0), a.window, limit);
    T* op = (T*)a.out + (int64_t)t * a.out_stride + h * DH;
    float most = 0.f;
#pragma unroll
    for (int f = 0; f < DH / 64; ++f) {
        v[f] = ks.last > ks.first ? v[f] / L : 0.f;
        most = __builtin_elementwise_maximum(most, v[f]);
    }
    if (__builtin_amdgcn_ballot_w64(most != most)) {                   // as in the kernels above
        const int64_t head = (int64_t)DH << a.table.shift;
        chunk_row<T, DH>((const T*)a.q + (int64_t)t * a.q_stride + h * DH, (const T*)a.kv_blocks + h / G * head, 2 * a.Hkv * head, a.Hkv * head, a.table, sq.b, ks,
                         a.scale * LOG2E, lane, op);
        return;
    }
#pragma unroll
    for (int f = 0; f < DH / 64; ++f) op[f * 64 + lane] = from_f32<T>(v[f]);
}

// ---------------------------------------------------------------- launches
struct ChunkPlan {
    bool stream, tile;               // which kernels run
    int qb;                          // row blocks per wave of the tile kernel
    int64_t slots;
    ChunkKernelArgs::Cut stream_cut, tile_cut;
    int parts() const { int a = stream ? stream_cut.parts : 1, b = tile ? tile_cut.parts : 1; return a > b ? a : b; }
};
static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Parts for `wgs` workgroups that each would take up to max_len keys: enough workgroups to fill the chip `rounds` times over, no part
// shorter than `least` keys.
static ChunkKernelArgs::Cut cut_keys(int64_t wgs, int64_t max_len, int64_t want, int least, int align)
{
    int64_t parts = want / wgs, most = ceil_div(max_len, least);
    parts = parts < most ? parts : most;
    if (parts <= 1) return {1, 0x7fffffff};
    int64_t keys = ceil_div(ceil_div(max_len, parts), align) * align;
    return {(int)ceil_div(max_len, keys), (int)keys};
}

static ChunkPlan chunk_plan(const ChunkAttnArgs& a)
{
    ChunkPlan p{};
    const int64_t G = a.H / a.Hkv, rows = (int64_t)a.max_new * G, seen = a.window && a.window + (int64_t)a.max_new < a.max_len ? a.window + (int64_t)a.max_new : a.max_len;
    p.tile = rows > STREAM_ROWS;
    // a sequence of up to 16 rows beside longer ones: not where there is one sequence, or all bring max_new tokens
    p.stream = !p.tile || (a.n_seqs > 1 && (int64_t)a.tokens <= (int64_t)(a.n_seqs - 1) * a.max_new + STREAM_ROWS / G);
    if (p.stream) p.stream_cut = cut_keys((int64_t)a.n_seqs * a.Hkv, seen, 2048, 256, ST_STEP);
    if (p.tile) {
        auto wgs = [&](int qb) { return (ceil_div((int64_t)a.tokens * G, 64 * qb) + (a.n_seqs - 1)) * a.Hkv; };
        p.qb = a.dtype == DT_BF16 && wgs(4) >= 224 ? 4 : wgs(2) >= 320 ? 2 : 1;
        p.slots = (int64_t)a.tokens * G / (64 * p.qb) + a.n_seqs;
        p.tile_cut = cut_keys(wgs(p.qb), seen, 640, 512, CT_KEYS);
    }
    return p;
}

size_t chunk_attn_workspace(const ChunkAttnArgs& a)
{
    const ChunkPlan p = chunk_plan(a);
    return p.parts() <= 1 ? 0 : (size_t)p.parts() * a.tokens * a.H * (a.dh + 2) * sizeof(float);
}

template <typename T, int DH, int QB> static hipError_t launch_tile(const ChunkKernelArgs& k, const ChunkPlan& p, hipStream_t s)
{
    static LdsLimit limit[MAX_DEVICES];
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= MAX_DEVICES) dev = 0;
    hipError_t e = limit[dev].raise((const void*)chunk_tile_kernel<T, DH, QB>, ct_lds<T, DH>());
    if (e != hipSuccess) return e;
    const int64_t wgs = p.slots * k.Hkv;
    if (p.slots > 0x7fffffff || wgs * CT_WAVES * 64 * p.tile_cut.parts > MAX_LAUNCH_THREADS) return hipErrorInvalidValue;
    chunk_tile_kernel<T, DH, QB><<<dim3((unsigned)wgs, p.tile_cut.parts), CT_WAVES * 64, ct_lds<T, DH>(), s>>>(k, (int)p.slots);
    return hipGetLastError();
}

template <typename T, int DH> static hipError_t launch_chunk(const ChunkAttnArgs& a, hipStream_t s)
{
    const ChunkPlan p = chunk_plan(a);
    ChunkKernelArgs k{a.cu, a.len, a.n_seqs, a.tokens, a.q, a.q_stride, a.kv_blocks, a.table, a.H, a.Hkv, a.H / a.Hkv, a.scale, a.window, a.out, a.out_stride,
                      p.stream_cut, p.tile_cut, 0, 64 * p.qb, a.workspace, nullptr};
    k.ml = a.workspace ? a.workspace + (size_t)p.parts() * a.tokens * a.H * a.dh : nullptr;
    // without a tile kernel the streaming one takes every sequence, in tiles of 16 rows
    k.stream_rows = !p.tile ? 0x7fffffff : p.stream ? STREAM_ROWS : 0;
    hipError_t e;
    if (p.stream) {
        static LdsLimit limit[MAX_DEVICES];
        int dev = 0;
        if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= MAX_DEVICES) dev = 0;
        e = limit[dev].raise((const void*)chunk_stream_kernel<T, DH>, Stream<T, DH>::LDS);
        if (e != hipSuccess) return e;
        const int64_t wgs = (int64_t)a.n_seqs * a.Hkv;
        if (wgs * ST_WAVES * 64 * p.stream_cut.parts > MAX_LAUNCH_THREADS) return hipErrorInvalidValue;
        chunk_stream_kernel<T, DH><<<dim3((unsigned)wgs, p.stream_cut.parts), ST_WAVES * 64, Stream<T, DH>::LDS, s>>>(k);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (p.tile) {
        if constexpr (sizeof(T) == 2) {
            if (p.qb == 4) e = launch_tile<T, DH, 4>(k, p, s);
        }
        if (p.qb == 2) e = launch_tile<T, DH, 2>(k, p, s);
        if (p.qb == 1) e = launch_tile<T, DH, 1>(k, p, s);
        if (e != hipSuccess) return e;
    }
    if (p.parts() > 1) {
        const int64_t wgs = ceil_div((int64_t)a.tokens * a.H, 4);
        if (wgs * 256 > MAX_LAUNCH_THREADS) return hipErrorInvalidValue;
        chunk_join_kernel<T, DH><<<(unsigned)wgs, 256, 0, s>>>(k);
        e = hipGetLastError();
    }
    return e;
}

hipError_t launch_chunk_attn(const ChunkAttnArgs& a, hipStream_t s)
{
    if (a.dtype == DT_F32) return a.dh == 64 ? launch_chunk<float, 64>(a, s) : launch_chunk<float, 128>(a, s);
    return a.dh == 64 ? launch_chunk<bf16_t, 64>(a, s) : launch_chunk<bf16_t, 128>(a, s);
}

}  // namespace exe
