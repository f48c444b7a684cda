// Attention of a chunk of new tokens over a paged cache.
//
// The query rows of one sequence that share a key/value head are its new tokens times the G = H / Hkv heads of the group, row r = token
// r / G, head r % G: they read the same keys, so they are packed into one tile.
//  * chunk_stream_kernel: up to 16 rows a sequence (single tokens, a few drafted ones), and calls of few rows in tiles of 16.  Bound by
//    reading the cache.
//  * chunk_tile_kernel: 64 or 128 rows a workgroup.  Bound by MFMAs and softmax, which overlap in part; with few rows to a sequence and
//    many heads by the cache, again.
//  * chunk_join_stream_kernel, chunk_join_tile_kernel: where the keys of a tile were cut into parts for several workgroups, add them up.
//  * chunk_row: a wave per row, for rows that a hidden infinity or NaN has spoilt, or whose sums passed a float's end.
// All hold scores and softmax in float, with the running maximum and sum of one pass over the keys.  Which run is chunk_plan's choice,
// from what the host knows (bounds of the lengths); which sequence is whose, and how many parts a tile has, each kernel finds from the
// lengths on the device, so that a captured launch follows them.
#include <type_traits>

#include "chunk_tile.h"

namespace exe {

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
    // tile kernel.  What part i makes of row r lies at acc[i * rows + r][DH], ml[i * rows + r][maximum, sum].
    struct Cut { int parts, keys; int64_t rows; float *acc, *ml; } stream, tile;
    int stream_rows;          // sequences of up to so many rows are the streaming kernel's, the others the tile kernel's
    int tile_rows;            // rows of a tile of the tile kernel
    __device__ __forceinline__ int64_t row(int t, int h) const { return (int64_t)t * H + h; }
    // of the streaming kernel's: beside the tile kernel, where its sequences have few of the tokens, 16 for each
    __device__ __forceinline__ int64_t stream_row(int b, int kvh, int r, int t, int h) const
    {
        return stream_rows == 16 ? ((int64_t)b * Hkv + kvh) * 16 + r : row(t, h);
    }
};

// Row (t, h) of sequence b, by one wave (see chunk_row)
template <typename T, int DH> __device__ __forceinline__ void row_again(const ChunkKernelArgs& a, int b, int t, int h, KeyRange r, int lane)
{
    const int64_t head = (int64_t)DH << a.table.shift;
    chunk_row<T, DH>((const T*)a.q + (int64_t)t * a.q_stride + h * DH, (const T*)a.kv_blocks + h / a.G * head, 2 * a.Hkv * head, a.Hkv * head, a.table.shift,
                     [&](int j) { return a.table.block(b, j); }, r, a.scale * LOG2E, lane, (T*)a.out + (int64_t)t * a.out_stride + h * DH);
}

constexpr int STREAM_ROWS = 16, MAX_PARTS = WAVE;
// Keys that the rows r0 .. r1 - 1 of a sequence see, the first one rounded down to a multiple of `align`; first >= last: none.
// p0: position of the first new token.
__device__ __forceinline__ KeyRange tile_keys(int p0, int G, int r0, int r1, int window, int limit, int align)
{
    KeyRange a = keys_of(p0 + r0 / G, window, limit), b = keys_of(p0 + (r1 - 1) / G, window, limit);
    return KeyRange{a.first & -align, b.last};
}
__device__ __forceinline__ int parts_of(KeyRange k, const ChunkKernelArgs::Cut& cut)
{
    if (k.last <= k.first) return 1;
    int n = (int)(((int64_t)k.last - k.first + cut.keys - 1) / cut.keys);
    return n < cut.parts ? n : cut.parts;
}
__device__ __forceinline__ KeyRange part_of(KeyRange k, const ChunkKernelArgs::Cut& cut, int part, int parts)
{
    int first = k.first + part * cut.keys;
    return KeyRange{first, part + 1 < parts ? first + cut.keys : k.last};
}

// Workgroup -> (slot, head), see prefill_mfma_kernel: the tiles of one sequence and head run side by side on one XCD.  Last rows (most
// keys) first.  Slot -> tile: those of sequence b begin at slot floor(cu[b] * G / rows of a tile) + b, which leaves room for every sequence's
// last, partly filled tile whatever the lengths are.  b = -1: no tile, or a sequence of up to `least` rows, which is another kernel's.
__device__ __forceinline__ ChunkTile find_tile(const ChunkKernelArgs& a, unsigned wg, int slots, int tile_shift, int least, int lane)
{
    int slot, kvh;
    if ((a.Hkv & 7) == 0) {
        int hpx = a.Hkv >> 3, j = wg >> 3;
        slot = j / hpx;
        kvh = (wg & 7) + 8 * (j - slot * hpx);
    } else {
        slot = wg / a.Hkv;
        kvh = wg - slot * a.Hkv;
    }
    slot = slots - 1 - slot;
    auto first_slot = [&](int64_t t, int b) { return (int)(t * a.G >> tile_shift) + b; };
    int b, t0, end, len;
    if (a.n_seqs < WAVE) {                                             // all of it in one trip to memory
        const int c = a.cu[lane < a.n_seqs ? lane : a.n_seqs], l = a.len[lane < a.n_seqs ? lane : a.n_seqs - 1];
        b = __popcll(__builtin_amdgcn_ballot_w64(lane < a.n_seqs && first_slot(c, lane) <= slot)) - 1;
        if (b < 0) return ChunkTile{-1};
        t0 = __builtin_amdgcn_readlane(c, b);
        end = __builtin_amdgcn_readlane(c, b + 1);
        len = __builtin_amdgcn_readlane(l, b);
    } else {
        b = __builtin_amdgcn_readfirstlane(wave_search(0, a.n_seqs, lane, [&](int i) { return first_slot(a.cu[i], i) <= slot; }));
        if (b < 0) return ChunkTile{-1};
        t0 = a.cu[b];
        end = a.cu[b + 1];
        len = a.len[b];
    }
    const int n = end - t0 < a.tokens ? end - t0 : a.tokens, rows = n * a.G, r0 = (slot - first_slot(t0, b)) << tile_shift;
    return ChunkTile{n <= 0 || r0 >= rows || rows <= least ? -1 : b, kvh, t0, rows, len - n, r0};
}

// ---------------------------------------------------------------- few rows: the cache streams by
// A workgroup of 4 or 8 waves takes the 16 rows of one (sequence, key/value head) and a part of its keys.  Every wave takes steps of 16 keys
// of its own (wave w steps w, w + WAVES, ..), through a ring of stages in LDS that it fills itself by direct global-to-LDS loads, so no
// wave waits for another one before the end.  16 KB of stages a wave (float x 128: 32 KB), 8 waves a CU: half of that is in flight while
// the rest is computed on.  (4 waves a CU with 32 KB each took 230 us where 8 take 182: a step is 400 instructions, most of them not
// the matrix's.)  Per step and wave: S^T = K . Q^T and O^T += V^T . P^T by MFMAs with the 16 rows as columns (see prefill_mfma_kernel);
// idle columns cost nothing that the loads do not hide.  Probabilities enter the second product as two bf16 parts, 2^-17 relative.
// Bound by memory where contexts are long.  Nontemporal loads: 200 -> 182 us for 64 sequences of 500 to 8100 keys, 8 heads x 128 (1.1 GB, 6.1 TB/s); of
// 4096 keys each 169 us (6.34 TB/s; whole 161, 6.66, where a plain read reaches 7.1): the cut into parts, which lengths that differ want, costs
// 5 %.  Shorter ones pay the start of a workgroup (5.4 us with 16 keys) in each of up to four rounds, and the join: 200 to 2000 keys
// 56 us, 5.1 TB/s, 100 to 1024 38 us, 4.0 TB/s; 64-wide heads of 500 to 4000 69 us, 4.7 TB/s.  Float, 500 to 4000 keys: x 64 116 us, 5.6 TB/s, x 128
// (4 waves a CU) 293 us, 4.4 TB/s.
constexpr int ST_WAVES = 4, ST_STEP = 16;
template <typename T, int DH, int WAVES> struct Stream {
    static constexpr int RB = DH * (int)sizeof(T), TILE = ST_STEP * RB, STAGE = 2 * TILE;
    static constexpr int FIT = 16384 / STAGE, STAGES = FIT < 2 ? 2 : FIT;
    static constexpr int LOADS = TILE / 1024;
    static constexpr int MERGE = WAVES * 16 * (DH + 4) * 4;               // bytes of the waves' results, over the stages
    static constexpr int LDS = WAVES * STAGES * STAGE > MERGE ? WAVES * STAGES * STAGE : MERGE;
};

// TILES: the workgroup's 16 rows are a tile of a longer chunk, else all of a sequence's (16 at a time).
template <typename T, int DH, int WAVES, bool TILES>
__global__ __launch_bounds__(WAVES * 64, 2) void chunk_stream_kernel(ChunkKernelArgs a, int slots)
{
    typedef Stream<T, DH, WAVES> S;
    constexpr int RB = S::RB, DS = RB / 64, DT = DH / 16;
    extern __shared__ __align__(16) unsigned char st_smem[];
    __shared__ float s_ml[WAVES][16][2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), qi = lane & 15, g = lane >> 4;
    const int part = blockIdx.y, G = a.G, limit = table_limit(a.table);
    ChunkTile tile;
    if constexpr (TILES) {
        tile = find_tile(a, blockIdx.x, slots, 4, 0, lane);
    } else {
        const int b = blockIdx.x / a.Hkv, t0 = a.cu[b], end = a.cu[b + 1], n = end - t0 < a.tokens ? end - t0 : a.tokens;
        tile = ChunkTile{n <= 0 || n * G > a.stream_rows ? -1 : b, (int)blockIdx.x - b * a.Hkv, t0, n * G, a.len[b] - n, 0};
    }
    if (tile.b < 0) return;
    const int b = tile.b, kvh = tile.kvh, t0 = tile.t0, rows = tile.rows, p0 = tile.p0;
    const unsigned lds = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)st_smem + wave * (S::STAGES * S::STAGE);
    const unsigned char* mine = st_smem + wave * (S::STAGES * S::STAGE);
    const float mul = exponent_scale(a.scale);

    for (int r0 = tile.r0; r0 < (TILES ? tile.r0 + 1 : rows); r0 += 16) {
        const int r1 = r0 + 16 < rows ? r0 + 16 : rows;
        const KeyRange all = tile_keys(p0, G, r0, r1, a.window, limit, ST_STEP);
        const int parts = parts_of(all, a.stream);
        if (part >= parts) continue;
        const KeyRange k = part_of(all, a.stream, part, parts);
        const int row = r0 + qi < r1 ? r0 + qi : r1 - 1, tok = row / G, t = t0 + tok;
        const KeyRange sees = keys_of(p0 + tok, a.window, limit);
        const int p_min = p0 + r0 / G, p_max = p0 + (r1 - 1) / G;
        // a token beyond the packed ones is none of this call's
        const bool live = r0 + qi < r1 && t >= 0 && t < a.tokens;
        u32x4 qf[DS];
        load_query<T, DS>((const T*)a.q + (int64_t)(live ? t : 0) * a.q_stride + (kvh * G + row % G) * DH, g, a.scale, qf);

        const int steps = k.last > k.first ? (k.last - k.first + ST_STEP - 1) / ST_STEP : 0, own = steps > wave ? (steps - wave + WAVES - 1) / WAVES : 0;
        // tiles of one sequence share their keys in L2: 4 x 64 tokens, 16 heads over 4, 1000 keys 14.3 us, nontemporal 15.4; 4 x 12 to 24 of 40
        // heads over 600 14.4 and 14.8, with 64 features 11.3 and 11.2; 200 tokens, 32 heads over 8, 512 keys 15.5 either way
        typedef RowLoader<T, DH, !TILES> Loader;
        const Loader from(a.table, a.kv_blocks, b, kvh, a.Hkv, limit, k.last, lane);
        auto first_of = [&](int i) { return k.first + (wave + i * WAVES) * ST_STEP; };
        typename Loader::Entries en{-1, -1};
        auto issue = [&](int i) {
            const unsigned dst = lds + i % S::STAGES * S::STAGE;
            const typename Loader::Rows r = from.rows(first_of(i), en);
            from.keys(first_of(i), r, dst);
            from.values(first_of(i), r, dst + S::TILE);
        };

        float m = -INFINITY, l = 0.f;                                  // l: this lane's share of the sum
        f32x4 o[DT];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
        const int ahead = S::STAGES - 1;
        for (int i = 0; i < ahead && i < own; ++i) {
            en = from.lookup(first_of(i));
            issue(i);
        }
        if (ahead < own) en = from.lookup(first_of(ahead));
        for (int i = 0; i < own; ++i) {
            if (i + ahead < own) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // step i - 1 has left its stage
                issue(i + ahead);
                if (i + ahead + 1 < own) en = from.lookup(first_of(i + ahead + 1));
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
            const unsigned char* sV = sK + S::TILE;
            const int v_row = 4 * g + (qi >> 2), v_q = qi & 3;
            uint2 fv[sizeof(T) == 2 ? DT : 1];                         // on their way while the softmax is made
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) fv[dt] = pf_read_tr(sV + v_row * RB + (((2 * dt + (v_q >> 1)) ^ pf_swz<RB>(v_row)) << 4) + (v_q & 1) * 8);
            }
            const int j = first_of(i);
            if (j + ST_STEP - 1 > p_min || (a.window && j <= p_max - a.window)) {
                int key0 = j + 4 * g;
                asm volatile("" : "+v"(key0));                         // keeps the mask arithmetic inside this branch
#pragma unroll
                for (int r = 0; r < 4; ++r) sc[r] = key0 + r >= sees.first && key0 + r < sees.last ? sc[r] : -INFINITY;
            }
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
            if constexpr (sizeof(T) == 2) {
                typedef __attribute__((ext_vector_type(4))) short v4s;
                bf16x4 hi, lo;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    hi[r] = (bf16_t)sc[r];
                    lo[r] = (bf16_t)(sc[r] - (float)hi[r]);
                }
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    o[dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(v4s, fv[dt]), __builtin_bit_cast(v4s, lo), o[dt], 0, 0, 0);
                    o[dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(v4s, fv[dt]), __builtin_bit_cast(v4s, hi), o[dt], 0, 0, 0);
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
        const int r = tid >> 4 & 15, c = tid & 15;                     // 16 threads a row (of the first 256), features 4 * c .. +3 of every 64
        const int wtok = (r0 + r) / G, wt = t0 + wtok, h = kvh * G + (r0 + r) % G;
        const bool write = tid < 256 && r0 + r < r1 && wt >= 0 && wt < a.tokens;
        float M = -INFINITY, L = 0.f, w[WAVES];
#pragma unroll
        for (int i = 0; i < WAVES; ++i) M = fmaxf(M, s_ml[i][r][0]);
        const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            w[i] = fast_exp2(s_ml[i][r][0] - ref);
            L += s_ml[i][r][1] * w[i];
        }
        f32x4 v[DH / 64];
#pragma unroll
        for (int f = 0; f < DH / 64; ++f) {
            v[f] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < WAVES; ++i) v[f] += *(const f32x4*)(s_o + (i * 16 + r) * (DH + 4) + f * 64 + 4 * c) * w[i];
        }
        if (parts > 1) {
            if (write) {
                const int64_t at = part * a.stream.rows + a.stream_row(b, kvh, r0 + r, wt, h);
#pragma unroll
                for (int f = 0; f < DH / 64; ++f) *(f32x4*)(a.stream.acc + at * DH + f * 64 + 4 * c) = v[f];
                if (c == 0) *(float2*)(a.stream.ml + at * 2) = float2{M, L};
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
                    most = magnitude(most, v[f][e]);
                }
            const unsigned long long again = __builtin_amdgcn_ballot_w64(write && spoilt(most, L));
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
                    row_again<T, DH>(a, b, t0 + tk, hh, keys_of(p0 + tk, a.window, limit), lane);
                }
        }
        __syncthreads();                                               // before the next tile's loads overwrite the results
    }
}

// ---------------------------------------------------------------- many rows: tiles
// A workgroup of 4 waves owns 64 * QB rows, 16 * QB a wave, and a part of their keys, which pass through LDS in tiles of 64 (or 32): two
// buffers for keys, two for values, filled by direct global-to-LDS loads a tile ahead, one barrier a tile.  The products are those of
// prefill_mfma_kernel; what is taken otherwise than there:
//  * The running maximum moves only where a score passes it by more than 2^8, so most tiles reduce nothing across lanes and rescale
//    nothing; probabilities stay below 2^8, which costs no precision.  Rows of bf16 sum their probabilities, as rounded for the second
//    product, by one more MFMA with ones (64 features 3 % faster than additions); float ones leave the sum spread over four lanes.
//  * Table entries are read a tile before their rows' addresses are made, and stay scalar; 4 (64-wide heads 2) loads follow one base.
//  * A wave stops at the last key that its rows see and then moves only its share.
//  * LDS reads of a product go before its MFMAs, 6 to 8 fragments ahead, by scheduling groups: placed by the compiler, each right before its
//    use, the MFMAs waited for them: 975 us at the size below.  12 ahead are no better.
// 2048 tokens, the last of 32768, 32 heads over 8 x 128: 900 us, 1180 TFLOP/s (a matrix product of 8192^3 reaches 1400 here); 4 prompts of
// 2048 x 40 heads 213 us, 810 TFLOP/s, where prefill_mfma_kernel takes 236.  What is left are MFMAs and softmax that take turns: two waves a
// SIMD overlap by chance, MFMAs at a raised priority gave 3 %, exponentials of one half tile between the MFMAs of the other -2 to -9 %,
// scores of the next tile before the second product 0 to -5 %; 64 rows as two waves of 32: 128 features 0 to +4 %, 64 -3 to -40 %.  64 rows a
// wave spill (650 TFLOP/s); 48 rows were 20 % faster per row where such tiles fill the chip, but they rarely do.  64 rows a workgroup: tiles
// of 32 keys, registers and LDS for 4 workgroups a CU.  40 heads of 97 to 256 tokens over 400 to 1280, 8 sequences: 51 us, 3.1 TB/s of keys
// and values.  Neither HBM nor L2 (9 TB/s), LDS (30 %), MFMAs (20 %) or vector ALU bound it, but a wave's own chain of reads, MFMAs and
// softmax, 0.6 us a tile when a CU has it alone and 1.6 us beside three others; loads two tiles ahead (3 workgroups a CU) 74 us, the keys in
// two parts 78.
template <typename T, int DH, int QB>
__global__ __launch_bounds__(CT_WAVES * 64, (ct_per_cu<T, DH, QB>())) void chunk_tile_kernel(ChunkKernelArgs a, int slots)
{
    constexpr int ROWS = 16 * QB * CT_WAVES;
    extern __shared__ __align__(16) unsigned char ct_smem[];
    const int lane = threadIdx.x & 63, part = blockIdx.y;
    const ChunkTile tile = find_tile(a, blockIdx.x, slots, QB == 2 ? 7 : 6, a.stream_rows, lane);
    if (tile.b < 0) return;
    const KeyRange all = tile_keys(tile.p0, a.G, tile.r0, tile.r0 + ROWS < tile.rows ? tile.r0 + ROWS : tile.rows, a.window, table_limit(a.table), CT_ALIGN);
    const int parts = parts_of(all, a.tile);
    if (part >= parts) return;
    tile_rows<T, DH, QB, false>(a, ct_smem, tile, part_of(all, a.tile, part, parts), part, parts,
                                [&](int t, int h, KeyRange r) { row_again<T, DH>(a, tile.b, t, h, r, lane); });
}

// ---------------------------------------------------------------- parts of the keys, joined
// The sum over the parts of 2^(m_i - M) times their sums, in the order of the parts.  Rows of a single part are complete.
// Of the streaming kernel's sequences: 4 workgroups per (sequence, key/value head), a wave per row, 2 or 4 of its parts at a time (one by
// one, and a workgroup for 16 rows: 32 parts of 4 rows 13.4 us with the streaming kernel, now 12.3).
template <typename T, int DH> __global__ __launch_bounds__(256) void chunk_join_stream_kernel(ChunkKernelArgs a)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), G = a.G;
    const int b = blockIdx.x / a.Hkv, kvh = blockIdx.x - b * a.Hkv;
    const int t0 = a.cu[b], end = a.cu[b + 1], n = end - t0 < a.tokens ? end - t0 : a.tokens, rows = n * G, p0 = a.len[b] - n, limit = table_limit(a.table);
    if (n <= 0 || rows > a.stream_rows) return;
    constexpr int PER = DH / 4, SUBS = 64 / PER;                      // lanes of a part's row, parts at a time
    const int sub = lane / PER, f = lane % PER * 4;
    for (int r = blockIdx.y * 4 + wave; r < rows; r += STREAM_ROWS) {
        const int r0 = r & -STREAM_ROWS, t = t0 + r / G, h = kvh * G + r % G;
        const int parts = parts_of(tile_keys(p0, G, r0, r0 + STREAM_ROWS < rows ? r0 + STREAM_ROWS : rows, a.window, limit, ST_STEP), a.stream);
        if (parts <= 1 || t < 0 || t >= a.tokens) continue;
        const int64_t at = a.stream_row(b, kvh, r, t, h), step = a.stream.rows;
        // MAX_PARTS is a wave's lanes
        const float2 x = lane < parts ? *(const float2*)(a.stream.ml + (at + lane * step) * 2) : float2{-INFINITY, 0.f};
        const float* acc = a.stream.acc + at * DH + f;
        const float M = wave_max(x.x), w = fast_exp2(x.x - (M == -INFINITY ? 0.f : M)), L = wave_sum(x.y * w);
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
        for (int i = 0; i < parts; i += SUBS) {                        // a part behind the last is the last again, with weight 0
            const int k = i + sub;
            const float wk = __shfl(w, k, WAVE);
            v += *(const f32x4*)(acc + (k < parts ? k : parts - 1) * step * DH) * (k < parts ? wk : 0.f);
        }
#pragma unroll
        for (int d = PER; d < 64; d <<= 1)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += __shfl_xor(v[e], d, WAVE);
        const KeyRange ks = keys_of(p0 + r / G, a.window, limit);
        float most = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = ks.last > ks.first ? v[e] / L : 0.f;
            most = magnitude(most, v[e]);
        }
        if (__builtin_amdgcn_ballot_w64(spoilt(most, L))) {
            row_again<T, DH>(a, b, t, h, ks, lane);
        } else if (sub == 0) {
            typename Vec4<T>::type y;
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = from_f32<T>(v[e]);
            *(typename Vec4<T>::type*)((T*)a.out + (int64_t)t * a.out_stride + h * DH + f) = y;
        }
    }
}
// Of the tile kernel's: 1024 / DH rows a workgroup, DH / 4 threads each.
template <typename T, int DH> __global__ __launch_bounds__(256) void chunk_join_tile_kernel(ChunkKernelArgs a, int slots)
{
    constexpr int PER = DH / 4;
    const int tid = threadIdx.x, lane = tid & 63, G = a.G;
    const ChunkTile tile = find_tile(a, blockIdx.x, slots, a.tile_rows == 128 ? 7 : 6, a.stream_rows, lane);
    if (tile.b < 0) return;
    const int limit = table_limit(a.table), r1 = tile.r0 + a.tile_rows < tile.rows ? tile.r0 + a.tile_rows : tile.rows;
    const int parts = parts_of(tile_keys(tile.p0, G, tile.r0, r1, a.window, limit, CT_ALIGN), a.tile);
    if (parts <= 1) return;
    const int64_t step = a.tile.rows;
    const int row = tile.r0 + (blockIdx.y * 256 + tid) / PER, f = tid % PER * 4, tok = row / G, t = tile.t0 + tok, h = tile.kvh * G + row % G;
    const bool live = row < r1 && t >= 0 && t < a.tokens;
    const int64_t at = live ? a.row(t, h) : 0;
    const float* ml = a.tile.ml + at * 2;
    const float* acc = a.tile.acc + at * DH + f;
    // the parts' weights: a lane of the row takes a part
    constexpr int EACH = MAX_PARTS / PER;
    __shared__ float s_w[1024 / DH][MAX_PARTS];
    float2 x[EACH];
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int k = i * PER + tid % PER;
        x[i] = k < parts ? *(const float2*)(ml + k * step * 2) : float2{-INFINITY, 0.f};
        M = fmaxf(M, x[i].x);
    }
#pragma unroll
    for (int d = PER / 2; d; d >>= 1) M = fmaxf(M, __shfl_xor(M, d, WAVE));
    const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const float w = fast_exp2(x[i].x - ref);
        s_w[tid / PER][i * PER + tid % PER] = w;
        L = fmaf(x[i].y, w, L);
    }
#pragma unroll
    for (int d = PER / 2; d; d >>= 1) L += __shfl_xor(L, d, WAVE);
    __syncthreads();
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int k = 0; k < parts; ++k) v += *(const f32x4*)(acc + k * step * DH) * s_w[tid / PER][k];
    const KeyRange ks = keys_of(tile.p0 + tok, a.window, limit);
    float most = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[e] = ks.last > ks.first ? v[e] / L : 0.f;
        most = magnitude(most, v[e]);
    }
    // the rows of a wave are whole ones
    const unsigned long long again = __builtin_amdgcn_ballot_w64(live && spoilt(most, L));
    const unsigned long long mine = PER == 32 ? 0xffffffffull << (lane & 32) : 0xffffull << (lane & 48);
    if (live && !(again & mine)) {
        typename Vec4<T>::type x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = from_f32<T>(v[e]);
        *(typename Vec4<T>::type*)((T*)a.out + (int64_t)t * a.out_stride + h * DH + f) = x;
    }
    for (int j = 0; j < 64 / PER; ++j)
        if (again >> (j * PER) & (PER == 32 ? 0xffffffffull : 0xffffull)) {
            const int rr = __builtin_amdgcn_readfirstlane(row - lane / PER) + j, tk = rr / G;
            row_again<T, DH>(a, tile.b, tile.t0 + tk, tile.kvh * G + rr % G, keys_of(tile.p0 + tk, a.window, limit), lane);
        }
}

// ---------------------------------------------------------------- launches
struct ChunkPlan {
    bool stream, tile;               // which kernels run
    bool small;                      // the streaming kernel, in tiles
    int waves;                       // of the streaming kernel's workgroups
    int qb;                          // row blocks per wave of the tile kernel
    int64_t slots;
    ChunkKernelArgs::Cut stream_cut, tile_cut;
};
static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

static ChunkKernelArgs::Cut cut_to(int64_t parts, int64_t max_len, int align)
{
    if (parts <= 1) return {1, 0x7fffffff, 0, nullptr, nullptr};
    int64_t keys = ceil_div(ceil_div(max_len, parts), align) * align;
    return {(int)ceil_div(max_len, keys), (int)keys, 0, nullptr, nullptr};
}
// Parts for `wgs` workgroups that each would take up to max_len keys, so that `want` come of them, no part shorter than `least` keys.
static ChunkKernelArgs::Cut cut_keys(int64_t wgs, int64_t max_len, int64_t want, int least, int align)
{
    int64_t parts = want / wgs, most = ceil_div(max_len, least);
    parts = parts < most ? parts : most;
    parts = parts < MAX_PARTS ? parts : MAX_PARTS;
    return cut_to(parts, max_len, align);
}

// Parts for the tile kernel, of `tiles` workgroups with `seen` keys each: those with which the chip is done first.  Time is counted in keys of
// a full CU: its `per_cu` workgroups take 2 of 10 shares together and 8 each by its own, and each part another 64 for its sums.  Joining
// takes as long as 256 keys (7 us), of float ones 64.  2 x 512 tokens, 32 heads over 8 x 128, of 4096 keys are 256 workgroups: in 2 parts
// 81 us, whole 98, in 3 parts, which a second round of workgroups has to take, 100; 1 x 512 behind 32000, 128 workgroups: 4 parts 258,
// 5 parts 342.  `tiles` are those of sequences of the mean length, the last one of each partly filled: as many as run where all bring the same,
// about as many where they do not.  (Counted as if packed without gaps, us of then / now: 32 x 20 tokens of 40 heads over 2000 keys 306 / 251, 32 x 5
// of 32 heads over 8, 4000 keys 115 / 103, 8 x 24 of 40 heads, 4000 keys 148 / 134; 10 x 20 to 90 of 16 heads over 4, 400 to 3000 keys 33.5 / 34.7.)
// Beside the streaming kernel, which takes an unknown number of the sequences, they are counted packed: 23 single tokens and 3 x 8 to 26 of 16 heads
// over 8 x 64, window 1000, 25.9, by the mean length of all 29.6.
static ChunkKernelArgs::Cut cut_tiles(int64_t tiles, int per_cu, int64_t seen, int least, int each, int join)
{
    const int64_t round = 256 * per_cu;
    int64_t parts = 1, best = 0;
    for (int64_t p = 1; p <= MAX_PARTS && (p == 1 || p <= ceil_div(seen, least)); ++p) {
        const int64_t wgs = tiles * p, left = ceil_div(wgs % round, 256);
        if (p > 1 && wgs > 4 * round) break;
        const int64_t shares = wgs / round * 10 * per_cu + (left ? 2 * per_cu + 8 * left : 0);
        const int64_t time = shares * (ceil_div(seen, p) + (p > 1 ? each : 0)) + (p > 1 ? 10 * per_cu * join : 0);
        if (p == 1 || time < best) {
            best = time;
            parts = p;
        }
    }
    return cut_to(parts, seen, CT_ALIGN);
}
static ChunkPlan chunk_plan(const ChunkAttnArgs& a)
{
    ChunkPlan p{};
    const int64_t G = a.H / a.Hkv, rows = (int64_t)a.max_new * G, T = a.tokens;
    const int64_t seen = a.window && (int64_t)a.window + a.max_new < a.max_len ? (int64_t)a.window + a.max_new : a.max_len;
    const bool f32 = a.dtype == DT_F32;
    const ChunkKernelArgs::Cut whole{1, 0x7fffffff, 0, nullptr, nullptr};
    p.stream_cut = p.tile_cut = whole;
    // A call of few rows by tiles of 16, whose keys go to 8 waves: shorter chains than the tile kernel's, and no second launch where that one
    // cuts them.  Up to 1024 keys and 512 workgroups; of 64 features, whose tiles are cheaper, 320 and no more than 1024 keys a CU; float x 128
    // has 4 waves and gains nothing.  us, tile kernel first: bf16 x 128, 32 heads over 8, 32 to 64 tokens over 512 16.1, 10.0, 128 to 256 16.9,
    // 15.2; 40 heads, 4 x 12 to 24 over 600 30.8, 13.1; 16 heads over 4, 4 x 64 over 2000 22.1, 21.7; x 64, 40 heads, 4 x 12 to 24 over 600 19.7, 10.0;
    // 32 over 8, 128 to 256 over 512 10.9, 12.7; float x 64, 16 over 4, 64 over 512 14.9, 12.0.
    const int64_t small = (ceil_div(T * G, STREAM_ROWS) + a.n_seqs - 1) * a.Hkv;
    p.small = rows > STREAM_ROWS && seen <= 1024 && (a.dh == 64 ? small <= 320 && small * seen <= 256 * 1024 : !f32 && small <= 512);
    p.tile = rows > STREAM_ROWS && !p.small;
    // Beside longer sequences one of up to 16 rows goes to the streaming kernel, not where there can be none (one sequence, or all bring
    // max_new tokens), and not where they are few and none is long: the tile kernel then takes it along, in the time that its other
    // sequences take, and a launch or two are saved (8 chunks of 97 to 256 tokens, 40 heads: 50 us).
    p.stream = !p.tile || (a.n_seqs > 1 && T <= (int64_t)(a.n_seqs - 1) * a.max_new + STREAM_ROWS / G && (T * G < (int64_t)64 * a.n_seqs || seen > 4096));
    if (p.small) {
        p.slots = T * G / STREAM_ROWS + a.n_seqs;
    } else if (p.stream) {
        const int64_t wgs = (int64_t)a.n_seqs * a.Hkv;
        // At most one workgroup a CU: of 8 waves (float x 128 fills a CU's LDS with 4), as many parts as CUs are left.  Short ones whole: a
        // second launch takes longer than the keys (1 x 40 heads of 512 keys: 10.3 us, in 4 parts 10.0 and a launch; of 1024: 15.4, 11.4).
        // 6 x 40 heads of 2048 keys: 41.7 us, with 4 waves in 8 parts 47.2.
        // More: two of 4 waves a CU; four times as many workgroups even out lengths that differ (64 x 8 heads of 500 to 8100 keys 182 us, whole
        // 200; of 4096 each 169 and 161).
        if (wgs <= 256) {
            p.waves = f32 && a.dh == 128 ? ST_WAVES : 8;
            p.stream_cut = seen <= 640 ? whole : cut_keys(wgs, seen, 256, 128, ST_STEP);
        } else {
            p.waves = ST_WAVES;
            p.stream_cut = cut_keys(wgs, seen, 2048, 256, ST_STEP);
        }
    }
    if (p.tile) {
        const int64_t wgs = (ceil_div(T * G, 128) + a.n_seqs - 1) * a.Hkv;
        // 128 rows a workgroup where several of its tiles share their keys, with 64 features only where the chip is full of them: bf16, us of
        // 64 / 128 rows: x 128, 40 heads of 128 tokens over 1024, 12 sequences 64 / 78, 50 251 / 241; 32 heads over 8, 512 tokens over 4096, 1
        // sequence 73 / 64, 16 629 / 492; the same x 64, 4 sequences 92 / 94, 8 170 / 166, 16 334 / 292.  Float: registers leave room for 64.
        p.qb = !f32 && rows >= 512 && (a.dh == 128 || wgs >= 1024) ? 2 : 1;
        p.slots = T * G / (64 * p.qb) + a.n_seqs;
        const int per_cu = f32 ? a.dh == 128 ? ct_per_cu<float, 128, 1>() : ct_per_cu<float, 64, 1>()
                         : p.qb == 1 ? ct_per_cu<bf16_t, 128, 1>() : a.dh == 128 ? ct_per_cu<bf16_t, 128, 2>() : ct_per_cu<bf16_t, 64, 2>();
        const int64_t seqs = p.stream ? 1 : a.n_seqs, tiles = seqs * ceil_div(ceil_div(T * G, seqs), 64 * p.qb) * a.Hkv;
        p.tile_cut = cut_tiles(tiles, per_cu, seen, f32 ? 128 : 256, f32 ? 32 : 64, f32 ? 64 : 256);
    }
    // rows of the parts: those of the packed tokens, or see stream_row
    p.tile_cut.rows = T * a.H;
    p.stream_cut.rows = p.tile ? (int64_t)a.n_seqs * a.Hkv * STREAM_ROWS : T * a.H;
    return p;
}
static size_t cut_floats(const ChunkKernelArgs::Cut& c, int dh) { return c.parts <= 1 ? 0 : (size_t)c.parts * c.rows * (dh + 2); }

size_t chunk_attn_workspace(const ChunkAttnArgs& a)
{
    const ChunkPlan p = chunk_plan(a);
    return (cut_floats(p.stream_cut, a.dh) + cut_floats(p.tile_cut, a.dh)) * sizeof(float);
}

template <typename T, int DH, int QB> static hipError_t launch_tile(const ChunkKernelArgs& k, const ChunkPlan& p, hipStream_t s)
{
    static LdsLimit limit[MAX_DEVICES];
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= MAX_DEVICES) dev = 0;
    hipError_t e = limit[dev].raise((const void*)chunk_tile_kernel<T, DH, QB>, ct_lds<T, DH, QB>());
    if (e != hipSuccess) return e;
    const int64_t wgs = p.slots * k.Hkv;
    if (p.slots > 0x7fffffff || wgs * CT_WAVES * 64 * p.tile_cut.parts > MAX_LAUNCH_THREADS) return hipErrorInvalidValue;
    chunk_tile_kernel<T, DH, QB><<<dim3((unsigned)wgs, p.tile_cut.parts), CT_WAVES * 64, ct_lds<T, DH, QB>(), s>>>(k, (int)p.slots);
    return hipGetLastError();
}

template <typename T, int DH, int WAVES, bool TILES> static hipError_t launch_stream(const ChunkKernelArgs& k, const ChunkPlan& p, hipStream_t s)
{
    typedef Stream<T, DH, WAVES> S;
    static LdsLimit limit[MAX_DEVICES];
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= MAX_DEVICES) dev = 0;
    hipError_t e = limit[dev].raise((const void*)chunk_stream_kernel<T, DH, WAVES, TILES>, S::LDS);
    if (e != hipSuccess) return e;
    const int64_t wgs = (TILES ? p.slots : k.n_seqs) * k.Hkv;
    if (wgs * WAVES * 64 * p.stream_cut.parts > MAX_LAUNCH_THREADS) return hipErrorInvalidValue;
    chunk_stream_kernel<T, DH, WAVES, TILES><<<dim3((unsigned)wgs, p.stream_cut.parts), WAVES * 64, S::LDS, s>>>(k, (int)p.slots);
    return hipGetLastError();
}

template <typename T, int DH> static hipError_t launch_chunk(const ChunkAttnArgs& a, hipStream_t s)
{
    const ChunkPlan p = chunk_plan(a);
    ChunkKernelArgs k{a.cu, a.len, a.n_seqs, a.tokens, a.q, a.q_stride, a.kv_blocks, a.table, a.H, a.Hkv, a.H / a.Hkv, a.scale, a.window, a.out, a.out_stride,
                      p.stream_cut, p.tile_cut, 0, 64 * p.qb};
    float* w = a.workspace;
    for (ChunkKernelArgs::Cut* c : {&k.stream, &k.tile}) {
        if (c->parts <= 1) continue;
        c->acc = w;
        c->ml = w + (size_t)c->parts * c->rows * DH;
        w += cut_floats(*c, DH);
    }
    // without a tile kernel the streaming one takes every sequence, in tiles of 16 rows
    k.stream_rows = !p.tile ? 0x7fffffff : p.stream ? STREAM_ROWS : 0;
    hipError_t e;
    if (p.stream) {
        if constexpr (sizeof(T) == 2 || DH == 64)
            e = p.small ? launch_stream<T, DH, 8, true>(k, p, s) : p.waves == 8 ? launch_stream<T, DH, 8, false>(k, p, s) : launch_stream<T, DH, ST_WAVES, false>(k, p, s);
        else e = launch_stream<T, DH, ST_WAVES, false>(k, p, s);
        if (e != hipSuccess) return e;
    }
    if (p.tile) {
        if constexpr (sizeof(T) == 2) e = p.qb == 2 ? launch_tile<T, DH, 2>(k, p, s) : launch_tile<T, DH, 1>(k, p, s);
        else e = launch_tile<T, DH, 1>(k, p, s);
        if (e != hipSuccess) return e;
    }
    if (p.stream && p.stream_cut.parts > 1) {
        chunk_join_stream_kernel<T, DH><<<dim3((unsigned)(a.n_seqs * a.Hkv), 4), 256, 0, s>>>(k);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (p.tile && p.tile_cut.parts > 1) {
        chunk_join_tile_kernel<T, DH><<<dim3((unsigned)(p.slots * a.Hkv), k.tile_rows * DH / 1024), 256, 0, s>>>(k, (int)p.slots);
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
