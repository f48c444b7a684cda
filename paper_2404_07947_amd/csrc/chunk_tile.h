// Tiles of many query rows against keys and values of a paged cache, by a workgroup: what chunk_tile_kernel and prefix_tile_kernel share.
#pragma once
#include "chunk.h"

namespace exe {

// Query rows from r0 on of a run of `rows`: row r is token t0 + r / G, head kvh * G + r % G, at position p0 + r / G; b: their row of the table.
struct ChunkTile { int b, kvh, t0, rows, p0, r0; };

constexpr int CT_WAVES = 4, CT_ALIGN = 64;
enum { VECTOR = 0x402, MATRIX = 0x008, LDS_READ = 0x100 };            // kinds of instructions, for the scheduler
template <typename T, int DH, int QB> constexpr int ct_keys() { return QB == 1 && DH * (int)sizeof(T) > 128 ? 32 : 64; }
template <typename T, int DH, int QB> constexpr int ct_lds() { return 4 * ct_keys<T, DH, QB>() * DH * (int)sizeof(T); }
template <typename T, int DH, int QB> constexpr int ct_per_cu()
{
    if (sizeof(T) == 4) return DH == 128 ? 2 : 3;
    return QB == 2 ? DH == 128 ? 2 : 3 : 4;
}

// The rows of a tile against keys k of theirs.  WHOLE: they see all of them, and the result goes to part `part` in any case; else each sees what its
// position and the window leave, and the result is a part's where there are several.  again_by: computes a row (token, head, its keys) once more.
template <typename T, int DH, int QB, bool WHOLE, typename Args, typename F>
__device__ __forceinline__ void tile_rows(const Args& a, unsigned char* ct_smem, const ChunkTile& tile, KeyRange k, int part, int parts, F again_by)
{
    constexpr int RB = DH * (int)sizeof(T), DS = RB / 64, DT = DH / 16, KT = ct_keys<T, DH, QB>(), KB = KT / 16, TILE = KT * RB;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), qi = lane & 15, g = lane >> 4, G = a.G;
    const int b = tile.b, kvh = tile.kvh, t0 = tile.t0, rows = tile.rows, p0 = tile.p0, r0 = tile.r0, limit = table_limit(a.table);
    const float mul = exponent_scale(a.scale);
    const int w0 = r0 + wave * (16 * QB);                              // this wave's first row
    const int wl = w0 + 16 * QB < rows ? w0 + 16 * QB - 1 : rows - 1;  // and last one
    const bool active = w0 < rows;
    const int p_min = p0 + w0 / G, p_max = p0 + wl / G;
    const int n_tiles = k.last > k.first ? (k.last - k.first + KT - 1) / KT : 0;
    // of these, the leading ones that hold a key which a row of this wave sees; in the others it only moves its share
    const int mine = !active ? 0 : WHOLE ? k.last - k.first : keys_of(p_max, a.window, limit).last - k.first, n_mine = mine <= 0 ? 0 : (mine + KT - 1) / KT < n_tiles ? (mine + KT - 1) / KT : n_tiles;

    u32x4 qf[QB][DS];
    KeyRange sees[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        int row = w0 + qb * 16 + qi;
        row = row < rows ? row : rows - 1;
        int t = t0 + row / G;
        sees[qb] = WHOLE ? KeyRange{0, k.last} : keys_of(p0 + row / G, a.window, limit);
        load_query<T, DS>((const T*)a.q + (int64_t)(t >= 0 && t < a.tokens ? t : 0) * a.q_stride + (kvh * G + row % G) * DH, g, a.scale, qf[qb]);
    }

    // ---- loaders.  Tiles of 64 keys: wave w fills rows 16 * w .. +15 of keys and of values; of 32: waves 0 and 1 the keys, 2 and 3 the values
    const unsigned lds = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)ct_smem;
    typedef RowLoader<T, DH, false> Loader;
    typedef typename Loader::Entries Entries;
    typedef typename Loader::Rows Rows;
    const Loader from(a.table, a.kv_blocks, b, kvh, a.Hkv, limit, k.last, lane);
    const int my_rows = wave % KB * 16;
    const unsigned dst = lds + my_rows * RB;
    auto first_of = [&](int kt) { return k.first + kt * KT + my_rows; };
    auto lookup = [&](int kt) { return from.lookup(first_of(kt)); };
    auto load_k = [&](int kt, const Rows& r) { from.keys(first_of(kt), r, dst + (kt & 1) * TILE); };
    auto load_v = [&](int kt, const Rows& r) { from.values(first_of(kt), r, dst + (2 + (kt & 1)) * TILE); };
    Entries en;
    auto bring = [&](int kt) {
        const Rows r = from.rows(first_of(kt), en);
        if (KT == 64 || wave < 2) load_k(kt, r);
        if (KT == 64 || wave >= 2) load_v(kt, r);
        en = lookup(kt + 1);
    };

    // sum: of float rows this lane's share, in [0]; of bf16 the whole, in each element
    f32x4 o[QB][DT], sum[QB];
    float m[QB];
    bf16x8 ones;
#pragma unroll
    for (int i = 0; i < 8; ++i) ones[i] = (bf16_t)1.f;
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        m[qb] = -INFINITY;
        sum[qb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[qb][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    typedef f32x4 Scores[QB][KB];
    auto scores = [&](int kt, Scores& s) {
        const unsigned char* sK = ct_smem + (kt & 1) * TILE;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
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
    // the largest raw score of this lane's
    auto largest = [&](Scores& s, float (&mx)[QB]) {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            mx[qb] = -INFINITY;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int r = 0; r < 4; ++r) mx[qb] = fmaxf(mx[qb], s[qb][kb][r]);
        }
    };
    // masks, and moves the running maxima where a score passes one by more than 2^8
    auto look = [&](int kt, Scores& s, float (&mx)[QB]) {
        const int j = k.first + kt * KT;
        if ((!WHOLE && j + KT - 1 > p_min) || j + KT > k.last || (!WHOLE && a.window && j <= p_max - a.window)) {
            int key0 = j + 4 * g;
            asm volatile("" : "+v"(key0));                             // keeps the mask arithmetic inside this branch
#pragma unroll
            for (int qb = 0; qb < QB; ++qb)
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        s[qb][kb][r] = key0 + kb * 16 + r < (sees[qb].last < k.last ? sees[qb].last : k.last) ? s[qb][kb][r] : -INFINITY;
            if (!WHOLE && a.window) {
#pragma unroll
                for (int qb = 0; qb < QB; ++qb)
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            s[qb][kb][r] = key0 + kb * 16 + r >= sees[qb].first ? s[qb][kb][r] : -INFINITY;
            }
            largest(s, mx);
        }
        bool grew = false;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            mx[qb] *= mul;
            grew |= mx[qb] > m[qb] + 8.f;
        }
        if (__builtin_amdgcn_ballot_w64(grew)) {
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                float to = fmaxf(m[qb], rows_max(mx[qb])), ref = to == -INFINITY ? 0.f : to, alpha = fast_exp2(m[qb] - ref);
                sum[qb] *= alpha;
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
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[qb][kb][r] = fast_exp2(fmaf(s[qb][kb][r], mul, -ref));
                    if (sizeof(T) == 4) sum[qb][0] += s[qb][kb][r];
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
                for (int kb = 0; kb < KB; ++kb)
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
            for (int ks = 0; ks < KB / 2; ++ks) {
                // One rounding to bf16 per probability, half a step of the result's own type.  WHOLE: two numbers of it, what is cut off and what that leaves, 15 bits
                // and more, as the rows of smaller groups and own positions have them (prefix_stream_kernel): how many sequences share a prefix does not
                // decide how exact they are.  Half as many products again, for a document of 30001 positions 95 us instead of 82; off by 1.66e-3
                // of the result instead of 2.3e-3, of which its own rounding to bf16 is 1.66e-3.
                bf16x8 pf[QB], low[QB];
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) {
                    auto p = [&](int e) { return s[qb][2 * ks + (e >> 2)][e & 3]; };
                    if constexpr (WHOLE) {
                        u32x4 high;
#pragma unroll
                        for (int e = 0; e < 8; e += 2) {
                            const unsigned x = __float_as_uint(p(e)), y = __float_as_uint(p(e + 1));
                            high[e / 2] = __builtin_amdgcn_perm(y, x, 0x07060302);               // the upper halves
                            low[qb][e] = (bf16_t)(p(e) - __uint_as_float(x & 0xffff0000u));
                            low[qb][e + 1] = (bf16_t)(p(e + 1) - __uint_as_float(y & 0xffff0000u));
                        }
                        pf[qb] = __builtin_bit_cast(bf16x8, high);
                        sum[qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, low[qb], sum[qb], 0, 0, 0);
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) pf[qb][e] = (bf16_t)p(e);
                    }
                }
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) sum[qb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pf[qb], sum[qb], 0, 0, 0);
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    const int at = ((2 * dt + (v_q >> 1)) ^ pf_swz<RB>(v_row)) << 4;
                    uint2 lo = pf_read_tr(sV + ks * 32 * RB + at), hi = pf_read_tr(sV + (ks * 32 + 16) * RB + at);
                    bf16x8 fv = __builtin_bit_cast(bf16x8, uint4{lo.x, lo.y, hi.x, hi.y});
                    if constexpr (WHOLE) {
#pragma unroll
                        for (int qb = 0; qb < QB; ++qb) o[qb][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fv, low[qb], o[qb][dt], 0, 0, 0);
                    }
#pragma unroll
                    for (int qb = 0; qb < QB; ++qb) o[qb][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fv, pf[qb], o[qb][dt], 0, 0, 0);
                }
            }
        }
    };

    if (n_tiles > 0) {
        // Some LDS reads go before the MFMAs and the others between them, the values' after the exponentials: left to itself the compiler reads
        // each fragment right before its use, and the MFMAs wait.
        constexpr int AHEAD = QB == 1 ? 6 : 8;
        Scores s;
        float mx[QB];
        en = lookup(0);
        bring(0);
        auto arrive = [&](int kt) {
            wait_loads<0>();
            __syncthreads();
            if (kt + 1 < n_tiles) bring(kt + 1);
        };
        auto iteration = [&](int kt) {
            arrive(kt);
            __builtin_amdgcn_s_setprio(1);                             // MFMAs go before another wave's softmax
            scores(kt, s);
            __builtin_amdgcn_sched_group_barrier(LDS_READ, AHEAD, 0);
#pragma unroll
            for (int i = 0; i < KB * DS; ++i) {
                __builtin_amdgcn_sched_group_barrier(MATRIX, QB, 0);
                __builtin_amdgcn_sched_group_barrier(LDS_READ, 1, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(0);
            largest(s, mx);
            look(kt, s, mx);
            exponentials(s);
            __builtin_amdgcn_s_setprio(1);
            values(kt, s);
            __builtin_amdgcn_sched_group_barrier(LDS_READ, AHEAD, 0);
            __builtin_amdgcn_sched_group_barrier(VECTOR, 20 * QB * KB, 0);
#pragma unroll
            for (int i = 0; i < KB / 2 * DT; ++i) {
                __builtin_amdgcn_sched_group_barrier(MATRIX, WHOLE ? 2 * QB : QB, 0);
                __builtin_amdgcn_sched_group_barrier(LDS_READ, 2, 0);
            }
            __builtin_amdgcn_s_setprio(0);
        };
        int kt = 0;
        for (; kt + 1 < n_mine; kt += 2) {
            iteration(kt);
            iteration(kt + 1);
        }
        if (kt < n_mine) iteration(kt++);
        for (; kt < n_tiles; ++kt) arrive(kt);
    }
    if (!active) return;

    // lane (qi, g) holds features 16 * dt + 4 * g .. +3 of its rows
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int row = w0 + qb * 16 + qi, t = t0 + row / G, h = kvh * G + row % G;
        const bool write = row < rows && t >= 0 && t < a.tokens;
        const float total = sizeof(T) == 4 ? rows_sum(sum[qb][0]) : sum[qb][0];
        if (WHOLE || parts > 1) {
            if (!write) continue;
            const int64_t at = part * a.tile.rows + ((int64_t)t * a.H + h);
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) *(f32x4*)(a.tile.acc + at * DH + dt * 16 + 4 * g) = o[qb][dt];
            if (g == 0) *(float2*)(a.tile.ml + at * 2) = float2{m[qb], total};
            continue;
        }
        const bool any = sees[qb].last > sees[qb].first;
        const float inv = 1.f / total;
        float most = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                o[qb][dt][e] = any ? o[qb][dt][e] * inv : 0.f;
                most = magnitude(most, o[qb][dt][e]);
            }
        const unsigned long long lanes = __builtin_amdgcn_ballot_w64(write && spoilt(most, total));
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
            again_by(t0 + tk, hh, keys_of(p0 + tk, a.window, limit));
        }
    }
}

}  // namespace exe
