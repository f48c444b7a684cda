// Attention of new tokens over a paged cache in which the sequences of a group share their first positions.
//
// The prefix of a group is read once for all of its sequences: the query rows of the group that share a key/value head, its new tokens times the
// G = H / Hkv heads, are packed into tiles of 16 * QB rows, which all see the whole prefix and need no mask there.  The positions behind
// it are each sequence's own, in tiles of 16 rows.  One launch takes both kinds, cut into parts of their keys; what a part makes of a row (the
// sum of values by 2^(score - maximum), the maximum and the sum of probabilities, in float) is joined by a second one.
// Which sequences are whose, and how many parts there are, the kernels find from what lies on the device, so that a captured launch follows
// it; the host's bounds only size the launch.
#include <algorithm>
#include <type_traits>

#include "chunk_tile.h"

namespace exe {

constexpr int PX_STEP = 16, PX_PARTS = WAVE;
constexpr float NO_PART = -2.f, NO_KEYS = -1.f;       // in place of a sum of probabilities: a part that is not there, a row without keys

// n / d for 0 <= n < 2^31 as (n + the upper half of n * mul) >> shift, where 2^shift is the first power of two from d on and mul is 2^32 (2^shift - d) / d, rounded
// up: 2^32 + mul = 2^(32 + shift) / d + e with e <= 1, and n e < 2^31 cannot reach the next whole number.  A division by a number that is not known takes 20 to 30
// instructions, one after the other, and a workgroup here begins with three of them (us a call, before and now: 12 groups 45.1, 44.1, float groups 11.6, 11.3).
struct Divisor {
    unsigned d, mul, shift;
    static Divisor of(int64_t d)
    {
        unsigned s = 0;
        while ((1ll << s) < d) ++s;
        return Divisor{(unsigned)d, (unsigned)(((uint64_t)((1ll << s) - d) << 32) / d + 1), s};
    }
    __device__ __forceinline__ int quotient(int n) const { return (int)((__umulhi(mul, (unsigned)n) + (unsigned)n) >> shift); }
    __device__ __forceinline__ int rest(int n, int q) const { return n - q * (int)d; }
};

struct PrefixKernelArgs {
    const int32_t *cu, *len, *cu_groups, *prefix;
    int n_seqs, tokens, n_groups;
    const void* q; int64_t q_stride;
    const void* kv_blocks;
    PagedTable table;
    int H, Hkv, G;
    float scale;
    void* out; int64_t out_stride;
    // Keys go to workgroups in parts of `keys`, at most `parts` (the last takes what is left).  Part i of row r: acc[i * rows + r][DH], ml[i * rows +
    // r][maximum, sum], the prefix's parts in front of the own ones'.
    struct Cut { int parts, keys; } shared, own;
    struct { int64_t rows; float *acc, *ml; } tile;
    static constexpr int window = 0;
    int own_tiles;                    // of a sequence's rows, side by side
    unsigned shared_units;            // workgroups of prefix tiles
    Divisor by_G, by_Hkv, by_parts, by_tiles, by_units, by_quarter;   // G, Hkv; own.parts, own_tiles; workgroups of a slot of tiles; of a token in the join
};

// A group: sequences b0 .. b1 - 1, new tokens t0 .. t1 - 1, and the positions that they share.  Those in front of every new token of the group
// count: what a call passes beyond is a sequence's own.  They are read through table row `front`, of the first sequence that has new tokens: nothing of one
// without any is looked at, so a continuation that has ended may stay in its place.  Group n_groups is what lies behind the last one, without a prefix.
struct PrefixGroup { int g, b0, b1, t0, t1, prefix, front; };
__device__ __forceinline__ int lanes_min(int v)
{
    auto with = [&](int w) { v = w < v ? w : v; };
    with(dpp_move_int<0xB1>(v));
    with(dpp_move_int<0x4E>(v));
    with(dpp_move_int<0x141>(v));
    with(dpp_move_int<0x140>(v));
    const int a = __builtin_amdgcn_readlane(v, 0), b = __builtin_amdgcn_readlane(v, 16), c = __builtin_amdgcn_readlane(v, 32), d = __builtin_amdgcn_readlane(v, 48);
    const int ab = a < b ? a : b, cd = c < d ? c : d;
    return ab < cd ? ab : cd;
}
// The group of tile slot `at` (those of group g begin at floor(first token * G / rows of a tile) + g, see ChunkTile), or of sequence `at`.
template <bool SLOT> __device__ __forceinline__ PrefixGroup find_group(const PrefixKernelArgs& a, int at, int tile_shift, int lane)
{
    auto before = [&](int first_seq, int first_token, int g) { return SLOT ? (int)((int64_t)first_token * a.G >> tile_shift) + g <= at : first_seq <= at; };
    PrefixGroup r;
    int least;
    if (a.n_seqs < WAVE && a.n_groups < WAVE - 1) {                    // all of it in one trip to memory
        const int c = a.cu[lane < a.n_seqs ? lane : a.n_seqs], l = a.len[lane < a.n_seqs ? lane : a.n_seqs - 1];
        int first = a.n_seqs, shared = 0;
        if (a.n_groups) {
            if (lane <= a.n_groups) first = a.cu_groups[lane];
            shared = a.prefix[lane < a.n_groups ? lane : a.n_groups - 1];
        } else if (lane == 0) first = 0;
        first = first < 0 ? 0 : first < a.n_seqs ? first : a.n_seqs;
        const int token = __shfl(c, first, WAVE), n = __shfl(c, lane + 1, WAVE) - c;
        r.g = __popcll(__builtin_amdgcn_ballot_w64(lane <= a.n_groups && before(first, token, lane))) - 1;
        if (r.g < 0) return PrefixGroup{-1, 0, 0, 0, 0, 0, 0};
        r.b0 = __builtin_amdgcn_readlane(first, r.g);
        r.b1 = __builtin_amdgcn_readlane(first, r.g + 1);
        r.t0 = __builtin_amdgcn_readlane(token, r.g);
        r.t1 = __builtin_amdgcn_readlane(token, r.g + 1);
        least = __builtin_amdgcn_readlane(shared, r.g);
        const bool counts = lane >= r.b0 && lane < r.b1 && n > 0;
        const unsigned long long some = __builtin_amdgcn_ballot_w64(counts);
        r.front = some ? __builtin_ctzll(some) : r.b0;
        const int p0 = lanes_min(counts ? l - n : 0x7fffffff);
        least = p0 < least ? p0 : least;
    } else {
        auto first_of = [&](int g) {
            const int first = g > a.n_groups ? a.n_seqs : a.n_groups ? a.cu_groups[g] : 0;
            return first < 0 ? 0 : first < a.n_seqs ? first : a.n_seqs;
        };
        r.g = wave_search(0, a.n_groups + 1, lane, [&](int g) {
            const int first = first_of(g);
            return before(first, SLOT ? a.cu[first] : 0, g);
        });
        r.g = __builtin_amdgcn_readfirstlane(r.g);
        if (r.g < 0) return PrefixGroup{-1, 0, 0, 0, 0, 0, 0};
        r.b0 = first_of(r.g);
        r.b1 = first_of(r.g + 1);
        r.t0 = a.cu[r.b0];
        r.t1 = a.cu[r.b1];
        least = r.g < a.n_groups ? a.prefix[r.g] : 0;
        int p0 = 0x7fffffff;
        r.front = 0x7fffffff;
        if (least > 0) {
            for (int b = r.b0 + lane; b < r.b1; b += WAVE) {
                const int n = a.cu[b + 1] - a.cu[b];
                if (n <= 0) continue;
                const int p = a.len[b] - n;
                p0 = p < p0 ? p : p0;
                r.front = b < r.front ? b : r.front;
            }
            p0 = lanes_min(p0);
            r.front = lanes_min(r.front);
        }
        if (r.front == 0x7fffffff) r.front = r.b0;
        least = p0 < least ? p0 : least;
    }
    auto scalar = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    return PrefixGroup{scalar(r.g), scalar(r.b0), scalar(r.b1), scalar(r.t0), scalar(r.t1), scalar(r.g < a.n_groups && least > 0 ? least : 0), scalar(r.front)};
}

__device__ __forceinline__ int parts_of(KeyRange k, const PrefixKernelArgs::Cut& cut)
{
    if (k.last <= k.first) return 1;
    const int n = (int)(((int64_t)k.last - k.first + cut.keys - 1) / cut.keys);
    return n < cut.parts ? n : cut.parts;
}
__device__ __forceinline__ KeyRange part_of(KeyRange k, const PrefixKernelArgs::Cut& cut, int part, int parts)
{
    const int first = k.first + part * cut.keys;
    return KeyRange{first, part + 1 < parts ? first + cut.keys : k.last};
}

template <typename T, int DH, int WAVES> struct PrefixStream {
    static constexpr int RB = DH * (int)sizeof(T), TILE = PX_STEP * RB, STAGE = 2 * TILE;
    static constexpr int FIT = 16384 / STAGE, STAGES = FIT < 2 ? 2 : FIT, LOADS = TILE / 1024;
    static constexpr int LDS = WAVES * STAGES * STAGE, MERGE = WAVES * 16 * (DH + 4) * 4;      // bytes of the waves' results, over the stages
    static_assert(MERGE + WAVES * 16 * 8 <= LDS, "results, maxima and sums");
};

// Row (t, h) of sequence b at position p, by one wave (see chunk_row).
template <typename T, int DH> __device__ __forceinline__ void prefix_row(const PrefixKernelArgs& a, const PrefixGroup& gr, int b, int p, int t, int h, int lane)
{
    const int64_t head = (int64_t)DH << a.table.shift;
    chunk_row<T, DH>((const T*)a.q + (int64_t)t * a.q_stride + h * DH, (const T*)a.kv_blocks + h / a.G * head, 2 * a.Hkv * head, a.Hkv * head, a.table.shift,
                     [&](int j) { return a.table.block(j < gr.prefix ? gr.front : b, j); }, keys_of(p, 0, table_limit(a.table)), a.scale * LOG2E, lane,
                     (T*)a.out + (int64_t)t * a.out_stride + h * DH);
}

// Query rows r0 .. r1 - 1 of a run of packed tokens from t0 on (row r: token t0 + r / G, head kvh * G + r % G) against keys k of table row b; row
// r sees keys lo .. hi(r / G) - 1 of them.  Every wave takes steps of 16 keys of its own through a ring of stages in LDS, as chunk_stream_kernel does,
// with QB blocks of 16 rows: S^T = K . Q^T, O^T += V^T . P^T.  The result goes to part `part`.
// WHOLE: behind the keys 0 .. lo - 1 of table row b0 (the front one), which all rows see, and to the results themselves; again: computes a row once more.
template <typename T, int DH, int QB, int WAVES, bool NT, bool WHOLE, typename F, typename R>
__device__ __forceinline__ void stream_rows(const PrefixKernelArgs& a, unsigned char* smem, int b0, int b, int kvh, int t0, int r0, int r1,
                                            KeyRange k, int lo, F hi, int part, R again)
{
    typedef PrefixStream<T, DH, WAVES> S;
    constexpr int RB = S::RB, DS = RB / 64, DT = DH / 16;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), qi = lane & 15, g = lane >> 4, G = a.G;
    const unsigned lds = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem + wave * (S::STAGES * S::STAGE);
    const unsigned char* mine = smem + wave * (S::STAGES * S::STAGE);
    const float mul = exponent_scale(a.scale);
    const int limit = table_limit(a.table);

    const int blocks = (r1 - r0 + 15) / 16;                              // those that are there
    u32x4 qf[QB][DS];
    int last[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int r = r0 + qb * 16 + qi, row = r < r1 ? r : r1 - 1, at = a.by_G.quotient(row), t = t0 + at;
        last[qb] = hi(at);
        load_query<T, DS>((const T*)a.q + (int64_t)(t >= 0 && t < a.tokens ? t : 0) * a.q_stride + (kvh * G + a.by_G.rest(row, at)) * DH, g, a.scale, qf[qb]);
    }
    const int least = hi(a.by_G.quotient(r0));                                            // the first row sees the fewest
    const int shared = WHOLE ? (lo + PX_STEP - 1) / PX_STEP : 0;             // steps in front
    const int steps = shared + (k.last > k.first ? (k.last - k.first + PX_STEP - 1) / PX_STEP : 0), own = steps > wave ? (steps - wave + WAVES - 1) / WAVES : 0;
    typedef RowLoader<T, DH, NT> Loader;
    const Loader from(a.table, a.kv_blocks, b, kvh, a.Hkv, limit, k.last, lane), front(a.table, a.kv_blocks, WHOLE ? b0 : b, kvh, a.Hkv, limit, WHOLE ? lo : k.last, lane);
    auto in_front = [&](int i) { return WHOLE && wave + i * WAVES < shared; };
    auto first_of = [&](int i) { return in_front(i) ? (wave + i * WAVES) * PX_STEP : k.first + (wave + i * WAVES - shared) * PX_STEP; };
    auto lookup = [&](int i) { return in_front(i) ? front.lookup(first_of(i)) : from.lookup(first_of(i)); };
    typename Loader::Entries en{-1, -1};
    auto issue = [&](int i) {
        const unsigned dst = lds + i % S::STAGES * S::STAGE;
        const Loader& f = in_front(i) ? front : from;
        const typename Loader::Rows r = f.rows(first_of(i), en);
        f.keys(first_of(i), r, dst);
        f.values(first_of(i), r, dst + S::TILE);
    };

    float m[QB], l[QB];                                                  // l: this lane's share of the sum
    f32x4 o[QB][DT];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        m[qb] = -INFINITY;
        l[qb] = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[qb][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int ahead = S::STAGES - 1;
    for (int i = 0; i < ahead && i < own; ++i) {
        en = lookup(i);
        issue(i);
    }
    if (ahead < own) en = lookup(ahead);
    for (int i = 0; i < own; ++i) {
        if (i + ahead < own) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // step i - 1 has left its stage
            issue(i + ahead);
            if (i + ahead + 1 < own) en = lookup(i + ahead + 1);
            wait_loads<2 * S::LOADS * (S::STAGES - 1)>();
        } else {
            wait_loads<0>();
        }
        const unsigned char* sK = mine + i % S::STAGES * S::STAGE;
        f32x4 s[QB][2];
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) s[qb][0] = s[qb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ds = 0; ds < DS; ++ds) {
            const u32x4 fk = *(const u32x4*)(sK + qi * RB + (((ds * 4 + g) ^ pf_swz<RB>(qi)) << 4));
#pragma unroll
            for (int qb = 0; qb < QB; ++qb)
                if (qb < blocks) s[qb][ds & 1] = HalfUnit<T>::mma(fk, qf[qb][ds], s[qb][ds & 1]);
        }
        const unsigned char* sV = sK + S::TILE;
        const int v_row = 4 * g + (qi >> 2), v_q = qi & 3;
        uint2 fv[sizeof(T) == 2 ? DT : 1];                               // on their way while the softmax is made
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) fv[dt] = pf_read_tr(sV + v_row * RB + (((2 * dt + (v_q >> 1)) ^ pf_swz<RB>(v_row)) << 4) + (v_q & 1) * 8);
        }
        const int j = first_of(i);
        float mx[QB];
        bool grew = false;
        const bool whole = in_front(i);
        if (whole ? j + PX_STEP > lo : j + PX_STEP > least || j < lo) {
            int key0 = j + 4 * g;
            asm volatile("" : "+v"(key0));                               // keeps the mask arithmetic inside this branch
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                s[qb][0] += s[qb][1];
#pragma unroll
                for (int r = 0; r < 4; ++r) s[qb][0][r] = (whole || key0 + r >= lo) && key0 + r < (whole ? lo : last[qb]) ? s[qb][0][r] : -INFINITY;
            }
        } else {
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) s[qb][0] += s[qb][1];
        }
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            mx[qb] = fmaxf(fmaxf(s[qb][0][0], s[qb][0][1]), fmaxf(s[qb][0][2], s[qb][0][3])) * mul;
            grew |= mx[qb] > m[qb] + 8.f;                                // the maximum follows only where it grew by more than 2^8: sums stay far from a float's ends
        }
        if (__builtin_amdgcn_ballot_w64(grew)) {
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                const float to = fmaxf(m[qb], rows_max(mx[qb])), ref = to == -INFINITY ? 0.f : to, alpha = fast_exp2(m[qb] - ref);
                l[qb] *= alpha;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) o[qb][dt] *= alpha;
                m[qb] = to;
            }
        }
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            if (qb >= blocks) break;
            const float ref = m[qb] == -INFINITY ? 0.f : m[qb];
            f32x4& p = s[qb][0];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                p[r] = fast_exp2(fmaf(p[r], mul, -ref));
                l[qb] += p[r];
            }
            if constexpr (sizeof(T) == 2) {
                typedef __attribute__((ext_vector_type(4))) short v4s;
                bf16x4 high, low;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    high[r] = (bf16_t)p[r];
                    low[r] = (bf16_t)(p[r] - (float)high[r]);
                }
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    o[qb][dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(v4s, fv[dt]), __builtin_bit_cast(v4s, low), o[qb][dt], 0, 0, 0);
                    o[qb][dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(v4s, fv[dt]), __builtin_bit_cast(v4s, high), o[qb][dt], 0, 0, 0);
                }
            }
        }
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                f32x4 c[QB];                                             // a sum per step, so that no chain of additions is as long as the cache
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) c[qb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float v = *(const float*)(sV + (4 * g + r) * RB + (((4 * dt + (qi >> 2)) ^ pf_swz<RB>(4 * g + r)) << 4) + (qi & 3) * 4);
#pragma unroll
                    for (int qb = 0; qb < QB; ++qb) c[qb] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, s[qb][0][r], c[qb], 0, 0, 0);
                }
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) o[qb][dt] += c[qb];
            }
        }
    }

    // the waves' results, joined, 16 rows at a time; lane (qi, g) holds features 16 * dt + 4 * g .. +3 of its row
    float* s_o = (float*)smem;
    float (*s_ml)[16][2] = (float (*)[16][2])(smem + S::MERGE);
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        if (r0 + qb * 16 >= r1) break;
        __syncthreads();                                                 // no wave reads its stages, or the block before, any more
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) *(f32x4*)(s_o + (wave * 16 + qi) * (DH + 4) + dt * 16 + 4 * g) = o[qb][dt];
        const float total = rows_sum(l[qb]);
        if (g == 0) {
            s_ml[wave][qi][0] = m[qb];
            s_ml[wave][qi][1] = total;
        }
        __syncthreads();
        // 16 threads a row, features 4 * c .. +3 of every 64
#pragma unroll
        for (int r = tid >> 4; r < 16; r += WAVES * 4) {                 // beyond 4 waves: nothing to do
            const int c = tid & 15, row = r0 + qb * 16 + r, token = a.by_G.quotient(row), t = t0 + token, h = kvh * G + a.by_G.rest(row, token);
            float M = -INFINITY, L = 0.f, w[WAVES];
#pragma unroll
            for (int i = 0; i < WAVES; ++i) M = fmaxf(M, s_ml[i][r][0]);
            const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) {
                w[i] = fast_exp2(s_ml[i][r][0] - ref);
                L += s_ml[i][r][1] * w[i];
            }
            const bool write = row < r1 && t >= 0 && t < a.tokens;
            if constexpr (WHOLE) {
                f32x4 v[DH / 64];
                float most = 0.f;
                const float inv = 1.f / L;
                const bool any = hi(token) > 0;
#pragma unroll
                for (int f = 0; f < DH / 64; ++f) {
                    v[f] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int i = 0; i < WAVES; ++i) v[f] += *(const f32x4*)(s_o + (i * 16 + r) * (DH + 4) + f * 64 + 4 * c) * w[i];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        v[f][e] = any ? v[f][e] * inv : 0.f;
                        most = magnitude(most, v[f][e]);
                    }
                }
                const unsigned long long bad = __builtin_amdgcn_ballot_w64(write && spoilt(most, L));
                if (write && !(bad >> (lane & 48) & 0xffff)) {
#pragma unroll
                    for (int f = 0; f < DH / 64; ++f) {
                        typename Vec4<T>::type y;
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[e] = from_f32<T>(v[f][e]);
                        *(typename Vec4<T>::type*)((T*)a.out + (int64_t)t * a.out_stride + h * DH + f * 64 + 4 * c) = y;
                    }
                }
                for (int i = 0; i < 4; ++i)                              // the four rows of this wave
                    if (bad >> (16 * i) & 0xffff) again(r0 + qb * 16 + (r & ~3) + i);
                continue;
            }
            if (!write) continue;
            const int64_t at = ((int64_t)part * a.tokens + t) * a.H + h;
#pragma unroll
            for (int f = 0; f < DH / 64; ++f) {
                f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < WAVES; ++i) v += *(const f32x4*)(s_o + (i * 16 + r) * (DH + 4) + f * 64 + 4 * c) * w[i];
                *(f32x4*)(a.tile.acc + at * DH + f * 64 + 4 * c) = v;
            }
            if (c == 0) *(float2*)(a.tile.ml + at * 2) = float2{M, hi(token) > lo ? L : NO_KEYS};
        }
    }
    __syncthreads();                                                     // before the next tile's loads overwrite the results
}
// The same rows where there is no such part.
__device__ __forceinline__ void no_part(const PrefixKernelArgs& a, int kvh, int t0, int r0, int r1, int part)
{
    const int row = r0 + threadIdx.x, at = a.by_G.quotient(row), t = t0 + at;
    if (row < r1 && t >= 0 && t < a.tokens)
        *(float2*)(a.tile.ml + (((int64_t)part * a.tokens + t) * a.H + kvh * a.G + a.by_G.rest(row, at)) * 2) = float2{-INFINITY, NO_PART};
}

// Tile of the prefix for workgroup wg: of tiles with 2^SHIFT rows, those that read the same keys follow each other on one XCD.  b = -1: there is
// none.  What the prefix has no keys for is marked here.
struct PrefixTile { ChunkTile tile; int r1, part; KeyRange k; };
template <int SHIFT> __device__ __forceinline__ PrefixTile find_prefix(const PrefixKernelArgs& a, unsigned wg, int limit, int lane)
{
    PrefixTile r;
    r.tile.b = -1;
    const int slot = a.by_units.quotient(wg), u = a.by_units.rest(wg, slot);
    if (u >= a.Hkv * a.shared.parts) return r;
    r.part = a.by_Hkv.quotient(u);
    const int kvh = a.by_Hkv.rest(u, r.part);
    const PrefixGroup gr = find_group<true>(a, slot, SHIFT, lane);
    if (gr.g < 0) return r;
    const int n = gr.t1 - gr.t0 < a.tokens ? gr.t1 - gr.t0 : a.tokens, rows = n * a.G;
    const int r0 = (slot - ((int)((int64_t)gr.t0 * a.G >> SHIFT) + gr.g)) << SHIFT;
    if (n <= 0 || r0 >= rows) return r;
    r.r1 = r0 + (1 << SHIFT) < rows ? r0 + (1 << SHIFT) : rows;
    const int end = gr.prefix < limit ? gr.prefix : limit;
    const KeyRange all{0, end};
    const int parts = end > 0 ? parts_of(all, a.shared) : 0;
    if (r.part >= parts) {
        no_part(a, kvh, gr.t0, r0, r.r1, r.part);
        return r;
    }
    r.tile = ChunkTile{gr.front, kvh, gr.t0, r.r1, 0, r0};
    r.k = part_of(all, a.shared, r.part, parts);
    return r;
}
// A sequence's own positions, by workgroup wg of those.
template <typename T, int DH, int WAVES> __device__ __forceinline__ void own_rows(const PrefixKernelArgs& a, unsigned char* smem, unsigned wg, int limit, int lane)
{
    const int G = a.G, u = a.by_parts.quotient(wg), part = a.by_parts.rest(wg, u), head = a.by_tiles.quotient(u), tile = a.by_tiles.rest(u, head), b = a.by_Hkv.quotient(head),
              kvh = a.by_Hkv.rest(head, b);
    const int t0 = a.cu[b], end = a.cu[b + 1], p_end = a.len[b], n = end - t0 < a.tokens ? end - t0 : a.tokens, p0 = p_end - n;
    const PrefixGroup gr = find_group<false>(a, b, 0, lane);
    if (n <= 0) return;
    const int lo = gr.prefix < limit ? gr.prefix : limit;
    auto hi = [&](int token) { return keys_of(p0 + token, 0, limit).last; };
    for (int r0 = tile * 16; r0 < n * G; r0 += a.own_tiles * 16) {
        const int r1 = r0 + 16 < n * G ? r0 + 16 : n * G;
        const KeyRange all{lo & -PX_STEP, hi(a.by_G.quotient(r1 - 1))};
        const int parts = parts_of(all, a.own);
        if (part >= parts) no_part(a, kvh, t0, r0, r1, a.shared.parts + part);
        else stream_rows<T, DH, 1, WAVES, true, false>(a, smem, b, b, kvh, t0, r0, r1, part_of(all, a.own, part, parts), lo, hi, a.shared.parts + part, [](int) {});
    }
}

// Up to 32 rows of a group and key/value head (float: in tiles of 32), and own positions.  Bound by reading the cache where contexts are long: 8 sequences of 40
// heads x 128, 1500 shared positions and 170 own ones 17 us, of which 6 go by before the first keys are there (the rest at 6 TB/s), and 4 for the join.
template <typename T, int DH, int QB, int WAVES> __global__ __launch_bounds__(WAVES * 64, 2) void prefix_stream_kernel(PrefixKernelArgs a)
{
    extern __shared__ __align__(16) unsigned char px_smem[];
    const int lane = threadIdx.x & 63, limit = table_limit(a.table);
    if (blockIdx.x >= a.shared_units) return own_rows<T, DH, WAVES>(a, px_smem, blockIdx.x - a.shared_units, limit, lane);
    const PrefixTile p = find_prefix<QB == 1 ? 4 : 5>(a, blockIdx.x, limit, lane);
    if (p.tile.b < 0) return;
    const int end = p.k.last;
    stream_rows<T, DH, QB, WAVES, false, false>(a, px_smem, p.tile.b, p.tile.b, p.tile.kvh, p.tile.t0, p.tile.r0, p.r1, p.k, 0, [&](int) { return end; }, p.part, [](int) {});
}
// Few and short sequences, each with its prefix by itself: the prefix, that comes from L2 for all but the first, costs less than a second launch (2 sequences of 12
// heads x 64 over 200 + 40 positions 6.6 us, of which two launches take 9).
template <typename T, int DH, int WAVES> __global__ __launch_bounds__(WAVES * 64, 2) void prefix_whole_kernel(PrefixKernelArgs a)
{
    extern __shared__ __align__(16) unsigned char px_smem[];
    const int lane = threadIdx.x & 63, limit = table_limit(a.table), G = a.G, head = a.by_tiles.quotient(blockIdx.x), tile = a.by_tiles.rest(blockIdx.x, head), b = a.by_Hkv.quotient(head),
              kvh = a.by_Hkv.rest(head, b);
    const int t0 = a.cu[b], end = a.cu[b + 1], p_end = a.len[b], n = end - t0 < a.tokens ? end - t0 : a.tokens, p0 = p_end - n;
    const PrefixGroup gr = find_group<false>(a, b, 0, lane);
    if (n <= 0) return;
    const int lo = gr.prefix < limit ? gr.prefix : limit;
    auto hi = [&](int token) { return keys_of(p0 + token, 0, limit).last; };
    auto again = [&](int row) { prefix_row<T, DH>(a, gr, b, p0 + row / G, t0 + row / G, kvh * G + row % G, lane); };
    for (int r0 = tile * 16; r0 < n * G; r0 += a.own_tiles * 16) {
        const int r1 = r0 + 16 < n * G ? r0 + 16 : n * G;
        stream_rows<T, DH, 1, WAVES, false, true>(a, px_smem, gr.g < 0 || !lo ? b : gr.front, b, kvh, t0, r0, r1, KeyRange{lo & -PX_STEP, hi(a.by_G.quotient(r1 - 1))}, lo, hi, 0, again);
    }
}
// More rows, in tiles of 128, in front of own positions.  Bound by MFMAs and softmax, as chunk_tile_kernel is, with half as many products again for the probabilities'
// lower bits: 64 sequences and 96 tokens of 32 heads over 8 x 128 on a document of 30001 positions 91 us, of which the own positions' 81 MB, behind the tiles, take 18
// (among them, whose places on a CU they take, 15 to 45 more; in front of them as long), and 6.4 for the join; 60002 more positions 165 us, 860 TFLOP/s.  12 groups of 1 to 16
// sequences 45 us, 4.4 TB/s, 5.1 behind the start.
template <typename T, int DH> __global__ __launch_bounds__(CT_WAVES * 64, 2) void prefix_tile_kernel(PrefixKernelArgs a)
{
    extern __shared__ __align__(16) unsigned char px_smem[];
    const int lane = threadIdx.x & 63, limit = table_limit(a.table);
    if (blockIdx.x >= a.shared_units) return own_rows<T, DH, CT_WAVES>(a, px_smem, blockIdx.x - a.shared_units, limit, lane);
    const PrefixTile p = find_prefix<7>(a, blockIdx.x, limit, lane);
    if (p.tile.b < 0) return;
    tile_rows<T, DH, 2, true>(a, px_smem, p.tile, p.k, p.part, 2, [](int, int, KeyRange) {});
}

// The sum over a row's parts of 2^(m_i - M) times their sums, in their order: a wave per row, DH / 4 lanes a part, 2 or 4 parts at a time.
template <typename T, int DH> __global__ __launch_bounds__(256) void prefix_join_kernel(PrefixKernelArgs a)
{
    constexpr int PER = DH / 4, SUBS = 64 / PER;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = a.by_quarter.quotient(blockIdx.x), h = a.by_quarter.rest(blockIdx.x, t) * 4 + wave;
    if (h >= a.H) return;
    const int parts = a.shared.parts + a.own.parts, sub = lane / PER, f = lane % PER * 4;
    const int64_t at = (int64_t)t * a.H + h, step = (int64_t)a.tokens * a.H;
    const int packed = a.cu[a.n_seqs];
    const float2 x = lane < parts ? *(const float2*)(a.tile.ml + (at + lane * step) * 2) : float2{-INFINITY, NO_PART};
    const float* acc = a.tile.acc + at * DH + f;
    auto part = [&](int k) { return *(const f32x4*)(acc + (k < parts ? k : parts - 1) * step * DH); };
    const f32x4 early[2] = {part(sub), part(SUBS + sub)};                // need no weights (12 groups 43.1 -> 42.6 us)
    asm volatile("" ::: "memory");                                       // not after the wait for those
    if (t >= packed) return;
    const float M = wave_max(x.x), w = x.y == NO_PART ? -1.f : fast_exp2(x.x - (M == -INFINITY ? 0.f : M)), L = wave_sum(x.y < 0.f ? 0.f : x.y * w);
    const bool none = __builtin_amdgcn_ballot_w64(x.y == NO_KEYS);
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    int first = 0;
    auto add = [&](const f32x4* p, auto count) {
#pragma unroll
        for (int u = 0; u < count; ++u) {
            const int k = first + u * SUBS + sub;
            const float wk = __shfl(w, k < parts ? k : parts - 1, WAVE);
            if (k < parts && wk >= 0.f) v += p[u] * wk;
        }
        first += count * SUBS;
    };
    auto take = [&](auto count) {                                        // parts of which the loads are on their way together
        f32x4 p[count];
#pragma unroll
        for (int u = 0; u < count; ++u) p[u] = part(first + u * SUBS + sub);
        add(p, count);
    };
    add(early, std::integral_constant<int, 2>{});
    // us of a call, one after the other / 8 of them: 8 sequences of 32 heads over 4 and 3746 shared positions, 64 parts 19.0 / 15.5, 17 of 24 over 3 and 11011 27.5 /
    // 19.0; up to 4 each: more loads than parts (12 groups 42.9 / 43.5).
    while (parts - first > 4 * SUBS) take(std::integral_constant<int, 8>{});
    while (first < parts) take(std::integral_constant<int, 2>{});
#pragma unroll
    for (int d = PER; d < 64; d <<= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += __shfl_xor(v[e], d, WAVE);
    float most = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[e] = none ? 0.f : v[e] / L;
        most = magnitude(most, v[e]);
    }
    T* out = (T*)a.out + (int64_t)t * a.out_stride + h * DH;
    if (!none && __builtin_amdgcn_ballot_w64(spoilt(most, L))) {
        const ChunkSeq sq = seq_of_token(a.cu, a.n_seqs, t, lane);
        if (sq.b < 0) return;
        const PrefixGroup gr = find_group<false>(a, sq.b, 0, lane);
        prefix_row<T, DH>(a, gr, sq.b, a.len[sq.b] - sq.n + (t - sq.t0), t, h, lane);
    } else if (sub == 0) {
        typename Vec4<T>::type y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = from_f32<T>(v[e]);
        *(typename Vec4<T>::type*)(out + f) = y;
    }
}

// ---------------------------------------------------------------- launches
struct PrefixPlan {
    bool whole;
    int qb, waves;                                        // blocks of 16 rows of a prefix tile; waves of a streaming workgroup
    PrefixKernelArgs::Cut shared, own;
    int own_tiles;
    int64_t slots, shared_units, own_units;
};
static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
static PrefixKernelArgs::Cut cut_keys(int64_t keys, int64_t target, int most)
{
    int64_t parts = ceil_div(keys, target);
    parts = parts < 1 ? 1 : parts < most ? parts : most;
    if (parts == 1) return {1, 0x7fffffff};
    const int64_t each = ceil_div(ceil_div(keys, parts), PX_STEP) * PX_STEP;
    return {(int)ceil_div(keys, each), (int)each};
}
static PrefixPlan prefix_plan(const PrefixAttnArgs& a)
{
    PrefixPlan p{};
    const int64_t G = a.H / a.Hkv, rows = (int64_t)a.max_group * G;
    // Tiles of 128 rows beyond 32 (us, streaming in blocks of 32 rows / tiles: 12 groups of 1 to 16 sequences, 32 heads over 8 x 128, 400 to 3000 shared positions
    // 51 / 48; over 30000 positions 96 sequences of 32 heads 234 / 132, 24 of 32 over 8 62 / 48, 10 of 32 over 8 38.6 / 38.3; 32 rows 35.0 / 35.6 and 105 / 104).
    p.qb = a.n_groups == 0 || rows <= 16 ? 1 : rows <= 32 || a.dtype == DT_F32 ? 2 : 8;
    p.slots = (int64_t)a.tokens * G / (16 * p.qb) + a.n_groups + 1;
    const int64_t most = (int64_t)a.tokens * G / (16 * p.qb) + a.n_groups, each = a.n_groups * ceil_div(rows, 16 * p.qb), tiles = (each < most ? each : most) * a.Hkv;
    const int64_t own = (int64_t)a.n_seqs * a.Hkv, own_rows = ceil_div(a.max_new * G, 16);
    // us of both launches / one: 2 sequences of 12 heads x 64 over 200 + 60 keys 9.0 / 6.9, 450 + 60 9.1 / 8.7, 800 + 60 9.4 / 10.6; 4 of 40 heads x 128, 300 + 60
    // 10.7 / 9.0; 4 of 32 over 8, 400 + 60 10.0 / 10.0; more than one workgroup a CU: 12 of 40, 300 + 60 15.0 / 16.9; float, 400 + 60 10.4 / 12.0; and a launch's
    // 4 us of the host.
    p.whole = own * own_rows <= 256 && (int64_t)a.max_prefix + a.max_own <= (a.dtype == DT_F32 ? 256 : 512);
    if (p.whole) {
        p.waves = a.dtype == DT_F32 && a.dh == 128 ? 4 : 8;
        p.own_tiles = (int)own_rows;
        p.own_units = own * own_rows;
        return p;
    }
    // Keys for a workgroup so that the chip, two of 4 waves a CU (float x 128: one), is filled once; parts of less than 128 gain nothing.
    const int64_t keys = tiles * a.max_prefix + own * own_rows * a.max_own, wgs = a.dtype == DT_F32 && a.dh == 128 ? 256 : 512;
    int64_t target = ceil_div(keys, wgs);
    // Workgroups of 2 waves, five a CU, where one round of 4 waves would have to hold parts of very different lengths (us of 4 / 2: 8 sequences of 40 heads, 1500 shared
    // positions and 40 to 300 own ones 21.8 / 17.3; 20 groups of 2, 4 heads 24.3 / 18.8; 8 of 16 heads, 6000 shared 17.3 / 15.7); not for shorter ones,
    // where both waves start late, or longer ones, whose rounds even out (6 groups of 8 of 40 heads 75 / 87).
    p.waves = p.qb == 1 && target >= 128 && target < 384 && wgs == 512 ? 2 : 4;
    if (p.waves == 2) target = ceil_div(keys, 768);
    target = target < 128 ? 128 : target;
    // Parts are whole: where what they are rounded up by would begin a second round, longer ones, up to twice, if those fit one (us: 32 sequences of 32 heads over
    // 8 x 128 and 6000 shared positions 29.4 -> 22.4, 16 of 32 over 4 x 64 and 8000 21.4 -> 17.8, 24 of 16 heads and 4000 23.1 -> 21.4; of 47 shapes 25 by 3 to
    // 20 % faster, two slower, by 2 and 5 %).  Up to three times as long: between 20 % faster and 65 % slower (47 of 24 heads over 8 x 64 and 15556 27.6, 45.7).  Where own positions alone are more than a
    // round, fewer or more parts were not better (the document 83; 79 to 98 by a target of 448 to 1024 workgroups, the ragged groups 45; 45 to 50).
    auto count = [&](int64_t t) { return tiles * ceil_div(a.max_prefix, t) + own * own_rows * ceil_div(a.max_own, t); };
    if (p.waves == 4)
        for (int i = 16; i <= 32; ++i)
            if (count(target * i / 16) <= wgs) {
                target = target * i / 16;
                break;
            }
    p.own = cut_keys(a.max_own, target, 16);
    p.shared = a.n_groups ? cut_keys(a.max_prefix, target, PX_PARTS - p.own.parts) : PrefixKernelArgs::Cut{0, 0x7fffffff};
    p.shared_units = ceil_div(a.Hkv * p.shared.parts, 8) * 8 * p.slots;
    p.own_tiles = (int)std::max<int64_t>(1, std::min(own_rows, (1 << 20) / (own * p.own.parts)));      // a workgroup goes on with what is left
    p.own_units = own * p.own_tiles * p.own.parts;
    return p;
}
size_t prefix_attn_workspace(const PrefixAttnArgs& a)
{
    const PrefixPlan p = prefix_plan(a);
    if (p.whole) return 0;
    return (size_t)(p.shared.parts + p.own.parts) * a.tokens * a.H * (a.dh + 2) * sizeof(float);
}

template <typename K> static hipError_t launch_kernel(K kernel, LdsLimit (&limit)[MAX_DEVICES], int waves, int lds, const PrefixKernelArgs& k, int64_t wgs, hipStream_t s)
{
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= MAX_DEVICES) dev = 0;
    hipError_t e = limit[dev].raise((const void*)kernel, lds);
    if (e != hipSuccess) return e;
    kernel<<<(unsigned)wgs, waves * 64, lds, s>>>(k);
    return hipGetLastError();
}
template <typename T, int DH, int QB, int WAVES> static hipError_t launch_stream(const PrefixKernelArgs& k, int64_t wgs, hipStream_t s)
{
    static LdsLimit limit[MAX_DEVICES];
    typedef PrefixStream<T, DH, WAVES> S;
    return launch_kernel(prefix_stream_kernel<T, DH, QB, WAVES>, limit, WAVES, S::LDS, k, wgs, s);
}
template <typename T, int DH, int WAVES> static hipError_t launch_whole(const PrefixKernelArgs& k, int64_t wgs, hipStream_t s)
{
    static LdsLimit limit[MAX_DEVICES];
    return launch_kernel(prefix_whole_kernel<T, DH, WAVES>, limit, WAVES, PrefixStream<T, DH, WAVES>::LDS, k, wgs, s);
}
template <typename T, int DH> static hipError_t launch_tile(const PrefixKernelArgs& k, int64_t wgs, hipStream_t s)
{
    static LdsLimit limit[MAX_DEVICES];
    return launch_kernel(prefix_tile_kernel<T, DH>, limit, CT_WAVES, std::max(PrefixStream<T, DH, CT_WAVES>::LDS, ct_lds<T, DH, 2>()), k, wgs, s);
}
template <typename T, int DH> static hipError_t launch_prefix(const PrefixAttnArgs& a, hipStream_t s)
{
    const PrefixPlan p = prefix_plan(a);
    const int64_t wgs = p.shared_units + p.own_units, rows = (int64_t)a.tokens * a.H;
    if (p.slots > 0x7fffffff || wgs * 512 > MAX_LAUNCH_THREADS || rows / 4 + a.tokens > MAX_LAUNCH_THREADS / 256) return hipErrorInvalidValue;
    PrefixKernelArgs k{};
    k.cu = a.cu; k.len = a.len; k.cu_groups = a.cu_groups; k.prefix = a.prefix;
    k.n_seqs = a.n_seqs; k.tokens = a.tokens; k.n_groups = a.n_groups;
    k.q = a.q; k.q_stride = a.q_stride;
    k.kv_blocks = a.kv_blocks;
    k.table = a.table;
    k.H = a.H; k.Hkv = a.Hkv; k.G = a.H / a.Hkv;
    k.scale = a.scale;
    k.out = a.out; k.out_stride = a.out_stride;
    k.shared = p.shared; k.own = p.own;
    k.tile = {rows, a.workspace, a.workspace + (size_t)(p.shared.parts + p.own.parts) * rows * DH};
    k.own_tiles = p.own_tiles;
    k.shared_units = (unsigned)p.shared_units;
    k.by_G = Divisor::of(k.G); k.by_Hkv = Divisor::of(k.Hkv);
    k.by_parts = Divisor::of(std::max(p.own.parts, 1)); k.by_tiles = Divisor::of(p.own_tiles);
    k.by_units = Divisor::of(std::max<int64_t>(8, ceil_div((int64_t)k.Hkv * p.shared.parts, 8) * 8)); k.by_quarter = Divisor::of(ceil_div(a.H, 4));
    hipError_t e;
    if (p.whole) {
        if constexpr (sizeof(T) == 4 && DH == 128) return launch_whole<T, DH, 4>(k, wgs, s);
        else return launch_whole<T, DH, 8>(k, wgs, s);
    }
    if (p.qb == 1) e = p.waves == 2 ? launch_stream<T, DH, 1, 2>(k, wgs, s) : launch_stream<T, DH, 1, 4>(k, wgs, s);
    else if (p.qb == 2) e = launch_stream<T, DH, 2, 4>(k, wgs, s);
    else if constexpr (sizeof(T) == 2) e = launch_tile<T, DH>(k, wgs, s);
    else e = hipErrorInvalidValue;
    if (e != hipSuccess) return e;
    prefix_join_kernel<T, DH><<<(unsigned)(a.tokens * ceil_div(a.H, 4)), 256, 0, s>>>(k);
    return hipGetLastError();
}
hipError_t launch_prefix_attn(const PrefixAttnArgs& a, hipStream_t s)
{
    if (a.dtype == DT_F32) return a.dh == 64 ? launch_prefix<float, 64>(a, s) : launch_prefix<float, 128>(a, s);
    return a.dh == 64 ? launch_prefix<bf16_t, 64>(a, s) : launch_prefix<bf16_t, 128>(a, s);
}

}  // namespace exe
