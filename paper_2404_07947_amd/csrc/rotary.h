// Rotary positions: the angles, and what the kernels that turn heads share (kernels_cache.hip, kernels_heads.hip).
#pragma once
#include "common.h"

namespace exe {

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

// Parts of a token: 16384 waves, two for each that the chip holds, where tokens are few; up to one per 64 slots.
static int rotary_parts(int tokens, int64_t slots)
{
    int64_t most = (slots + 63) / 64, want = (16384 + tokens - 1) / tokens;
    return (int)(most < want ? most : want);
}
static bool aligned_rows(const void* p, int64_t stride, int esz) { return !p || (((uintptr_t)p & 15) == 0 && stride * esz % 16 == 0); }

// Chunks of 16 bytes where rows and (half layout) both halves of the turned part begin on 16 bytes, else single elements.
template <typename T> static bool rotary_wide(int rot, int interleaved) { return interleaved || rot % (32 / (int)sizeof(T)) == 0; }

}  // namespace exe
