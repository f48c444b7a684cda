// Key and value tiles in LDS, as the MFMA attention kernels (kernels_attn.hip, kernels_chunk.hip) read them.
#pragma once
#include "common.h"

namespace exe {

// A key or value tile [64 rows] in LDS, row-major in 16-byte chunks.  Rows of 256 bytes and more keep chunk c of row r at
// slot c ^ (r & 15), rows of 128 bytes at slot c ^ ((r >> 1) & 7): the fragment reads below touch every bank group
// equally.  Rows 16 apart share their swizzle.
template <int RB> __device__ __forceinline__ int pf_swz(int row) { return RB >= 256 ? row & 15 : (row >> 1) & 7; }

typedef __attribute__((ext_vector_type(4))) short pf_v4s;
// Transposing LDS read (ds_read_b64_tr_b16).  Within each block of 16 lanes, lane L points at 4 consecutive 16-bit
// elements M[L][0..3]; lane i receives M[4*j + i/4][i%4], j = 0..3.  With lane L = 4*j + q pointing at columns
// d0 + 4*q .. +3 of row j, lane i ends up with column d0 + i of rows 0..3: four values along the row index for one
// column, which is how an MFMA operand wants a row-major tile whose rows are the contraction index.
__device__ __forceinline__ uint2 pf_read_tr(const unsigned char* p)
{
    pf_v4s r = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) pf_v4s*)p);
    return __builtin_bit_cast(uint2, r);
}

}  // namespace exe
