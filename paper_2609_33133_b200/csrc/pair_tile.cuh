// What the products of CTA pairs share (256 x 256 output tiles, tcgen05 cta_group::2): the tile, the way results leave.
#pragma once
#include "ptx.cuh"

namespace augtree {

constexpr int kLmTile = 256;     // tile rows and columns of a CTA pair

// A row's columns into the warp's 4 KB block, in the 128-byte swizzle (16-byte chunk j of row r sits at j ^ (r % 8)): 32 columns
// of 16 bits as the chunks from `chunk`, or 32 columns of 32 bits.
__device__ __forceinline__ void stage_bf16(uint32_t s_out, int row, int chunk, const float (&x)[32]) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    st_shared_v4(s_out + row * 128 + (((chunk + e) ^ (row & 7)) << 4), pack_bf16(x[8 * e], x[8 * e + 1]), pack_bf16(x[8 * e + 2], x[8 * e + 3]),
                 pack_bf16(x[8 * e + 4], x[8 * e + 5]), pack_bf16(x[8 * e + 6], x[8 * e + 7]));
}
__device__ __forceinline__ void stage_f32(uint32_t s_out, int row, const float (&x)[32]) {
#pragma unroll
  for (int e = 0; e < 8; ++e)
    st_shared_v4(s_out + row * 128 + ((e ^ (row & 7)) << 4), __float_as_uint(x[4 * e]), __float_as_uint(x[4 * e + 1]),
                 __float_as_uint(x[4 * e + 2]), __float_as_uint(x[4 * e + 3]));
}

}  // namespace augtree
