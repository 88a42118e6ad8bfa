// Activation checkpoints in 8 bits: the format, and 8 values at a time between it, the floating-point types and registers.
//
// A row of `cols` values is kept as ceil16(cols) bytes of integers and ceil16(ceil(cols / 32)) bytes of exponents (what lies behind
// the last column or group is not defined).  32 neighbouring columns share 2^e, kept as the byte e + 127: the smallest power of two with max |x| < 127.5 2^e,
// e >= -126; each value is x / 2^e rounded to the nearest integer (ties to even), which is then within -127 .. 127, and off by at most
// half of 2^e, 1 / 127.5 of the group's largest value.  A group that holds a NaN or an infinity gets the byte 255 and reads as NaN.
// Why so: with a power of two both directions are exact but for the one rounding, so the form of a tensor does not depend on which
// kernel made it, and what it stands for fits bf16 exactly (8 significant bits), which the tensor core takes as an operand without
// a second rounding.  For normal values 32 of which share an exponent the error is 0.0075 of their deviation (rms); 8-bit floating
// point with 3 bits of mantissa leaves 0.026 of each value.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ptx.cuh"

namespace augtree {

enum : int { T_BF16 = 0, T_F16 = 1, T_F32 = 2, T_CKPT = 3 };   // as AUGTREE_BF16 ..

__host__ __device__ inline long long ckpt_scale_offset(long long cols) { return (cols + 15) / 16 * 16; }
__host__ __device__ inline long long ckpt_pitch(long long cols) { return ckpt_scale_offset(cols) + ((cols + 31) / 32 + 15) / 16 * 16; }

// ---------------------------------------------------------------- 8 values to and from memory
template <typename T> struct Row8;
template <> struct Row8<__nv_bfloat16> {
  static __device__ __forceinline__ void unpack(uint4 w, float (&x)[8]) {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(v[i] << 16); x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u); }
  }
  static __device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
  }
  static __device__ __forceinline__ void load(const __nv_bfloat16 *p, float (&x)[8]) { unpack(*reinterpret_cast<const uint4 *>(p), x); }
  static __device__ __forceinline__ void store(__nv_bfloat16 *p, const float (&x)[8]) { *reinterpret_cast<uint4 *>(p) = pack(x); }
  static __device__ __forceinline__ float round(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }
};
template <> struct Row8<__half> {
  static __device__ __forceinline__ void load(const __half *p, float (&x)[8]) {
    const uint4 w = *reinterpret_cast<const uint4 *>(p);
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&v[i]));
      x[2 * i] = f.x; x[2 * i + 1] = f.y;
    }
  }
  static __device__ __forceinline__ void store(__half *p, const float (&x)[8]) {
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]); v[i] = *reinterpret_cast<const uint32_t *>(&h); }
    *reinterpret_cast<uint4 *>(p) = make_uint4(v[0], v[1], v[2], v[3]);
  }
  static __device__ __forceinline__ float round(float x) { return __half2float(__float2half_rn(x)); }
};
template <> struct Row8<float> {
  static __device__ __forceinline__ void load(const float *p, float (&x)[8]) {
    const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
  // (base pointers are aligned to 16 bytes, not to the 32 of one wide store)
  static __device__ __forceinline__ void store(float *p, const float (&x)[8]) {
    if ((reinterpret_cast<uintptr_t>(p) & 31) == 0) {
      uint32_t w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(x[i]);
      st_global_v8(p, w);
    } else {
      reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
      reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    }
  }
  static __device__ __forceinline__ float round(float x) { return x; }
};

// ---------------------------------------------------------------- the 8-bit form
// 8 columns of a thread; the four threads of a lane quad hold a group of 32.  Every lane of the warp takes part; columns behind the
// row's end are zero.
__device__ __forceinline__ void ckpt_encode(const float (&x)[8], uint2 &q, uint32_t &byte) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);   // magnitudes order like their bits, NaN on top
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
  const bool finite = m < 0x7f800000u;
  // m = f 2^k, 1 <= f < 2: e = k - 6, one more from f = 127.5 / 64 on, where the added bits carry into the exponent
  const int biased = (int)((m + 0x10000u) >> 23);
  byte = finite ? (uint32_t)max(biased - 6, 1) : 255u;
  const float per = finite ? __uint_as_float((254u - byte) << 23) : 0.f;          // 2^-e
  uint32_t b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) b[i] = __float_as_uint(fmaf(x[i], per, 12582912.f));  // + 1.5 2^23: the integer in the low bits
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t lo = __byte_perm(b[4 * h], b[4 * h + 1], 0x0040), hi = __byte_perm(b[4 * h + 2], b[4 * h + 3], 0x0040);
    (h ? q.y : q.x) = __byte_perm(lo, hi, 0x5410);
  }
}
__device__ __forceinline__ float ckpt_unit(uint32_t byte) {   // 2^e
  return byte == 255u ? __uint_as_float(0x7fffffffu) : __uint_as_float(byte << 23);
}
__device__ __forceinline__ void ckpt_decode(uint2 q, float unit, float (&x)[8]) {
  // the byte q + 128 in the low bits of 2^23 is 2^23 + 128 + q; both steps are exact
  const uint32_t w[2] = {q.x ^ 0x80808080u, q.y ^ 0x80808080u};
#pragma unroll
  for (int i = 0; i < 8; ++i)
    x[i] = (__uint_as_float(__byte_perm(w[i >> 2], 0x4b000000u, 0x7650 | (i & 3))) - 8388736.f) * unit;
}

}  // namespace augtree
