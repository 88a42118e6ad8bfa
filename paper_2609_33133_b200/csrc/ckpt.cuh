// Activation checkpoints in 8 bits: the format, and 8 values at a time between it, the floating-point types and registers.
//
// A row of `cols` values is kept as ceil16(cols) bytes of integers and ceil16(ceil(cols / 32)) bytes of exponents (what lies behind
// the last column or group is not defined).  32 neighbouring columns share 2^e, kept as the byte e + 127: the smallest power of two with max |x| < 127.5 2^e,
// but -126 <= e <= 121; each value is x / 2^e rounded to the nearest integer (ties to even) within -127 .. 127, and off by at most
// half of 2^e, 1 / 127.5 of the group's largest value.  (With e = 122 the largest integer, 64, would stand for 2^128.  So magnitudes from 127.5 2^121 = 1.992 2^127 on, the
// last 0.4 % of the range, read as 127 2^121 and are off by less than 2^121.)  A group that holds a NaN or an infinity gets the byte 255 and reads as NaN.
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

// ---------------------------------------------------------------- 8 values in registers
// In pairs, for the packed fp32 instructions of sm_100 (one issue slot for two values: these kernels are as near to the issue rate as
// to the memory's).
struct V8 {
  float2 p[4];
  __device__ __forceinline__ float &operator[](int i) { return (i & 1) ? p[i >> 1].y : p[i >> 1].x; }
  __device__ __forceinline__ float operator[](int i) const { return (i & 1) ? p[i >> 1].y : p[i >> 1].x; }
};
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ V8 v8(float x) { return {{both(x), both(x), both(x), both(x)}}; }
__device__ __forceinline__ V8 operator*(const V8 &a, const V8 &b) {
  return {{__fmul2_rn(a.p[0], b.p[0]), __fmul2_rn(a.p[1], b.p[1]), __fmul2_rn(a.p[2], b.p[2]), __fmul2_rn(a.p[3], b.p[3])}};
}
__device__ __forceinline__ V8 operator*(const V8 &a, float s) { return a * v8(s); }
__device__ __forceinline__ V8 operator+(const V8 &a, const V8 &b) {
  return {{__fadd2_rn(a.p[0], b.p[0]), __fadd2_rn(a.p[1], b.p[1]), __fadd2_rn(a.p[2], b.p[2]), __fadd2_rn(a.p[3], b.p[3])}};
}
__device__ __forceinline__ V8 fma(const V8 &a, const V8 &b, const V8 &c) {
  return {{__ffma2_rn(a.p[0], b.p[0], c.p[0]), __ffma2_rn(a.p[1], b.p[1], c.p[1]), __ffma2_rn(a.p[2], b.p[2], c.p[2]), __ffma2_rn(a.p[3], b.p[3], c.p[3])}};
}
__device__ __forceinline__ V8 fma(const V8 &a, float s, const V8 &c) { return fma(a, v8(s), c); }
__device__ __forceinline__ float2 dot2(const V8 &a, const V8 &b, float2 s) {
#pragma unroll
  for (int i = 0; i < 4; ++i) s = __ffma2_rn(a.p[i], b.p[i], s);
  return s;
}

// ---------------------------------------------------------------- to and from memory
template <typename T> struct Row8;
template <> struct Row8<__nv_bfloat16> {
  static __device__ __forceinline__ V8 load(const __nv_bfloat16 *p) {
    const uint4 w = *reinterpret_cast<const uint4 *>(p);
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
    V8 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.p[i] = make_float2(__uint_as_float(v[i] << 16), __uint_as_float(v[i] & 0xffff0000u));
    return x;
  }
  static __device__ __forceinline__ void store(__nv_bfloat16 *p, const V8 &x) {
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(x.p[0].x, x.p[0].y), pack_bf16(x.p[1].x, x.p[1].y), pack_bf16(x.p[2].x, x.p[2].y),
                                               pack_bf16(x.p[3].x, x.p[3].y));
  }
  static __device__ __forceinline__ float2 round(float2 x) {
    const uint32_t w = pack_bf16(x.x, x.y);
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
  }
};
template <> struct Row8<__half> {
  static __device__ __forceinline__ V8 load(const __half *p) {
    const uint4 w = *reinterpret_cast<const uint4 *>(p);
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
    V8 x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.p[i] = __half22float2(*reinterpret_cast<const __half2 *>(&v[i]));
    return x;
  }
  static __device__ __forceinline__ void store(__half *p, const V8 &x) {
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { const __half2 h = __floats2half2_rn(x.p[i].x, x.p[i].y); v[i] = *reinterpret_cast<const uint32_t *>(&h); }
    *reinterpret_cast<uint4 *>(p) = make_uint4(v[0], v[1], v[2], v[3]);
  }
  static __device__ __forceinline__ float2 round(float2 x) { return __half22float2(__floats2half2_rn(x.x, x.y)); }
};
template <> struct Row8<float> {
  static __device__ __forceinline__ V8 load(const float *p) {
    const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
    return {{make_float2(a.x, a.y), make_float2(a.z, a.w), make_float2(b.x, b.y), make_float2(b.z, b.w)}};
  }
  // (base pointers are aligned to 16 bytes, not to the 32 of one wide store)
  static __device__ __forceinline__ void store(float *p, const V8 &x) {
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
  static __device__ __forceinline__ float2 round(float2 x) { return x; }
};

// ---------------------------------------------------------------- the 8-bit form
// max(a, |b|, |c|), NaN if one of them is
__device__ __forceinline__ float max_magnitude(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(fabsf(b)), "f"(fabsf(c)));
  return d;
}
// The exponent byte of a group whose largest magnitude is `top` (magnitudes order like their bits, infinity and NaN on top).  It grows with
// `top`, so the byte of a group is also the largest of its parts' bytes.  One more than kCkptTop if the group's largest values have to be cut (ckpt_cut).
__device__ __forceinline__ uint32_t ckpt_byte(float top) {
  const uint32_t m = __float_as_uint(top);
  // m = f 2^k, 1 <= f < 2: e = k - 6, one more from f = 127.5 / 64 on, where the added bits carry into the exponent
  return m < 0x7f800000u ? (uint32_t)max((int)((m + 0x10000u) >> 23) - 6, 1) : 255u;
}
__device__ __forceinline__ float ckpt_per(uint32_t byte) { return byte == 255u ? 0.f : __uint_as_float((254u - byte) << 23); }   // 2^-e
constexpr uint32_t kCkptTop = 121 + 127;     // the byte of the largest power of two
// Values of a group whose byte is above that: finite ones (the byte says 2^122) are cut to 127 2^121.
__device__ __forceinline__ void ckpt_cut(V8 &x, uint32_t &byte) {
  if (byte <= kCkptTop || byte == 255u) return;
  byte = kCkptTop;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = fminf(fmaxf(x[i], -127.f * 0x1p121f), 127.f * 0x1p121f);
}
__device__ __forceinline__ uint2 ckpt_integers(const V8 &x, float per) {
  const V8 b = fma(x, per, v8(12582912.f));    // + 1.5 2^23: the integer in the low bits
  uint32_t q[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t lo = __byte_perm(__float_as_uint(b.p[2 * h].x), __float_as_uint(b.p[2 * h].y), 0x0040);
    const uint32_t hi = __byte_perm(__float_as_uint(b.p[2 * h + 1].x), __float_as_uint(b.p[2 * h + 1].y), 0x0040);
    q[h] = __byte_perm(lo, hi, 0x5410);
  }
  return make_uint2(q[0], q[1]);
}
__device__ __forceinline__ float ckpt_unit(uint32_t byte) {   // 2^e
  return __uint_as_float(byte == 255u ? 0x7fffffffu : byte << 23);
}
__device__ __forceinline__ float max_magnitude(const V8 &x) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) top = max_magnitude(top, x.p[i].x, x.p[i].y);
  return top;
}
// 16 columns of a thread; a lane pair holds a group.  Every lane of the warp takes part; columns behind the row's end are zero.
__device__ __forceinline__ void ckpt_encode(V8 lo, V8 hi, uint4 &q, uint32_t &byte) {
  byte = ckpt_byte(max_magnitude(max_magnitude(lo), max_magnitude(hi), 0.f));
  byte = max(byte, __shfl_xor_sync(0xffffffffu, byte, 1));
  if (__builtin_expect(byte > kCkptTop, 0)) {
    uint32_t same = byte;
    ckpt_cut(lo, same);
    ckpt_cut(hi, byte);
  }
  const float per = ckpt_per(byte);
  const uint2 a = ckpt_integers(lo, per), b = ckpt_integers(hi, per);
  q = make_uint4(a.x, a.y, b.x, b.y);
}
// The values times a number: (2^e q) factor with one rounding, as 2^e factor is exact.
__device__ __forceinline__ V8 ckpt_decode(uint2 q, float unit) {
  // the byte q + 128 in the low bits of 2^23 is 2^23 + 128 + q; both steps are exact
  const uint32_t w[2] = {q.x ^ 0x80808080u, q.y ^ 0x80808080u};
  V8 x;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(__byte_perm(w[i >> 2], 0x4b000000u, 0x7650 | (i & 3)));
  return (x + v8(-8388736.f)) * unit;
}

}  // namespace augtree
