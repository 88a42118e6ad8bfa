// Element-wise kernels around the 8-bit activation checkpoints: to 8 bits and back, and the gated MLP's activation.
//
//   a = g s u,  s = 1 / (1 + e^-g)          dg = da u s (1 + g (1 - s)),   du = da g s
//
// All are bound by memory: every value passes once, in 16-byte accesses.  A thread takes 8 columns (one 16-byte piece of a 16-bit
// row, 8 bytes of an 8-bit one) at kPieces places of a block's range, all loads before the first use.  Rows are
// counted in pieces rounded up to a multiple of four, so that four neighbouring lanes always hold one group of 32 columns.
#pragma once
#include "ckpt.cuh"

namespace augtree {

constexpr int kActThreads = 256;

// Piece number -> row, piece of the row.  One multiplication: inv = ceil(2^64 / per_row) is exact while number x per_row < 2^64.
struct Pieces {
  unsigned long long inv;
  long long total;      // rows x per_row
  int per_row;          // pieces of a row, a multiple of four
  int valid;            // pieces of a row that exist
  __device__ __forceinline__ bool at(long long i, long long &row, int &piece) const {
    row = (long long)__umul64hi((unsigned long long)i, inv);
    piece = (int)(i - row * per_row);
    return i < total && piece < valid;
  }
};

// e^-g by the special-function unit (2 units in the last place of g log2(e) and of 2^x), the quotient by its reciprocal: relative
// error below 1e-6 for |g| < 8 and absolute below 1e-6 everywhere, far under the rounding of 16-bit results.
__device__ __forceinline__ float logistic(float g) { return __fdividef(1.f, 1.f + __expf(-g)); }

__device__ __forceinline__ V8 logistic(const V8 &g) {
  V8 s;
#pragma unroll
  for (int i = 0; i < 8; ++i) s[i] = logistic(g[i]);
  return s;
}

struct CkptRows {        // where a checkpoint is read or written
  uint8_t *base;
  long long pitch, scales;
  __device__ __forceinline__ void store(long long row, int piece, uint2 q, uint32_t byte) const {
    uint8_t *r = base + row * pitch;
    *reinterpret_cast<uint2 *>(r + piece * 8) = q;
    if ((piece & 3) == 0) r[scales + (piece >> 2)] = (uint8_t)byte;
  }
  __device__ __forceinline__ uint2 bytes(long long row, int piece) const { return *reinterpret_cast<const uint2 *>(base + row * pitch + piece * 8); }
  __device__ __forceinline__ uint32_t scale(long long row, int piece) const { return base[row * pitch + scales + (piece >> 2)]; }
};

// 8 columns of a row's checkpoint; every lane of the warp takes part, pieces from `valid` on are not written
__device__ __forceinline__ void ckpt_store(uint8_t *row, int piece, int valid, long long scales, const V8 &x) {
  uint2 q;
  uint32_t byte;
  ckpt_encode(x, q, byte);
  if (piece >= valid) return;
  *reinterpret_cast<uint2 *>(row + piece * 8) = q;
  if ((piece & 3) == 0) row[scales + (piece >> 2)] = (uint8_t)byte;
}

template <typename In>
__global__ void __launch_bounds__(kActThreads)
ckpt_pack_kernel(const In *x, long long ld, const Pieces p, const CkptRows out) {
  constexpr int kPieces = 4;
  launch_next();
  wait_previous();
  const long long first = (long long)blockIdx.x * (kActThreads * kPieces) + threadIdx.x;
  V8 v[kPieces];
  long long row[kPieces];
  int piece[kPieces];
  bool ok[kPieces];
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    ok[k] = p.at(first + k * kActThreads, row[k], piece[k]);
    v[k] = ok[k] ? Row8<In>::load(x + row[k] * ld + piece[k] * 8) : v8(0.f);
  }
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    uint2 q;
    uint32_t byte;
    ckpt_encode(v[k], q, byte);
    if (ok[k]) out.store(row[k], piece[k], q, byte);
  }
}

template <typename Out>
__global__ void __launch_bounds__(kActThreads)
ckpt_unpack_kernel(const CkptRows in, const Pieces p, int have, const float *row_factor, const void *col_factor, int col_type, Out *out, long long ld) {
  constexpr int kPieces = 4;
  launch_next();
  wait_previous();
  const long long first = (long long)blockIdx.x * (kActThreads * kPieces) + threadIdx.x;
  uint2 q[kPieces];
  uint32_t byte[kPieces];
  long long row[kPieces];
  int piece[kPieces];
  bool ok[kPieces];
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    ok[k] = p.at(first + k * kActThreads, row[k], piece[k]);
    const bool there = ok[k] && piece[k] < have;      // pieces behind them, where an output has any, are zero
    q[k] = there ? in.bytes(row[k], piece[k]) : make_uint2(0, 0);
    byte[k] = there ? in.scale(row[k], piece[k]) : 0;
  }
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    if (!ok[k]) continue;
    V8 v = ckpt_decode(q[k], ckpt_unit(byte[k]));
    if (row_factor) v = v * row_factor[row[k]];
    if (col_factor) {
      const long long c = piece[k] * 8;
      if (col_type == T_BF16) v = v * Row8<__nv_bfloat16>::load(static_cast<const __nv_bfloat16 *>(col_factor) + c);
      else if (col_type == T_F16) v = v * Row8<__half>::load(static_cast<const __half *>(col_factor) + c);
      else v = v * Row8<float>::load(static_cast<const float *>(col_factor) + c);
    }
    Row8<Out>::store(out + row[k] * ld + piece[k] * 8, v);
  }
}

template <typename T, bool kKeep>
__global__ void __launch_bounds__(kActThreads)
glu_fwd_kernel(const T *g, const T *u, long long ld, const Pieces p, T *a, long long cols, const CkptRows ckpt_g, const CkptRows ckpt_u) {
  constexpr int kPieces = 2;
  launch_next();
  wait_previous();
  const long long first = (long long)blockIdx.x * (kActThreads * kPieces) + threadIdx.x;
  V8 x[kPieces], y[kPieces];
  long long row[kPieces];
  int piece[kPieces];
  bool ok[kPieces];
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    ok[k] = p.at(first + k * kActThreads, row[k], piece[k]);
    x[k] = ok[k] ? Row8<T>::load(g + row[k] * ld + piece[k] * 8) : v8(0.f);
    y[k] = ok[k] ? Row8<T>::load(u + row[k] * ld + piece[k] * 8) : v8(0.f);
  }
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    if constexpr (kKeep) {
      uint2 q;
      uint32_t byte;
      ckpt_encode(x[k], q, byte);
      if (ok[k]) ckpt_g.store(row[k], piece[k], q, byte);
      ckpt_encode(y[k], q, byte);
      if (ok[k]) ckpt_u.store(row[k], piece[k], q, byte);
    }
    if (!ok[k]) continue;
    Row8<T>::store(a + row[k] * cols + piece[k] * 8, x[k] * logistic(x[k]) * y[k]);
  }
}

template <typename T, bool kKept>
__global__ void __launch_bounds__(kActThreads)
glu_bwd_kernel(const T *da, const T *g, const T *u, long long ld, const CkptRows ckpt_g, const CkptRows ckpt_u, const Pieces p, long long cols,
               T *dg, T *du, long long ld_grad, T *a) {
  constexpr int kPieces = 2;
  launch_next();
  wait_previous();
  const long long first = (long long)blockIdx.x * (kActThreads * kPieces) + threadIdx.x;
  V8 d[kPieces], x[kPieces], y[kPieces];
  uint2 qg[kPieces], qu[kPieces];
  uint32_t bg[kPieces], bu[kPieces];
  long long row[kPieces];
  int piece[kPieces];
  bool ok[kPieces];
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    ok[k] = p.at(first + k * kActThreads, row[k], piece[k]);
    if (!ok[k]) continue;
    d[k] = Row8<T>::load(da + row[k] * cols + piece[k] * 8);
    if constexpr (kKept) {
      qg[k] = ckpt_g.bytes(row[k], piece[k]); bg[k] = ckpt_g.scale(row[k], piece[k]);
      qu[k] = ckpt_u.bytes(row[k], piece[k]); bu[k] = ckpt_u.scale(row[k], piece[k]);
    } else {
      x[k] = Row8<T>::load(g + row[k] * ld + piece[k] * 8);
      y[k] = Row8<T>::load(u + row[k] * ld + piece[k] * 8);
    }
  }
#pragma unroll
  for (int k = 0; k < kPieces; ++k) {
    if (!ok[k]) continue;
    if constexpr (kKept) {
      x[k] = ckpt_decode(qg[k], ckpt_unit(bg[k]));
      y[k] = ckpt_decode(qu[k], ckpt_unit(bu[k]));
    }
    const V8 s = logistic(x[k]), silu = x[k] * s;
    Row8<T>::store(dg + row[k] * ld_grad + piece[k] * 8, d[k] * y[k] * s * fma(x[k], fma(s, -1.f, v8(1.f)), v8(1.f)));
    Row8<T>::store(du + row[k] * ld_grad + piece[k] * 8, d[k] * silu);
    if (a) Row8<T>::store(a + row[k] * cols + piece[k] * 8, silu * y[k]);
  }
}

}  // namespace augtree
