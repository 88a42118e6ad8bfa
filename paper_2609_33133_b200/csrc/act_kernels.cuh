// Element-wise kernels around the 8-bit activation checkpoints: to 8 bits and back, and the gated MLP's activation.
//
//   a = g s u,  s = 1 / (1 + e^-g)          dg = da u s (1 + g (1 - s)),   du = da g s
//
// All are bound by memory: every value passes once.  A thread takes 16 columns at a time (32 bytes of a 16-bit row, 16 of an 8-bit one) and
// walks through the tensors in steps of the whole grid; what it needs some steps on is on its way while it works.  Rows are counted in
// pieces of 16 columns rounded up to an even number, so that two neighbouring lanes always hold one group of 32 columns.
// With 8 columns a thread the instructions per value were the bound (to 8 bits from bf16: 42 us for 16384 x 3584), and blocks that load,
// compute, store and leave kept too little in flight (gated MLP forward of 16384 x 18944 with checkpoints: 572 us).
#pragma once
#include <type_traits>

#include "ckpt.cuh"

namespace augtree {

constexpr int kActThreads = 256;
// Blocks an SM (so many registers a thread) and steps ahead.  Measured, us for (blocks, steps): to 8 bits, 24576 x 3584 fp32, (3, 2) 68, (4, 1) 71, (4, 2) 82;
// 16384 x 3584 bf16, (4, 2) 28, (4, 1) 31, (3, 2) 30; from 8 bits to bf16, 24576 x 3584, (4, 2) 45, (3, 2) 48, (4, 1) 50; gated MLP, 16384 x 18944 bf16 with
// checkpoints, forward (2, 1) 397, (3, 1) 461, (2, 2) 454, backward (2, 1) 491, (2, 2) 541, (3, 1) 594.
template <typename T> constexpr int kPackBlocks = sizeof(T) == 4 ? 3 : 4;
constexpr int kUnpackBlocks = 4, kCkptAhead = 2, kGluBlocks = 2, kGluAhead = 1;

// A walk over the pieces of [rows, per_row].
struct Pieces {
  unsigned long long inv;   // ceil(2^64 / per_row): one multiplication divides, exact while number x per_row < 2^64
  long long total;          // rows x per_row
  int per_row;              // pieces of a row, an even number
  int valid;                // runs of 8 columns that exist: the last piece may have one or none
  bool wide;                // 32-byte accesses: every row of every matrix starts on 32 bytes
  long long step_rows;      // a step of the grid, in rows and pieces
  int step_pieces;
};
struct PieceWalk {
  long long i, row;
  int piece;
  __device__ __forceinline__ explicit PieceWalk(const Pieces &p) {
    i = (long long)blockIdx.x * kActThreads + threadIdx.x;
    row = (long long)__umul64hi((unsigned long long)i, p.inv);
    piece = (int)(i - row * p.per_row);
  }
  // runs of 8 columns of this piece: 0, 1 or 2
  __device__ __forceinline__ int there(const Pieces &p) const { return i < p.total ? min(max(p.valid - 2 * piece, 0), 2) : 0; }
  __device__ __forceinline__ void next(const Pieces &p) {
    i += (long long)gridDim.x * kActThreads;
    row += p.step_rows;
    piece += p.step_pieces;
    if (piece >= p.per_row) { piece -= p.per_row; ++row; }
  }
};
// Runs `use` on every piece of the walk with what `load` fetched for it kAhead steps before.  Whole warps stay together (the checkpoints'
// shuffles): the loop ends where the warp's first lane is behind the end, and both get to know how much of their piece exists.
template <class T, int kAhead, class Load, class Use>
__device__ __forceinline__ void walk_pieces(const Pieces &p, Load load, Use use) {
  T ahead[kAhead];
  PieceWalk in(p), at(p);
#pragma unroll
  for (int k = 0; k < kAhead; ++k) {
    load(in, in.there(p), ahead[k]);
    in.next(p);
  }
  const int lane = threadIdx.x & 31;
  while (true) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (at.i - lane >= p.total) return;
      const T now = ahead[k];
      load(in, in.there(p), ahead[k]);
      in.next(p);
      use(at, at.there(p), now);
      at.next(p);
    }
  }
}
// 16 values as they come from memory
template <typename T> struct Raw16 { uint4 w[sizeof(T) == 4 ? 4 : 2]; };
__device__ __forceinline__ void load_32(const void *p, uint4 (&w)[2]) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0].x), "=r"(w[0].y), "=r"(w[0].z), "=r"(w[0].w), "=r"(w[1].x), "=r"(w[1].y), "=r"(w[1].z), "=r"(w[1].w) : "l"(p));
}
template <typename T> __device__ __forceinline__ Raw16<T> raw16(const T *p, int there, bool wide) {
  constexpr int kRun = sizeof(T) == 4 ? 2 : 1;    // 16-byte words of 8 values
  Raw16<T> r;
  const uint4 *q = reinterpret_cast<const uint4 *>(p);
  if (wide && there == 2) {
#pragma unroll
    for (int i = 0; i < kRun; ++i) load_32(q + 2 * i, reinterpret_cast<uint4 (&)[2]>(r.w[2 * i]));
  } else {
#pragma unroll
    for (int i = 0; i < 2 * kRun; ++i) r.w[i] = i / kRun < there ? q[i] : make_uint4(0, 0, 0, 0);
  }
  return r;
}
// run 0 or 1 of them
template <typename T> __device__ __forceinline__ V8 values(const Raw16<T> &r, int run) { return Row8<T>::load(reinterpret_cast<const T *>(&r) + run * 8); }
template <typename T> __device__ __forceinline__ void store16(T *p, int there, bool wide, const V8 &lo, const V8 &hi) {
  if (sizeof(T) == 2 && wide && there == 2) {
    alignas(16) T v[16];
    Row8<T>::store(v, lo);
    Row8<T>::store(v + 8, hi);
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = reinterpret_cast<const uint32_t *>(v)[i];
    st_global_v8(p, w);
    return;
  }
  if (there > 0) Row8<T>::store(p, lo);
  if (there > 1) Row8<T>::store(p + 8, hi);
}

// e^-g by the special-function unit (2 units in the last place of g log2(e) and of 2^x), the quotient by its reciprocal: relative
// error below 1e-6 for |g| < 8 and absolute below 1e-6 everywhere, far under the rounding of 16-bit results.  An fp32 result carries it, up to 17 of its half steps, beside
// inputs that mostly come from 16-bit products; the exact exponential and quotient take some 20 instructions more a value.
__device__ __forceinline__ float logistic(float g) { return __fdividef(1.f, 1.f + __expf(-g)); }
// With its derivative a (1 - a), as e^-|g| a^2 or the like: the difference would lose all its figures where a is near one.
struct Logistic { float a, slope; };
__device__ __forceinline__ Logistic logistic_pair(float g) {
  const float t = __expf(-fabsf(g)), s = __fdividef(1.f, 1.f + t), ts = t * s;
  return {g < 0.f ? ts : s, ts * s};
}

__device__ __forceinline__ V8 logistic(const V8 &g) {
  V8 s;
#pragma unroll
  for (int i = 0; i < 8; ++i) s[i] = logistic(g[i]);
  return s;
}

struct CkptRows {        // where a checkpoint is read or written
  uint8_t *base;
  long long pitch, scales;
};
// 16 columns of a checkpoint as they come from memory (its rows go on to 16 columns)
struct RawCkpt {
  uint4 q;
  uint32_t byte;
};
__device__ __forceinline__ RawCkpt raw_ckpt(const CkptRows &c, long long row, int piece, bool there) {
  RawCkpt r = {make_uint4(0, 0, 0, 0), 0};
  if (there) {
    const uint8_t *p = c.base + row * c.pitch;
    r.q = *reinterpret_cast<const uint4 *>(p + piece * 16);
    r.byte = p[c.scales + (piece >> 1)];
  }
  return r;
}
__device__ __forceinline__ V8 values(const RawCkpt &r, int run, float f = 1.f) {
  return ckpt_decode(run ? make_uint2(r.q.z, r.q.w) : make_uint2(r.q.x, r.q.y), ckpt_unit(r.byte) * f);
}

// 16 columns of a row's checkpoint; every lane of the warp takes part
__device__ __forceinline__ void ckpt_store16(uint8_t *row, int piece, bool there, long long scales, const V8 &lo, const V8 &hi) {
  uint4 q;
  uint32_t byte;
  ckpt_encode(lo, hi, q, byte);
  if (!there) return;
  *reinterpret_cast<uint4 *>(row + piece * 16) = q;
  if ((piece & 1) == 0) row[scales + (piece >> 1)] = (uint8_t)byte;
}

template <typename In>
__global__ void __launch_bounds__(kActThreads, kPackBlocks<In>)
ckpt_pack_kernel(const In *x, long long ld, const Pieces p, const CkptRows out) {
  launch_next();
  wait_previous();
  walk_pieces<Raw16<In>, kCkptAhead>(
      p, [&](const PieceWalk &w, int there, Raw16<In> &r) { r = raw16(x + w.row * ld + w.piece * 16, there, p.wide); },
      [&](const PieceWalk &w, int there, const Raw16<In> &r) { ckpt_store16(out.base + w.row * out.pitch, w.piece, there, out.scales, values(r, 0), values(r, 1)); });
}

// Runs of 8 columns from `have` on, where the output has any, are zero.
template <typename Out>
__global__ void __launch_bounds__(kActThreads, kUnpackBlocks)
ckpt_unpack_kernel(const CkptRows in, const Pieces p, int have, const float *row_factor, const void *col_factor, int col_type, Out *out, long long ld) {
  launch_next();
  wait_previous();
  struct Item { RawCkpt x; float f; };
  walk_pieces<Item, kCkptAhead>(
      p,
      [&](const PieceWalk &w, int there, Item &r) {
        r.x = raw_ckpt(in, w.row, w.piece, there && 2 * w.piece < have);
        r.f = row_factor && there ? row_factor[w.row] : 1.f;
      },
      [&](const PieceWalk &w, int there, const Item &r) {
        if (!there) return;
        V8 v[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          v[h] = values(r.x, h, r.f);
          if (2 * w.piece + h >= have) v[h] = v8(0.f);      // (what lies behind the last column is not defined)
          if (col_factor && h < there) {
            const int c = w.piece * 16 + h * 8;
            if (col_type == T_BF16) v[h] = v[h] * Row8<__nv_bfloat16>::load(static_cast<const __nv_bfloat16 *>(col_factor) + c);
            else if (col_type == T_F16) v[h] = v[h] * Row8<__half>::load(static_cast<const __half *>(col_factor) + c);
            else v[h] = v[h] * Row8<float>::load(static_cast<const float *>(col_factor) + c);
          }
        }
        store16(out + w.row * ld + w.piece * 16, there, p.wide, v[0], v[1]);
      });
}

template <typename T, bool kKeep>
__global__ void __launch_bounds__(kActThreads, kGluBlocks)
glu_fwd_kernel(const T *g, const T *u, long long ld, const Pieces p, T *a, long long cols, const CkptRows ckpt_g, const CkptRows ckpt_u) {
  launch_next();
  wait_previous();
  struct Item { Raw16<T> g, u; };
  walk_pieces<Item, kGluAhead>(
      p,
      [&](const PieceWalk &w, int there, Item &r) {
        const long long at = w.row * ld + w.piece * 16;
        r.g = raw16(g + at, there, p.wide);
        r.u = raw16(u + at, there, p.wide);
      },
      [&](const PieceWalk &w, int there, const Item &r) {
        const V8 x[2] = {values(r.g, 0), values(r.g, 1)}, y[2] = {values(r.u, 0), values(r.u, 1)};
        if constexpr (kKeep) {
          const long long at = w.row * ckpt_g.pitch;
          ckpt_store16(ckpt_g.base + at, w.piece, there, ckpt_g.scales, x[0], x[1]);
          ckpt_store16(ckpt_u.base + at, w.piece, there, ckpt_g.scales, y[0], y[1]);
        }
        store16(a + w.row * cols + w.piece * 16, there, p.wide, x[0] * logistic(x[0]) * y[0], x[1] * logistic(x[1]) * y[1]);
      });
}

template <typename T, bool kKept>
__global__ void __launch_bounds__(kActThreads, kGluBlocks)
glu_bwd_kernel(const T *da, const T *g, const T *u, long long ld, const CkptRows ckpt_g, const CkptRows ckpt_u, const Pieces p, long long cols,
               T *dg, T *du, long long ld_grad, T *a) {
  launch_next();
  wait_previous();
  using Saved = std::conditional_t<kKept, RawCkpt, Raw16<T>>;
  struct Item { Raw16<T> d; Saved g, u; };
  walk_pieces<Item, kGluAhead>(
      p,
      [&](const PieceWalk &w, int there, Item &r) {
        r.d = raw16(da + w.row * cols + w.piece * 16, there, p.wide);
        if constexpr (kKept) {
          r.g = raw_ckpt(ckpt_g, w.row, w.piece, there);
          r.u = raw_ckpt(ckpt_u, w.row, w.piece, there);
        } else {
          const long long at = w.row * ld + w.piece * 16;
          r.g = raw16(g + at, there, p.wide);
          r.u = raw16(u + at, there, p.wide);
        }
      },
      [&](const PieceWalk &w, int there, const Item &r) {
        V8 dg8[2], du8[2], a8[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const V8 d = values(r.d, h), x = values(r.g, h), y = values(r.u, h), s = logistic(x), silu = x * s;
          dg8[h] = d * y * s * fma(x, fma(s, -1.f, v8(1.f)), v8(1.f));
          du8[h] = d * silu;
          a8[h] = silu * y;
        }
        const long long at = w.row * ld_grad + w.piece * 16;
        store16(dg + at, there, p.wide, dg8[0], dg8[1]);
        store16(du + at, there, p.wide, du8[0], du8[1]);
        if (a) store16(a + w.row * cols + w.piece * 16, there, p.wide, a8[0], a8[1]);
      });
}

}  // namespace augtree
