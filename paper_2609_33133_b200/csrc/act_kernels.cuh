// Element-wise kernels around the 8-bit activation checkpoints: to 8 bits and back, and the gated MLP's activation.
//
//   a = g s u,  s = 1 / (1 + e^-g)          dg = da u s (1 + g (1 - s)),   du = da g s
//
// All are bound by memory: every value passes once, in 16-byte accesses.  A thread takes 8 columns at a time (one 16-byte piece of a
// 16-bit row, 8 bytes of an 8-bit one) and walks through the tensors in steps of the whole grid; what it needs some steps on is on its way
// while it works (blocks that load, compute, store and leave kept 6/10 of that in flight: gated MLP forward of 16384 x 18944 with
// checkpoints 572 us).  Rows are counted in pieces rounded up to a multiple of four, so that four neighbouring lanes always hold one group of 32 columns.
#pragma once
#include <type_traits>

#include "ckpt.cuh"

namespace augtree {

constexpr int kActThreads = 256;
// Blocks an SM (so many registers a thread), and steps ahead.  Gated MLP, 16384 x 18944 bf16 with checkpoints, us for (blocks, steps): forward (4, 2) 479,
// (3, 2) 419, (3, 4) 471, (2, 2) 533, (2, 6) 423; backward (4, 2) 752, (3, 2) 544, (3, 3) 571, (2, 3) 509, (2, 6) 573.  To 8 bits and back, 24576 x 3584
// from fp32 to bf16: (4, 2) 66 and 55, (3, 2) 73 and 67, (2, 3) 83 and 76.
constexpr int kPackBlocks = 4, kPackAhead = 2, kGluFwdBlocks = 3, kGluFwdAhead = 2, kGluBwdBlocks = 2;
template <typename T> constexpr int kGluBwdAhead = sizeof(T) == 4 ? 2 : 3;     // (fp32 takes twice the registers)

// A walk over the pieces of [rows, per_row].
struct Pieces {
  unsigned long long inv;   // ceil(2^64 / per_row): one multiplication divides, exact while number x per_row < 2^64
  long long total;          // rows x per_row
  int per_row;              // pieces of a row, a multiple of four
  int valid;                // pieces of a row that exist
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
  __device__ __forceinline__ bool there(const Pieces &p) const { return i < p.total && piece < p.valid; }
  __device__ __forceinline__ void next(const Pieces &p) {
    i += (long long)gridDim.x * kActThreads;
    row += p.step_rows;
    piece += p.step_pieces;
    if (piece >= p.per_row) { piece -= p.per_row; ++row; }
  }
};
// Runs `use` on every piece of the walk with what `load` fetched for it kAhead steps before.  Whole warps stay together (the checkpoints'
// shuffles): the loop ends where the warp's first lane is behind the end, and both get to know whether their piece exists.
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
// 8 values as they come from memory
template <typename T> struct Raw8 { uint4 w; };
template <> struct Raw8<float> { uint4 w, v; };
template <typename T> __device__ __forceinline__ Raw8<T> raw8(const T *p, bool there) {
  Raw8<T> r;
  r.w = there ? *reinterpret_cast<const uint4 *>(p) : make_uint4(0, 0, 0, 0);
  if constexpr (sizeof(T) == 4) r.v = there ? reinterpret_cast<const uint4 *>(p)[1] : make_uint4(0, 0, 0, 0);
  return r;
}
template <typename T> __device__ __forceinline__ V8 values(const Raw8<T> &r) { return Row8<T>::load(reinterpret_cast<const T *>(&r)); }

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
};
// 8 columns of a checkpoint as they come from memory
struct RawCkpt {
  uint2 q;
  uint32_t byte;
};
__device__ __forceinline__ RawCkpt raw_ckpt(const CkptRows &c, long long row, int piece, bool there) {
  RawCkpt r = {make_uint2(0, 0), 0};
  if (there) {
    const uint8_t *p = c.base + row * c.pitch;
    r.q = *reinterpret_cast<const uint2 *>(p + piece * 8);
    r.byte = p[c.scales + (piece >> 2)];
  }
  return r;
}
__device__ __forceinline__ V8 values(const RawCkpt &r) { return ckpt_decode(r.q, ckpt_unit(r.byte)); }

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
__global__ void __launch_bounds__(kActThreads, kPackBlocks)
ckpt_pack_kernel(const In *x, long long ld, const Pieces p, const CkptRows out) {
  launch_next();
  wait_previous();
  walk_pieces<Raw8<In>, kPackAhead>(
      p, [&](const PieceWalk &w, bool there, Raw8<In> &r) { r = raw8(x + w.row * ld + w.piece * 8, there); },
      [&](const PieceWalk &w, bool there, const Raw8<In> &r) { ckpt_store(out.base + w.row * out.pitch, w.piece, there ? p.valid : 0, out.scales, values(r)); });
}

// Pieces from `have` on, where the output has any, are zero.
template <typename Out>
__global__ void __launch_bounds__(kActThreads, kPackBlocks)
ckpt_unpack_kernel(const CkptRows in, const Pieces p, int have, const float *row_factor, const void *col_factor, int col_type, Out *out, long long ld) {
  launch_next();
  wait_previous();
  struct Item { RawCkpt x; float f; };
  walk_pieces<Item, kPackAhead>(
      p,
      [&](const PieceWalk &w, bool there, Item &r) {
        r.x = raw_ckpt(in, w.row, w.piece, there && w.piece < have);
        r.f = row_factor && there ? row_factor[w.row] : 1.f;
      },
      [&](const PieceWalk &w, bool there, const Item &r) {
        if (!there) return;
        V8 v = values(r.x) * r.f;
        if (col_factor) {
          const int c = w.piece * 8;
          if (col_type == T_BF16) v = v * Row8<__nv_bfloat16>::load(static_cast<const __nv_bfloat16 *>(col_factor) + c);
          else if (col_type == T_F16) v = v * Row8<__half>::load(static_cast<const __half *>(col_factor) + c);
          else v = v * Row8<float>::load(static_cast<const float *>(col_factor) + c);
        }
        Row8<Out>::store(out + w.row * ld + w.piece * 8, v);
      });
}

template <typename T, bool kKeep>
__global__ void __launch_bounds__(kActThreads, kGluFwdBlocks)
glu_fwd_kernel(const T *g, const T *u, long long ld, const Pieces p, T *a, long long cols, const CkptRows ckpt_g, const CkptRows ckpt_u) {
  launch_next();
  wait_previous();
  struct Item { Raw8<T> g, u; };
  walk_pieces<Item, kGluFwdAhead>(
      p,
      [&](const PieceWalk &w, bool there, Item &r) {
        const long long at = w.row * ld + w.piece * 8;
        r.g = raw8(g + at, there);
        r.u = raw8(u + at, there);
      },
      [&](const PieceWalk &w, bool there, const Item &r) {
        const V8 x = values(r.g), y = values(r.u);
        if constexpr (kKeep) {
          const long long at = w.row * ckpt_g.pitch;
          const int valid = there ? p.valid : 0;
          ckpt_store(ckpt_g.base + at, w.piece, valid, ckpt_g.scales, x);
          ckpt_store(ckpt_u.base + at, w.piece, valid, ckpt_g.scales, y);
        }
        if (there) Row8<T>::store(a + w.row * cols + w.piece * 8, x * logistic(x) * y);
      });
}

template <typename T, bool kKept>
__global__ void __launch_bounds__(kActThreads, kGluBwdBlocks)
glu_bwd_kernel(const T *da, const T *g, const T *u, long long ld, const CkptRows ckpt_g, const CkptRows ckpt_u, const Pieces p, long long cols,
               T *dg, T *du, long long ld_grad, T *a) {
  launch_next();
  wait_previous();
  using Saved = std::conditional_t<kKept, RawCkpt, Raw8<T>>;
  struct Item { Raw8<T> d; Saved g, u; };
  walk_pieces<Item, kGluBwdAhead<T>>(
      p,
      [&](const PieceWalk &w, bool there, Item &r) {
        r.d = raw8(da + w.row * cols + w.piece * 8, there);
        if constexpr (kKept) {
          r.g = raw_ckpt(ckpt_g, w.row, w.piece, there);
          r.u = raw_ckpt(ckpt_u, w.row, w.piece, there);
        } else {
          const long long at = w.row * ld + w.piece * 8;
          r.g = raw8(g + at, there);
          r.u = raw8(u + at, there);
        }
      },
      [&](const PieceWalk &w, bool there, const Item &r) {
        if (!there) return;
        const V8 d = values(r.d), x = values(r.g), y = values(r.u), s = logistic(x), silu = x * s;
        const long long at = w.row * ld_grad + w.piece * 8;
        Row8<T>::store(dg + at, d * y * s * fma(x, fma(s, -1.f, v8(1.f)), v8(1.f)));
        Row8<T>::store(du + at, d * silu);
        if (a) Row8<T>::store(a + w.row * cols + w.piece * 8, silu * y);
      });
}

}  // namespace augtree
