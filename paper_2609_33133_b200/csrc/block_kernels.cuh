// The ends of a decoder block: norm after the block, gate, residual scale, residual, norm before the next block, and their gradients.
//
//   forward    z = w_o o r_o,  r_o = rsqrt(mean o^2 + eps)        (z = o without a norm after the block)
//              y = x + s a(g) z,  h = w_i y r_i,  r_i = rsqrt(mean y^2 + eps)
//   backward   v = y r_i,  d = dy + r_i (w_i dh - v mean(w_i dh v)) = dx,      dw_i = sum over tokens of dh v
//              u = o r_o,  do = r_o (w_o s a d - u mean(w_o s a d u)),           dw_o = sum over tokens of s a d u
//              dg = s a'(g) d w_o u, summed over the channels for a gate of one number a token and over the tokens for one a channel
//
// Bound by memory: a row passes once, all arithmetic is in registers.  Rows are fetched ahead by the copy engine (one bulk copy per tensor and
// block of rows, which are contiguous) into a ring of stages in shared memory, so what is in flight does not depend on how many threads
// wait: 44 GB/s and SM at 6.5 TB/s need 35 KB in flight against 0.8 us of latency, and a row of 3584 channels is 21 KB forward and 43 KB
// backward.  One CTA an SM; its warps form `groups`, and each takes a row of a stage at a time, so one group's reductions run under another's
// arithmetic.  A thread holds kParts pieces of 8 columns of a row.  (Rings of single rows, one for each group, took a sixth longer for the backward pass of
// 24576 x 3584 fp32, with the same instructions: copies of one row keep the memory less busy than copies of two.)
// A group's sum over a row: shuffles, then the warps' sums through shared memory behind one named barrier.
// The sums over tokens stay in registers (every thread owns its columns for all rows of its group), go over the groups through shared memory
// and from CTA to CTA through scratch and a second kernel, in an order that depends on the sizes alone: no atomics, bitwise repeatable.
// Measured (share of the bytes' time at 6.56 TB/s): 24576 x 3584 with an fp32 stream, forward and backward 411 to 421 us (97 %; a loop of one direction alone takes
// 181 and 260, 89 and 93 %); 16384 x 3584 with a bf16 stream and checkpoints, which has 10 bytes a value for about the same arithmetic, forward 108 to 115 us (80 %),
// backward 134 us (67 %; 136 with a logistic gate of a token): 37 and 36 instructions a value, of which half are arithmetic on the values, issue slots 60 % busy.  Forward 16 warps, backward 14 of 128 registers
// are all that fit, and the rest is waits for fixed latencies, shared memory and the row's sums.  (Both means of the backward pass from three sums behind
// one barrier, which d's linearity allows: one more product a value, and no faster.)
// Every sum, statistic and product is fp32; values are rounded once, on delivery.  The 8-bit form of y is made from y as it is
// delivered, so that it is the form that ckpt_pack makes of the tensor.
#pragma once
#include "act_kernels.cuh"

namespace augtree {

enum : int { GATE_NONE = 0, GATE_TOKEN = 1, GATE_CHANNEL = 2, GATE_FULL = 3 };
enum : int { WAIT_BLOCK_FULL = 90, WAIT_BLOCK_EMPTY = 91 };

constexpr int kBlockMaxHidden = 8192;
// Warps that compute; one more loads.  With it the count divides by the four schedulers of an SM, whose registers a thread's share is
// cut from: 96 forward, 128 backward.  Rows of more than 7680 columns take 16 warps backward, with 96 and some spills.
constexpr int kBlockFwdWarps = 19, kBlockBwdWarps = 15, kBlockBwdWarpsWide = 16;
constexpr int kBlockSmem = 227 * 1024;
constexpr int kBlockFixed = 256 + kBlockFwdWarps * 256;   // barriers, the groups' sums
constexpr int kBlockMaxStages = 8;
constexpr int kBlockMaxInputs = 5;

// The shape of a launch, chosen on the host.
struct BlockShape {
  int rows, hidden, vecs;         // vecs: pieces of 8 columns of a row
  int warps_row, groups;          // warps of a group; groups of a CTA
  int block_rows, blocks;         // rows of a stage; blocks of rows of the call
  int stages, stage_bytes;
  int n_inputs;
  const uint8_t *input[kBlockMaxInputs];
  int row_bytes[kBlockMaxInputs], offset[kBlockMaxInputs];   // bytes of a row; where its block lies in a stage
  int weights;                    // fp32 copies of per-channel vectors behind the stages: how many
};

struct BlockParams {
  BlockShape s;
  float inv_hidden, eps, scale;
  int gate, sigmoid, gate_type;
  const void *gate_ptr;
  const void *w_out, *w_in;       // null: no such norm
  int w_type;
  float *r_out, *r_in;            // forward: written where not null; backward: read
  int x_type, o_type, h_type, y_type;    // x: stream (x, y, dy, dx); o: branch or its 8-bit form; backward: y_type of what v is read from
  int do_type;
  int has_branch, has_dy, has_dh;
  void *y, *h;                    // forward
  CkptRows ckpt_y, ckpt_o;        // forward: base null = not kept
  void *dx, *d_o, *dg;            // backward
  float *part;                    // backward: [CTAs][2][hidden]
  int *status;
  long long wait_budget;
  int test_flags;
};

// What is compiled in.  Types for the usual pairs of stream and branch (fp32 or bf16 with bf16); kAny: looked up.  Form of the call:
// kBoth (a branch, a norm before the next block, every gradient wanted; the norm after the block is looked up) with its gate, kBefore
// (the norm before a block alone), kAny.  With everything looked up a value cost 60 instructions forward and 90 backward (bf16, checkpoints) where
// its arithmetic is about 20, and the issue rate was the bound.
constexpr int kAny = -1;
enum : int { kBoth = 0, kBefore = 1 };

__device__ __forceinline__ int type_bytes(int type) { return type == T_F32 ? 4 : 2; }

// 8 columns of a row in shared memory, from the row's first byte
template <int T>
__device__ __forceinline__ V8 block_load8(const uint8_t *row, int vec, int type, int scales) {
  const int k = T == kAny ? type : T;
  if (k == T_BF16) return Row8<__nv_bfloat16>::load(reinterpret_cast<const __nv_bfloat16 *>(row + vec * 16));
  if (k == T_F32) return Row8<float>::load(reinterpret_cast<const float *>(row + vec * 32));
  if (k == T_CKPT) return ckpt_decode(*reinterpret_cast<const uint2 *>(row + vec * 8), ckpt_unit(row[scales + (vec >> 2)]));
  return Row8<__half>::load(reinterpret_cast<const __half *>(row + vec * 16));
}
// the same times a number (one rounding either way)
template <int T>
__device__ __forceinline__ V8 block_load8_times(const uint8_t *row, int vec, int type, int scales, float f) {
  if constexpr (T == T_CKPT) return ckpt_decode(*reinterpret_cast<const uint2 *>(row + vec * 8), ckpt_unit(row[scales + (vec >> 2)]) * f);
  else return block_load8<T>(row, vec, type, scales) * f;
}
__device__ __forceinline__ V8 only_if(bool there, V8 x) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = there ? x[i] : 0.f;
  return x;
}
template <int T>
__device__ __forceinline__ void block_store8(uint8_t *row, int vec, int type, const V8 &x) {
  const int k = T == kAny ? type : T;
  if (k == T_BF16) Row8<__nv_bfloat16>::store(reinterpret_cast<__nv_bfloat16 *>(row + vec * 16), x);
  else if (k == T_F32) Row8<float>::store(reinterpret_cast<float *>(row + vec * 32), x);
  else Row8<__half>::store(reinterpret_cast<__half *>(row + vec * 16), x);
}
// A thread's kParts pieces of a row into its checkpoint.  The four lanes of a quad hold a group of 32 columns in each part; two parts' exponents go
// through one pair of shuffles, and each lane of the quad writes one part's.  Returns the largest of the thread's bytes, for block_cut.
template <int kParts>
__device__ __forceinline__ uint32_t block_keep(uint8_t *row, int v0, int step, int vecs, int scales, const V8 (&x)[kParts]) {
  uint32_t byte[kParts];
#pragma unroll
  for (int k = 0; k < kParts; ++k) byte[k] = ckpt_byte(max_magnitude(x[k]));
#pragma unroll
  for (int k = 0; k < kParts; k += 2) {
    uint32_t two = byte[k];
    if (k + 1 < kParts) two |= byte[k + 1] << 16;
    two = __vmaxu2(two, __shfl_xor_sync(0xffffffffu, two, 1));
    two = __vmaxu2(two, __shfl_xor_sync(0xffffffffu, two, 2));
    byte[k] = two & 0xffffu;
    if (k + 1 < kParts) byte[k + 1] = two >> 16;
  }
  const int quad = v0 & 3;
  uint32_t mine = byte[0];
#pragma unroll
  for (int k = 0; k < kParts; ++k) {
    const int v = v0 + k * step;
    const uint2 q = ckpt_integers(x[k], ckpt_per(byte[k]));
    if (v < vecs) *reinterpret_cast<uint2 *>(row + v * 8) = q;
    if (k == quad) mine = byte[k];
  }
  const int v = (v0 - quad) + quad * step;     // the group's first piece in part `quad`
  if (quad < kParts && v < vecs) row[scales + (v >> 2)] = (uint8_t)mine;
  uint32_t top = byte[0];
#pragma unroll
  for (int k = 1; k < kParts; ++k) top = max(top, byte[k]);
  return top;
}
// Makes the groups of a kept row again whose largest values have to be cut (ckpt_cut), from where the row still stands.  Behind everything else of the row and hardly ever: with the
// cut in block_keep, whose arithmetic runs among that of the rest of the row, the forward pass of 16384 x 3584 bf16 with checkpoints takes 119 to 138 us instead of 108.
template <int kParts, int T>
__device__ __forceinline__ void block_cut(uint8_t *row, const uint8_t *from, int type, int v0, int step, int vecs, int scales) {
  const uint32_t quad = threadIdx.x & 3, mask = 15u << (threadIdx.x & 28);     // (the four lanes of a quad come here together)
#pragma unroll 1
  for (int k = 0; k < kParts; ++k) {
    const int v = v0 + k * step;
    V8 x = only_if(v < vecs, block_load8<T>(from, min(v, vecs - 1), type, 0));
    uint32_t byte = ckpt_byte(max_magnitude(x));
    byte = max(byte, __shfl_xor_sync(mask, byte, 1));
    byte = max(byte, __shfl_xor_sync(mask, byte, 2));
    if (byte <= kCkptTop || byte == 255u) continue;
    ckpt_cut(x, byte);
    if (v < vecs) *reinterpret_cast<uint2 *>(row + v * 8) = ckpt_integers(x, ckpt_per(byte));
    if (quad == k && v - quad < vecs) row[scales + (v >> 2)] = (uint8_t)byte;      // (the lane that has written it before)
  }
}
// row t of a matrix in global memory
template <int T>
__device__ __forceinline__ uint8_t *block_row(void *base, unsigned t, int hidden, int type) {
  return static_cast<uint8_t *>(base) + (size_t)t * (unsigned)(hidden * type_bytes(T == kAny ? type : T));
}
__device__ __forceinline__ float block_scalar(const void *p, long long i, int type) {
  if (type == T_BF16) return __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
  if (type == T_F32) return static_cast<const float *>(p)[i];
  return __half2float(static_cast<const __half *>(p)[i]);
}
__device__ __forceinline__ void block_scalar_store(void *p, long long i, int type, float v) {
  if (type == T_BF16) static_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(v);
  else if (type == T_F32) static_cast<float *>(p)[i] = v;
  else static_cast<__half *>(p)[i] = __float2half_rn(v);
}
template <int T>
__device__ __forceinline__ V8 block_round(const V8 &x, int type) {
  const int k = T == kAny ? type : T;
  V8 y = x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (k == T_BF16) y.p[i] = Row8<__nv_bfloat16>::round(x.p[i]);
    else if (k == T_F16) y.p[i] = Row8<__half>::round(x.p[i]);
  }
  return y;
}

// What the roles of a CTA share.
struct BlockCta {
  uint8_t *smem;
  uint32_t base, bar_full, bar_empty;
  float *sums;        // [groups][2][32]
  volatile int *abort_flag;
  float *weights;     // [s.weights][hidden]
};

__device__ __forceinline__ BlockCta block_setup(uint8_t *smem, const BlockParams &p) {
  BlockCta c;
  c.smem = smem;
  c.base = smem_u32(smem);
  c.bar_full = c.base;
  c.bar_empty = c.base + 8 * kBlockMaxStages;
  c.abort_flag = reinterpret_cast<volatile int *>(smem + 16 * kBlockMaxStages);
  c.sums = reinterpret_cast<float *>(smem + 256);
  c.weights = reinterpret_cast<float *>(smem + kBlockFixed);
  if (threadIdx.x == 0) {
    for (int i = 0; i < p.s.stages; ++i) { mbar_init(c.bar_full + 8 * i, 1); mbar_init(c.bar_empty + 8 * i, p.s.groups * p.s.warps_row); }
    *c.abort_flag = 0;
    fence_barrier_init();
  }
  // (the entries behind a group's warps stay zero, so that the sums are read four at a time)
  for (int i = threadIdx.x; i < p.s.groups * 64; i += blockDim.x) c.sums[i] = 0.f;
  return c;
}
__device__ __forceinline__ uint8_t *block_stage(const BlockCta &c, const BlockParams &p, int stage) {
  return c.smem + kBlockFixed + p.s.weights * p.s.hidden * 4 + stage * p.s.stage_bytes;
}
// A vector of one number a channel into shared memory as fp32, the halves of its pieces of 8 in two runs, so that neighbouring lanes read
// neighbouring 16 bytes.
__device__ __forceinline__ V8 block_weight(const float *w, int vec, int vecs) {
  const float4 a = reinterpret_cast<const float4 *>(w)[vec], b = reinterpret_cast<const float4 *>(w)[vecs + vec];
  return {{make_float2(a.x, a.y), make_float2(a.z, a.w), make_float2(b.x, b.y), make_float2(b.z, b.w)}};
}
__device__ __forceinline__ void block_weights(const BlockCta &c, const BlockParams &p, int slot, const void *w, int type) {
  float *dst = c.weights + slot * p.s.hidden;
  for (int i = threadIdx.x; i < p.s.vecs; i += blockDim.x - 32) {      // (all warps but the loading one)
    V8 x;
    if (type == T_BF16) x = Row8<__nv_bfloat16>::load(static_cast<const __nv_bfloat16 *>(w) + i * 8);
    else if (type == T_F32) x = Row8<float>::load(static_cast<const float *>(w) + i * 8);
    else x = Row8<__half>::load(static_cast<const __half *>(w) + i * 8);
    reinterpret_cast<float4 *>(dst)[i] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4 *>(dst)[p.s.vecs + i] = make_float4(x[4], x[5], x[6], x[7]);
  }
}

// The loading warp: one thread, a ring of stages.  After a wait that gave up it loads nothing more; the copies that are under way
// are waited for by those who read them, and the CTA stays for a while before it leaves (block_leave).
__device__ __forceinline__ void block_produce(const BlockCta &c, const BlockParams &p, const AbortCtx &ab) {
  const BlockShape &s = p.s;
  int st = 0;
  uint32_t phase = 1;
  bool skip = (p.test_flags & TEST_SKIP_FWD_LOAD) && blockIdx.x == 0;
  for (long long b = blockIdx.x; b < s.blocks; b += gridDim.x) {
    if (!mbar_wait(c.bar_empty + 8 * st, phase, ab, WAIT_BLOCK_EMPTY)) return;
    const long long row0 = b * s.block_rows;
    const int rows = (int)min((long long)s.block_rows, s.rows - row0);
    const uint32_t full = c.bar_full + 8 * st, dst = smem_u32(block_stage(c, p, st));
    if (!skip) {
      int bytes = 0;
#pragma unroll
      for (int i = 0; i < kBlockMaxInputs; ++i) if (i < s.n_inputs) bytes += rows * s.row_bytes[i];
      mbar_expect_tx(full, bytes);
#pragma unroll
      for (int i = 0; i < kBlockMaxInputs; ++i)
        if (i < s.n_inputs) bulk_load_1d(dst + s.offset[i], s.input[i] + row0 * s.row_bytes[i], rows * s.row_bytes[i], full);
    }
    skip = false;
    if (++st == s.stages) { st = 0; phase ^= 1; }
  }
}
// A barrier of the warps that compute (the groups' own have the numbers from 1 on, ten at most).
__device__ __forceinline__ void block_sync_compute() { asm volatile("bar.sync 15, %0;" ::"r"(blockDim.x - 32) : "memory"); }
__device__ __forceinline__ void block_leave(const BlockCta &c) {
  __syncwarp();
  if (*c.abort_flag) {
    const long long t0 = clock64();
    while (clock64() - t0 < 400000) {}
  }
}

// Sum over a row, the same in every thread of the group.  `flip` alternates between two places, so that one barrier is enough: whoever
// writes a place again has passed the barrier of the sum between, behind which everybody has read it.
struct BlockGroup {
  float *sums;
  int warps, warp, bar, flip;
  __device__ __forceinline__ float sum(float v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if (warps == 1) return v;
    float *place = sums + flip * 32;
    if ((threadIdx.x & 31) == 0) place[warp] = v;
    asm volatile("bar.sync %0, %1;" ::"r"(bar), "r"(warps * 32) : "memory");
    // (16 warps at most, and zeros behind the last one)
    const float4 *q = reinterpret_cast<const float4 *>(place);
    const float4 a = q[0], b = q[1];
    v = ((a.x + a.y) + (a.z + a.w)) + ((b.x + b.y) + (b.z + b.w));
    if (warps > 8) {
      const float4 c = q[2], d = q[3];
      v += ((c.x + c.y) + (c.z + c.w)) + ((d.x + d.y) + (d.z + d.w));
    }
    flip ^= 1;
    return v;
  }
};

// A group's walk over its rows: block after block of the CTA, in each the rows group, group + groups, ..  `next` is the row behind
// the present one, kNone if there is none: its numbers are fetched while this one is worked on.  (Rows and blocks in 32 bits: there are less than 2^31 rows, and
// a turn of the grid is not longer than they are.)
struct BlockWalk {
  int group, groups, block_rows, rows;
  unsigned t, next;              // row; the one behind it
  static constexpr unsigned kNone = ~0u;
  __device__ __forceinline__ BlockWalk(const BlockShape &s, int group_)
      : group(group_), groups(s.groups), block_rows(s.block_rows), rows(s.rows) {
    const unsigned first = blockIdx.x * block_rows + group;
    next = group < block_rows && first < (unsigned)rows ? first : kNone;
  }
  __device__ __forceinline__ void at(unsigned row0, int r, int block) {      // `block`: rows of this block
    t = row0 + r;
    if (r + groups < block) { next = t + groups; return; }
    const unsigned first = row0 + gridDim.x * block_rows + group;
    next = first < (unsigned)rows ? first : kNone;     // (a group without a row in a block has none behind it either)
  }
};

template <int kParts, int XT, int OT, int FORM, int GATE>
__global__ void __launch_bounds__((kBlockFwdWarps + 1) * 32, 1)
block_fwd_kernel(const __grid_constant__ BlockParams p) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const BlockShape &s = p.s;
  const bool branch = FORM == kAny ? p.has_branch : FORM == kBoth, norm_in = FORM == kAny ? p.w_in != nullptr : true, norm_out = branch && p.w_out;
  const int gate = GATE == kAny ? p.gate : GATE;
  launch_next();
  const BlockCta c = block_setup(smem_raw, p);
  __syncthreads();
  wait_previous();
  const int hidden = s.hidden;
  // per-channel vectors: w_in, w_out, gate of a channel
  const float *w_in = c.weights, *w_out = w_in + (norm_in ? hidden : 0), *g_ch = w_out + (norm_out ? hidden : 0);
  const AbortCtx ab{c.abort_flag, p.status, p.wait_budget};
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (warp == s.groups * s.warps_row) {
    if (lane == 0) block_produce(c, p, ab);
  } else {
    if (norm_in) block_weights(c, p, 0, p.w_in, p.w_type);
    if (norm_out) block_weights(c, p, (int)(w_out - w_in) / hidden, p.w_out, p.w_type);
    if (gate == GATE_CHANNEL) block_weights(c, p, (int)(g_ch - w_in) / hidden, p.gate_ptr, p.gate_type);
    block_sync_compute();
    const int group = warp / s.warps_row;
    BlockGroup g{c.sums + group * 64, s.warps_row, warp - group * s.warps_row, group + 1, 0};
    const int v0 = g.warp * 32 + lane, step = s.warps_row * 32, vecs = s.vecs;     // pieces of 8 columns: v0, v0 + step, ..
    const bool writer = g.warp == 0 && lane == 0;
    int at[kParts];
    bool there[kParts];
#pragma unroll
    for (int k = 0; k < kParts; ++k) { there[k] = v0 + k * step < vecs; at[k] = min(v0 + k * step, vecs - 1); }
    int st = 0;
    uint32_t phase = 0;
    BlockWalk walk(s, group);
    float gt_next = gate == GATE_TOKEN && walk.next != BlockWalk::kNone ? block_scalar(p.gate_ptr, walk.next, p.gate_type) : 0.f;
    for (unsigned b = blockIdx.x; b < (unsigned)s.blocks; b += gridDim.x) {
      const unsigned row0 = b * s.block_rows;
      const int rows = min(s.block_rows, (int)(s.rows - row0));
      // A wait that gave up: the group goes on with whatever is there, so that nobody is left alone at a barrier; its results are
      // void, which the status word says, and every later wait gives up at once.
      mbar_wait(c.bar_full + 8 * st, phase, ab, WAIT_BLOCK_FULL);
      const uint8_t *stage = block_stage(c, p, st);
      for (int r = group; r < rows; r += s.groups) {
        walk.at(row0, r, rows);
        const unsigned t = walk.t;
        const uint8_t *rx = stage + s.offset[0] + r * s.row_bytes[0], *ro = stage + s.offset[1] + r * s.row_bytes[1];
        float ga = p.scale;
        if (gate == GATE_TOKEN) {
          ga *= p.sigmoid ? logistic(gt_next) : gt_next;
          if (walk.next != BlockWalk::kNone) gt_next = block_scalar(p.gate_ptr, walk.next, p.gate_type);
        }
        // Straight through, without a branch for the pieces behind the row's end: their threads work on the last piece (at[k]) and count for nothing.
        V8 y[kParts];
        uint32_t top_o = 0, top_y = 0;
        if (branch) {
          // (o is read twice rather than kept: registers are warps)
          float r_o = 1.f;
          if (norm_out || p.ckpt_o.base) {
            V8 o[kParts];
            float2 ss = both(0.f);
#pragma unroll
            for (int k = 0; k < kParts; ++k) {
              o[k] = only_if(there[k], block_load8<OT>(ro, at[k], p.o_type, 0));
              ss = dot2(o[k], o[k], ss);
            }
            if (p.ckpt_o.base) top_o = block_keep(p.ckpt_o.base + (size_t)t * (unsigned)p.ckpt_o.pitch, v0, step, vecs, (int)p.ckpt_o.scales, o);
            if (norm_out) {
              r_o = rsqrtf(fmaf(g.sum(ss.x + ss.y), p.inv_hidden, p.eps));
              if (p.r_out && writer) p.r_out[t] = r_o;
            }
          }
          uint8_t *ry = block_row<XT>(p.y, t, hidden, p.x_type);
#pragma unroll
          for (int k = 0; k < kParts; ++k) {
            V8 z = block_load8<OT>(ro, at[k], p.o_type, 0);
            if (norm_out) z = block_weight(w_out, at[k], vecs) * (z * r_o);
            if (gate >= GATE_CHANNEL) {
              const V8 a = gate == GATE_FULL ? block_load8<OT>(stage + s.offset[2] + r * s.row_bytes[2], at[k], p.gate_type, 0) : block_weight(g_ch, at[k], vecs);
              z = z * (p.sigmoid ? logistic(a) : a);
            }
            y[k] = only_if(there[k], fma(z, ga, block_load8<XT>(rx, at[k], p.x_type, 0)));
            if (there[k]) block_store8<XT>(ry, at[k], p.x_type, y[k]);
          }
        } else {
#pragma unroll
          for (int k = 0; k < kParts; ++k) y[k] = only_if(there[k], block_load8<XT>(rx, at[k], p.x_type, 0));
        }
        if (norm_in) {
          float2 ss = both(0.f);
#pragma unroll
          for (int k = 0; k < kParts; ++k) ss = dot2(y[k], y[k], ss);
          const float r_i = rsqrtf(fmaf(g.sum(ss.x + ss.y), p.inv_hidden, p.eps));
          if (p.r_in && writer) p.r_in[t] = r_i;
          uint8_t *rh = block_row<OT>(p.h, t, hidden, p.h_type);
#pragma unroll
          for (int k = 0; k < kParts; ++k) {
            const V8 h = block_weight(w_in, at[k], vecs) * (y[k] * r_i);
            if (there[k]) block_store8<OT>(rh, at[k], p.h_type, h);
          }
        }
        if (p.ckpt_y.base) {
#pragma unroll
          for (int k = 0; k < kParts; ++k) y[k] = block_round<XT>(y[k], p.x_type);
          top_y = block_keep(p.ckpt_y.base + (size_t)t * (unsigned)p.ckpt_y.pitch, v0, step, vecs, (int)p.ckpt_y.scales, y);
        }
        if (max(top_o, top_y) > kCkptTop) {
          if (top_o > kCkptTop) block_cut<kParts, OT>(p.ckpt_o.base + (size_t)t * (unsigned)p.ckpt_o.pitch, ro, p.o_type, v0, step, vecs, (int)p.ckpt_o.scales);
          if (top_y > kCkptTop)
            block_cut<kParts, XT>(p.ckpt_y.base + (size_t)t * (unsigned)p.ckpt_y.pitch, branch ? block_row<XT>(p.y, t, hidden, p.x_type) : rx, p.x_type, v0, step, vecs,
                                  (int)p.ckpt_y.scales);
        }
      }
      warp_arrive(c.bar_empty + 8 * st);
      if (++st == s.stages) { st = 0; phase ^= 1; }
    }
  }
  block_leave(c);
}

// kKept: v and u are read from checkpoints, both (with kAny each from what its type says).
template <int kParts, int kWarps, int XT, int OT, int FORM, int GATE, bool kKept>
__global__ void __launch_bounds__((kWarps + 1) * 32, 1)
block_bwd_kernel(const __grid_constant__ BlockParams p) {
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  constexpr int YT = XT == kAny ? kAny : kKept ? (int)T_CKPT : XT, ST = OT == kAny ? kAny : kKept ? (int)T_CKPT : OT;   // of the saved y and o
  const BlockShape &s = p.s;
  const bool branch = FORM == kAny ? p.has_branch : FORM == kBoth, has_dy = FORM == kAny ? p.has_dy : true, has_dh = FORM == kAny ? p.has_dh : true;
  const bool norm_out = branch && p.w_out, put_dx = FORM == kAny ? p.dx != nullptr : true, put_do = FORM == kAny ? p.d_o != nullptr : true;
  const int gate = GATE == kAny ? p.gate : GATE;
  launch_next();
  const BlockCta c = block_setup(smem_raw, p);
  __syncthreads();
  wait_previous();
  const int hidden = s.hidden;
  const float *w_in = c.weights, *w_out = w_in + (p.w_in ? hidden : 0), *g_ch = w_out + (norm_out ? hidden : 0);
  const AbortCtx ab{c.abort_flag, p.status, p.wait_budget};
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  V8 acc_in[kParts], acc_out[kParts];
#pragma unroll
  for (int k = 0; k < kParts; ++k) acc_in[k] = acc_out[k] = v8(0.f);
  const int group = warp / s.warps_row;
  BlockGroup g{c.sums + group * 64, s.warps_row, warp - group * s.warps_row, group + 1, 0};
  const int v0 = g.warp * 32 + lane, step = s.warps_row * 32, vecs = s.vecs;
  const bool computes = group < s.groups, writer = g.warp == 0 && lane == 0;
  int at[kParts];        // the thread's pieces, those behind the row's end replaced by the last one: see the forward kernel
  bool there[kParts];
#pragma unroll
  for (int k = 0; k < kParts; ++k) { there[k] = v0 + k * step < vecs; at[k] = min(v0 + k * step, vecs - 1); }
  if (!computes) {
    if (lane == 0) block_produce(c, p, ab);
    __syncwarp();
  } else {
    if (p.w_in) block_weights(c, p, 0, p.w_in, p.w_type);
    if (norm_out) block_weights(c, p, (int)(w_out - w_in) / hidden, p.w_out, p.w_type);
    if (gate == GATE_CHANNEL) block_weights(c, p, (int)(g_ch - w_in) / hidden, p.gate_ptr, p.gate_type);
    block_sync_compute();
    int st = 0;
    uint32_t phase = 0;
    // inputs in the order that the host lists them: dy, dh, y, o, gate, each only where there is one
    const int at_dh = has_dy, at_y = at_dh + has_dh, at_o = at_y + has_dh, at_g = at_o + branch;
    const int scales = (int)ckpt_scale_offset(hidden);
    BlockWalk walk(s, group);
    float ri_next = 0.f, ro_next = 1.f, gt_next = 1.f;
    auto fetch = [&]() {
      if (walk.next == BlockWalk::kNone) return;
      if (has_dh) ri_next = p.r_in[walk.next];
      if (norm_out) ro_next = p.r_out[walk.next];
      if (gate == GATE_TOKEN) gt_next = block_scalar(p.gate_ptr, walk.next, p.gate_type);
    };
    fetch();
    for (unsigned b = blockIdx.x; b < (unsigned)s.blocks; b += gridDim.x) {
      const unsigned row0 = b * s.block_rows;
      const int rows = min(s.block_rows, (int)(s.rows - row0));
      mbar_wait(c.bar_full + 8 * st, phase, ab, WAIT_BLOCK_FULL);
      const uint8_t *stage = block_stage(c, p, st);
      for (int r = group; r < rows; r += s.groups) {
        walk.at(row0, r, rows);
        const unsigned t = walk.t;
        auto row = [&](int i) { return stage + s.offset[i] + r * s.row_bytes[i]; };
        const float r_i = ri_next, r_o = ro_next, gate_t = gate == GATE_TOKEN && p.sigmoid ? logistic(gt_next) : gt_next;
        fetch();
        // v and u from checkpoints are kept between their two uses, others are read again (24576 x 3584 fp32, both directions: 414 us against 420 kept; 16384 x 3584
        // bf16 with checkpoints, backward: 133 us kept against 143).
        V8 d[kParts];
        if (has_dh) {
          V8 v[kParts];
          float2 dot = both(0.f);
          const uint8_t *rh = row(at_dh), *ry = row(at_y);
#pragma unroll
          for (int k = 0; k < kParts; ++k) {
            const V8 dh = only_if(there[k], block_load8<OT>(rh, at[k], p.h_type, 0));
            v[k] = block_load8_times<YT>(ry, at[k], p.y_type, scales, r_i);
            acc_in[k] = fma(dh, v[k], acc_in[k]);
            d[k] = block_weight(w_in, at[k], vecs) * dh;
            dot = dot2(d[k], v[k], dot);
          }
          const float mean = -g.sum(dot.x + dot.y) * p.inv_hidden;
#pragma unroll
          for (int k = 0; k < kParts; ++k) {
            if (YT != T_CKPT) v[k] = block_load8_times<YT>(ry, at[k], p.y_type, scales, r_i);
            d[k] = fma(v[k], mean, d[k]) * r_i;
          }
        } else {
#pragma unroll
          for (int k = 0; k < kParts; ++k) d[k] = v8(0.f);
        }
        {
          const uint8_t *ry = row(0);
          uint8_t *rx = block_row<XT>(p.dx, t, hidden, p.x_type);
#pragma unroll
          for (int k = 0; k < kParts; ++k) {
            if (has_dy) d[k] = d[k] + block_load8<XT>(ry, at[k], p.x_type, 0);
            if (put_dx && there[k]) block_store8<XT>(rx, at[k], p.x_type, d[k]);
          }
        }
        if (branch) {
          V8 u[kParts];
          float2 dot = both(0.f);    // sum of w_o q u a(g), without the a(g) of a token
          const uint8_t *ro = row(at_o);
#pragma unroll
          for (int k = 0; k < kParts; ++k) {
            u[k] = only_if(there[k], block_load8_times<ST>(ro, at[k], p.o_type, scales, r_o));
            const V8 q = d[k] * p.scale;
            if (gate >= GATE_CHANNEL) {
              V8 a = gate == GATE_FULL ? block_load8<OT>(row(at_g), at[k], p.gate_type, 0) : block_weight(g_ch, at[k], vecs), slope = v8(1.f);
              if (p.sigmoid) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                  const Logistic l = logistic_pair(a[i]);
                  a[i] = l.a;
                  slope[i] = l.slope;
                }
              }
              const V8 qa = q * a, w = norm_out ? block_weight(w_out, at[k], vecs) : v8(1.f);
              acc_out[k] = fma(gate == GATE_CHANNEL ? q : qa, u[k], acc_out[k]);
              d[k] = w * qa;
              if (gate == GATE_FULL && p.dg && there[k]) {
                V8 dg = q * (w * u[k]);
                if (p.sigmoid) dg = dg * slope;
                block_store8<OT>(block_row<OT>(p.dg, t, hidden, p.gate_type), at[k], p.gate_type, dg);
              }
            } else {
              acc_out[k] = fma(gate == GATE_TOKEN ? q * gate_t : q, u[k], acc_out[k]);
              d[k] = norm_out ? block_weight(w_out, at[k], vecs) * q : q;
            }
            dot = dot2(d[k], u[k], dot);
          }
          float mean = 0.f;
          if (norm_out || gate == GATE_TOKEN) {
            const float total = g.sum(dot.x + dot.y);
            mean = -total * p.inv_hidden;
            // (the slope from the gate once more, by the one thread that needs it: 16384 x 3584 bf16 with checkpoints 136 us; kept over the row in a register 138, in
            // shared memory 137)
            if (gate == GATE_TOKEN && p.dg && writer)
              block_scalar_store(p.dg, t, p.gate_type, total * (p.sigmoid ? logistic_pair(block_scalar(p.gate_ptr, t, p.gate_type)).slope : 1.f));
          }
          if (put_do) {
            const float f = r_o * gate_t;      // (1 without a norm, 1 without a gate of one number a token)
            uint8_t *rd = block_row<OT>(p.d_o, t, hidden, p.do_type);
#pragma unroll
            for (int k = 0; k < kParts; ++k) {
              if (norm_out) {
                if (ST != T_CKPT) u[k] = block_load8_times<ST>(ro, at[k], p.o_type, scales, r_o);
                d[k] = fma(u[k], mean, d[k]);
              }
              const V8 out = d[k] * f;
              if (there[k]) block_store8<OT>(rd, at[k], p.do_type, out);
            }
          }
        }
      }
      warp_arrive(c.bar_empty + 8 * st);
      if (++st == s.stages) { st = 0; phase ^= 1; }
    }
  }
  block_leave(c);
  // the groups' sums, one after the other, where the stages were (every copy into them has been read)
  __syncthreads();
  float *sum = reinterpret_cast<float *>(block_stage(c, p, 0));      // [groups][2][hidden]
  if (computes) {
    auto put = [&](float *dst, const V8 &x) {
      reinterpret_cast<float4 *>(dst)[0] = make_float4(x[0], x[1], x[2], x[3]);
      reinterpret_cast<float4 *>(dst)[1] = make_float4(x[4], x[5], x[6], x[7]);
    };
    float *mine = sum + (long long)group * 2 * hidden;
#pragma unroll
    for (int k = 0; k < kParts; ++k) {
      const int at8 = v0 + k * step;
      if (at8 >= vecs) continue;
      put(mine + at8 * 8, acc_in[k]);
      put(mine + hidden + at8 * 8, acc_out[k]);
    }
  }
  __syncthreads();
  const bool any_in = p.has_dh, any_out = p.w_out || p.gate == GATE_CHANNEL;
  for (int i = threadIdx.x; i < 2 * s.hidden; i += blockDim.x) {
    if (!(i < s.hidden ? any_in : any_out)) continue;
    float v = sum[i];
    for (int j = 1; j < s.groups; ++j) v += sum[(long long)j * 2 * s.hidden + i];
    p.part[(long long)blockIdx.x * 2 * s.hidden + i] = v;
  }
}

// The CTAs' sums over tokens into dw_in, dw_out and the gradient of a gate of one number a channel: 32 columns a block, 32 runs of CTAs
// side by side, a run's loads all at once (with 8 runs this kernel waited for memory five times, 2 us more).
// With such a gate the second sum is S = sum s d u, and dw_out = a(g) S, dg = a'(g) w_out S.
struct BlockSums {
  const float *part;
  int parts, hidden;
  const void *w_out, *gate;
  int w_type, gate_type, sigmoid, accumulate;
  void *dw_in, *dw_out, *dg;       // null: not wanted
};
__global__ void __launch_bounds__(1024) block_sums_kernel(const BlockSums p) {
  launch_next();
  wait_previous();
  __shared__ float run[32][33];
  const int lane = threadIdx.x & 31, slice = threadIdx.x >> 5, second = blockIdx.y;
  const int c = blockIdx.x * 32 + lane;
  float v = 0.f;
  if (c < p.hidden) {
    const float *q = p.part + (long long)second * p.hidden + c;
#pragma unroll 5
    for (int i = slice; i < p.parts; i += 32) v += q[(long long)i * 2 * p.hidden];
  }
  run[slice][lane] = v;
  __syncthreads();
  if (slice || c >= p.hidden) return;
#pragma unroll
  for (int i = 1; i < 32; ++i) v += run[i][lane];
  auto put = [&](void *dst, int type, float x) {
    if (p.accumulate) x += static_cast<const float *>(dst)[c];    // (fp32 only)
    block_scalar_store(dst, c, type, x);
  };
  if (!second) {
    if (p.dw_in) put(p.dw_in, p.w_type, v);
    return;
  }
  float a = 1.f, slope = 1.f;
  if (p.gate) {
    a = block_scalar(p.gate, c, p.gate_type);
    if (p.sigmoid) { const Logistic l = logistic_pair(a); a = l.a; slope = l.slope; }
    if (p.dg) put(p.dg, p.gate_type, v * slope * (p.w_out ? block_scalar(p.w_out, c, p.w_type) : 1.f));
  }
  if (p.dw_out) put(p.dw_out, p.w_type, v * a);
}

}  // namespace augtree
