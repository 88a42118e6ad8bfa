// Element-wise kernels around the vocabulary loss, and the embedding lookup with its gradient.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "ptx.cuh"

namespace augtree {

// an id beyond the vocabulary is left out like padding, and reported
template <typename Id>
__device__ __forceinline__ void check_id(Id id, int t, int vocab, int *status) {
  if ((long long)id >= vocab && atomicCAS(status, 0, -1) == 0) status[1] = t;
}

// ---------------------------------------------------------------- compaction of the scored rows
// Rows with a negative target are not scored.  They are left out of every product: their hidden states may hold
// anything, NaN included, and 0 x NaN in the contraction of dW would spoil it; and their work is saved.
// One block walks the targets in order, so the compacted order is that of the tokens.
struct LmRows {
  int *n_rows;      // [1]
  int *idx;         // [rows_pad] compacted row -> token
  int *pos;         // [tokens] token -> compacted row or -1
  int *target;      // [rows_pad]
  float *lse2;      // [rows_pad] backward only
  float *gscale;    // [rows_pad] backward only
  float *x_target;  // [rows_pad] forward: h . W_target; backward: the target's gradient a c (p - 1)
};

template <typename Id>
__global__ void __launch_bounds__(1024)
lm_compact_kernel(const Id *targets, int tokens, int vocab, LmRows o, const float *lse, const float *d_loss, float logit_scale,
                  float *loss_out, float *lse_out, int *status) {
  launch_next();
  wait_previous();
  __shared__ int warp_sum[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int n = 0;
  for (int t0 = 0; t0 < tokens; t0 += 1024) {
    const int t = t0 + (int)threadIdx.x;
    const long long id = t < tokens ? (long long)targets[t] : -1;
    const bool live = id >= 0 && id < vocab;
    check_id(id, t, vocab, status);
    const unsigned m = __ballot_sync(0xffffffffu, live);
    if (lane == 0) warp_sum[warp] = __popc(m);
    __syncthreads();
    if (warp == 0) {
      int s = warp_sum[lane];
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int u = __shfl_up_sync(0xffffffffu, s, d);
        if (lane >= d) s += u;
      }
      warp_sum[lane] = s;
    }
    __syncthreads();
    const int r = n + (warp ? warp_sum[warp - 1] : 0) + __popc(m & ((1u << lane) - 1));
    const int total = warp_sum[31];
    if (t < tokens) o.pos[t] = live ? r : -1;
    if (live) {
      o.idx[r] = t;
      o.target[r] = (int)id;
      if (lse) {
        o.lse2[r] = lse[t] * 1.4426950408889634f;
        o.gscale[r] = d_loss[t] * logit_scale;
      }
    } else if (t < tokens && loss_out) {
      loss_out[t] = 0.f;
      lse_out[t] = 0.f;
    }
    n += total;
    __syncthreads();
  }
  if (threadIdx.x == 0) *o.n_rows = n;
}

// h . W_target of a row in fp32 by a whole block, from 16-byte vectors of eight bf16 numbers.  The tensor core's adder drops
// what does not fit its accumulator, 224 times for 3584 columns, always towards zero: 3e-6 of a large logit, and the
// target's is the large one in a confident row.  This sum rounds to nearest, in short chains.  Valid in thread 0.  (The backward
// pass needs it too: p - 1 of a confident target is small, and 4e-5 of logit is 4 % of it where p is 0.999.)
__device__ __forceinline__ float dot8(const uint4 a, const uint4 b) {
  const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 u = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&x[i]));
    const float2 v = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&y[i]));
    s = fmaf(u.x, v.x, s);
    s = fmaf(u.y, v.y, s);
  }
  return s;
}
template <int THREADS>
__device__ __forceinline__ float block_sum(float s, float *sh) {
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0)
    for (int w = 1; w < THREADS / 32; ++w) s += sh[w];
  return s;
}

// p - 1 of the target from its logit, without the cancellation
__device__ __forceinline__ float target_gradient(float gscale, float x_target, float logit_scale, float lse) {
  return gscale * expm1f(fmaf(x_target, logit_scale, -lse));
}

// Hidden states of the scored rows, packed; zeros up to the next multiple of 256 rows (they enter contractions), and up to the next
// multiple of 64 columns, so that every box of the copy engine is whole lines.  Also their targets' logits (lse null) or gradients.
__global__ void __launch_bounds__(256)
lm_gather_kernel(const uint4 *hidden, const LmRows rows, uint4 *out, int row_vecs, int out_vecs, const uint4 *weight, const float *lse,
                 float logit_scale) {
  launch_next();
  wait_previous();
  __shared__ float sh[8];
  const int n = *rows.n_rows, n_pad = (n + 255) / 256 * 256;
  for (long long r = blockIdx.x; r < n_pad; r += gridDim.x) {   // (64 bits, here and below: a step past the last row passes 2^31)
    const uint4 *src = r < n ? hidden + (long long)rows.idx[r] * row_vecs : nullptr;
    const uint4 *wt = src ? weight + (long long)rows.target[r] * row_vecs : nullptr;
    uint4 *dst = out + r * out_vecs;
    float s = 0.f;
    for (int i = threadIdx.x; i < out_vecs; i += 256) {
      const uint4 v = src && i < row_vecs ? src[i] : make_uint4(0, 0, 0, 0);
      if (wt && i < row_vecs) s += dot8(v, wt[i]);
      dst[i] = v;
    }
    if (wt) {
      s = block_sum<256>(s, sh);
      if (threadIdx.x == 0) rows.x_target[r] = lse ? target_gradient(rows.gscale[r], s, logit_scale, lse[rows.idx[r]]) : s;
    }
  }
}

// Both in one launch for as many tokens as a block has threads: a block per packed row, each finds its token for itself.  With
// `twice` the rows are written a second time behind the first ones (they multiply the two halves of G).
template <typename Id, int THREADS>
__global__ void __launch_bounds__(THREADS)
lm_rows_kernel(const Id *targets, int tokens, int vocab, LmRows o, const float *lse, const float *d_loss, float logit_scale,
                   float *loss_out, float *lse_out, int *status, const uint4 *hidden, uint4 *out, int row_vecs,
                   int out_vecs, int twice, const uint4 *weight) {
  launch_next();
  wait_previous();
  __shared__ int warp_sum[THREADS / 32];
  __shared__ float sh[THREADS / 32];
  __shared__ int from;
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, row = blockIdx.x;
  const long long id = t < tokens ? (long long)targets[t] : -1;
  const bool live = id >= 0 && id < vocab;
  const unsigned m = __ballot_sync(0xffffffffu, live);
  if (lane == 0) warp_sum[warp] = __popc(m);
  if (t == 0) from = -1;
  __syncthreads();
  int r = __popc(m & ((1u << lane) - 1)), n = 0;
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < warp) r += warp_sum[w];
    n += warp_sum[w];
  }
  if (live && r == row) from = t;
  if (row == 0) {
    check_id(id, t, vocab, status);
    if (t < tokens) o.pos[t] = live ? r : -1;
    if (live) {
      o.idx[r] = t;
      o.target[r] = (int)id;
      if (lse) {
        o.lse2[r] = lse[t] * 1.4426950408889634f;
        o.gscale[r] = d_loss[t] * logit_scale;
      }
    } else if (t < tokens && loss_out) {
      loss_out[t] = 0.f;
      lse_out[t] = 0.f;
    }
    if (t == 0) *o.n_rows = n;
  }
  __syncthreads();
  const uint4 *src = from >= 0 ? hidden + (long long)from * row_vecs : nullptr;
  const uint4 *wt = src ? weight + (long long)targets[from] * row_vecs : nullptr;
  float s = 0.f;
  for (int i = t; i < out_vecs; i += THREADS) {
    const uint4 v = src && i < row_vecs ? src[i] : make_uint4(0, 0, 0, 0);
    if (wt && i < row_vecs) s += dot8(v, wt[i]);
    out[(long long)row * out_vecs + i] = v;
    if (twice) out[(long long)(gridDim.x + row) * out_vecs + i] = v;
  }
  if (wt) {
    s = block_sum<THREADS>(s, sh);
    if (t == 0) o.x_target[row] = lse ? target_gradient(d_loss[from] * logit_scale, s, logit_scale, lse[from]) : s;
  }
}

// ---------------------------------------------------------------- row statistics
__device__ __forceinline__ float2 merge_stats(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x), ref = m == -INFINITY ? 0.f : m;
  return make_float2(m, a.y * ex2(a.x - ref) + b.y * ex2(b.x - ref));
}

// Loss and lse of a row from its merged (m, l).  The target's term of the sum is 2^(t2 - m) with t2 = c log2(e) tlogit as the
// tile kernels rounded it (__fmul_rn there and here: a product left to be fused into the subtraction of m would not be that number);
// d is what t2 lacks of the exact x_target, and puts the term right.  The loss is taken as
// log of the sum relative to the target's term, so that a small loss is not the difference of two large numbers.
// A target that is ruled out (a logit of minus infinity, or one so low that base 2 makes it that) has no term in the sum and nothing
// to put right: the lse is that of the others.  (A logit of plus infinity leaves NaN in the sum, and so in both.)
__device__ __forceinline__ void write_loss(float2 s, float tlogit, float x_target, float logit_scale, float *loss, float *lse) {
  constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
  const float c = logit_scale * kLog2e, t2 = __fmul_rn(tlogit, c);
  const float d = fmaf(tlogit, c, -t2) + (x_target - tlogit) * c;
  if (!isfinite(d)) {
    const float v = s.x * kLn2 + logf(s.y);
    *lse = v;
    *loss = v - x_target * logit_scale;
    return;
  }
  const float l = s.y + ex2(t2 - s.x) * expm1f(d * kLn2);
  const float v = (s.x - t2 - d) * kLn2 + logf(l);
  *loss = v;
  *lse = v + x_target * logit_scale;
}

// Few rows: a block per token, its pairs one after the other in memory, and its target's logit beside them.
template <typename Id>
__global__ void __launch_bounds__(256)
lm_few_finish_kernel(const float2 *part, int n_part, const Id *targets, int vocab, const uint4 *hidden, const uint4 *weight, int row_vecs,
                     const float *tlogit, float logit_scale, float *loss, float *lse, int *status) {
  launch_next();
  wait_previous();
  __shared__ float2 sh[8];
  __shared__ float dot[8];
  const int t = blockIdx.x;
  const long long id = targets[t];
  if (threadIdx.x == 0) check_id(targets[t], t, vocab, status);
  if (id < 0 || id >= vocab) {
    if (threadIdx.x == 0) { loss[t] = 0.f; lse[t] = 0.f; }
    return;
  }
  float x = 0.f;
  for (int i = threadIdx.x; i < row_vecs; i += 256) x += dot8(hidden[(long long)t * row_vecs + i], weight[id * row_vecs + i]);
  float2 s = make_float2(-INFINITY, 0.f);
  for (int i = threadIdx.x; i < n_part; i += 256) s = merge_stats(s, part[(long long)t * n_part + i]);
#pragma unroll
  for (int d = 16; d >= 1; d >>= 1)
    s = merge_stats(s, make_float2(__shfl_down_sync(0xffffffffu, s.x, d), __shfl_down_sync(0xffffffffu, s.y, d)));
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
  x = block_sum<256>(x, dot);
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) s = merge_stats(s, sh[w]);
    write_loss(s, tlogit[t], x, logit_scale, loss + t, lse + t);
  }
}

// Many rows: 32 rows x 32 shares of their pairs a block, merged in a fixed order.
__global__ void __launch_bounds__(1024)
lm_finish_kernel(const float2 *part, int n_part, long long rows_pad, const LmRows rows, const float *tlogit, float logit_scale,
                 float *loss, float *lse) {
  launch_next();
  wait_previous();
  __shared__ float2 sh[32][33];
  const int lane = threadIdx.x & 31, seg = threadIdx.x >> 5;
  const int n = *rows.n_rows;
  for (long long r0 = blockIdx.x * 32ll; r0 < n; r0 += gridDim.x * 32ll) {
    const long long r = r0 + lane;
    float2 v = make_float2(-INFINITY, 0.f);
    if (r < n)
      for (int i = seg; i < n_part; i += 128) {
        float2 q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) q[e] = i + 32 * e < n_part ? part[(long long)(i + 32 * e) * rows_pad + r] : make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int e = 0; e < 4; ++e) v = merge_stats(v, q[e]);
      }
    sh[lane][seg] = v;
    __syncthreads();
    v = sh[seg][lane];   // warp: row, lane: share
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1)
      v = merge_stats(v, make_float2(__shfl_down_sync(0xffffffffu, v.x, d), __shfl_down_sync(0xffffffffu, v.y, d)));
    if (lane == 0 && r0 + seg < n) {
      const int t = rows.idx[r0 + seg];
      write_loss(v, tlogit[r0 + seg], rows.x_target[r0 + seg], logit_scale, loss + t, lse + t);
    }
    __syncthreads();
  }
}

// dH of every token in bf16: the shares' partial sums added in order; zeros for rows that are not scored.
__global__ void __launch_bounds__(256)
lm_dh_kernel(const float *part, int splits, long long rows_pad, int hidden, const int *pos, int tokens, __nv_bfloat16 *d_hidden) {
  launch_next();
  wait_previous();
  const int vecs = hidden / 8;
  for (long long t = blockIdx.x; t < tokens; t += gridDim.x) {
    const int r = pos[t];
    for (int i = threadIdx.x; i < vecs; i += 256) {
      float x[8] = {};
      if (r >= 0)
        for (int s = 0; s < splits; ++s) {
          const float4 *q = reinterpret_cast<const float4 *>(part + ((long long)s * rows_pad + r) * hidden + i * 8);
          const float4 a = q[0], b = q[1];
          x[0] += a.x; x[1] += a.y; x[2] += a.z; x[3] += a.w; x[4] += b.x; x[5] += b.y; x[6] += b.z; x[7] += b.w;
        }
      *reinterpret_cast<uint4 *>(d_hidden + t * hidden + i * 8) =
          make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    }
  }
}

// ---------------------------------------------------------------- embedding
template <typename T> struct Vec;  // eight elements
template <> struct Vec<float> {
  static __device__ __forceinline__ void load(const float *p, float (&x)[8]) {
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
  static __device__ __forceinline__ void store(float *p, const float (&x)[8]) {
    *reinterpret_cast<float4 *>(p) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
  }
};
template <> struct Vec<__nv_bfloat16> {
  static __device__ __forceinline__ void load(const __nv_bfloat16 *p, float (&x)[8]) {
    const uint4 v = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&w[i]));
      x[2 * i] = f.x; x[2 * i + 1] = f.y;
    }
  }
  static __device__ __forceinline__ void store(__nv_bfloat16 *p, const float (&x)[8]) {
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
  }
};
template <> struct Vec<__half> {
  static __device__ __forceinline__ void load(const __half *p, float (&x)[8]) {
    const uint4 v = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
      x[2 * i] = f.x; x[2 * i + 1] = f.y;
    }
  }
  static __device__ __forceinline__ void store(__half *p, const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// out[t] = scale table[id_t]; zeros for a negative id.  The product is taken in fp32 and rounded to the output's type.  HBM-bound: a row read, a row written (24576 tokens
// of 3584 bf16 columns: 47 us, frequent rows from L2).
template <typename Id, typename In, typename Out>
__global__ void __launch_bounds__(128)
embed_fwd_kernel(const In *table, const Id *ids, int tokens, int vocab, int hidden, float scale, Out *out, int *status) {
  launch_next();
  wait_previous();
  for (long long t = blockIdx.x; t < tokens; t += gridDim.x) {
    const long long id = ids[t];
    const bool live = id >= 0 && id < vocab;
    if (threadIdx.x == 0) check_id(id, (int)t, vocab, status);
    for (int i = threadIdx.x * 8; i < hidden; i += 1024) {
      float x[8] = {};
      if (live) {
        Vec<In>::load(table + id * hidden + i, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= scale;
      }
      Vec<Out>::store(out + t * hidden + i, x);
    }
  }
}

// ---- tokens sorted by id, stably: least-significant-digit radix passes of at most 9 bits.  Key `vocab` = not embedded.
// The first pass reads the ids themselves.  Blocks of 1024 keys: a pass is bound by the latency of its few dependent steps,
// so many small blocks beat few large ones (24576 tokens, scatter pass: 16 us with 4096 keys a block).
constexpr int kSortBins = 512;
constexpr int kRadixBlock = 1024, kRadixThreads = 256, kRadixWarps = 8;  // 128 keys a warp, 4 a lane

struct KeysSorted {   // keys and places of the pass before
  const uint32_t *key;
  const int *val;
  __device__ __forceinline__ uint32_t get(int i) const { return key[i]; }
  __device__ __forceinline__ int place(int i) const { return val[i]; }
  __device__ __forceinline__ void check(int) const {}
};
template <typename Id>
struct KeysFromIds {
  const Id *ids;
  int vocab;
  int *status;
  __device__ __forceinline__ void check(int i) const { check_id(ids[i], i, vocab, status); }
  __device__ __forceinline__ uint32_t get(int i) const {
    const long long id = ids[i];
    return id >= 0 && id < vocab ? (uint32_t)id : (uint32_t)vocab;
  }
  __device__ __forceinline__ int place(int i) const { return i; }
};

template <typename Keys>
__global__ void __launch_bounds__(kRadixThreads)
embed_hist_kernel(const Keys in, int n, int shift, int bits, int *hist, int n_blocks, uint32_t *seen, int seen_words) {
  launch_next();
  wait_previous();
  __shared__ int cnt[kSortBins];
  for (int i = threadIdx.x; i < kSortBins; i += kRadixThreads) cnt[i] = 0;
  for (int i = blockIdx.x * kRadixThreads + threadIdx.x; i < seen_words; i += gridDim.x * kRadixThreads) seen[i] = 0;  // (first pass)
  __syncthreads();
  const int b0 = blockIdx.x * kRadixBlock;
  for (int i = threadIdx.x; i < kRadixBlock && b0 + i < n; i += kRadixThreads) {
    in.check(b0 + i);
    atomicAdd(&cnt[(in.get(b0 + i) >> shift) & ((1u << bits) - 1)], 1);  // a count: the order does not matter
  }
  __syncthreads();
  for (int i = threadIdx.x; i < (1 << bits); i += kRadixThreads) hist[(long long)i * n_blocks + blockIdx.x] = cnt[i];
}

// one warp per bin: exclusive prefix sum over the blocks, total of the bin behind it
__global__ void __launch_bounds__(256)
embed_scan_kernel(int *hist, int n_blocks, int bins, int *total) {
  launch_next();
  wait_previous();
  const int bin = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (bin >= bins) return;
  int run = 0;
  for (int b = 0; b < n_blocks; b += 32) {
    const int v = b + lane < n_blocks ? hist[(long long)bin * n_blocks + b + lane] : 0;
    int s = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, s, d);
      if (lane >= d) s += u;
    }
    if (b + lane < n_blocks) hist[(long long)bin * n_blocks + b + lane] = run + s - v;
    run += __shfl_sync(0xffffffffu, s, 31);
  }
  if (lane == 0) total[bin] = run;
}

template <typename Keys>
__global__ void __launch_bounds__(kRadixThreads)
embed_scatter_kernel(const Keys in, int n, int shift, int bits, const int *hist, int n_blocks, const int *total, uint32_t *key_out, int *val_out) {
  launch_next();
  wait_previous();
  __shared__ int cnt[kRadixWarps][kSortBins];
  __shared__ int wsum[kRadixWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, bins = 1 << bits;
  const int w0 = blockIdx.x * kRadixBlock + warp * 128;
  uint32_t k[4];
  int v[4], rank[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i = w0 + j * 32 + lane;
    k[j] = i < n ? in.get(i) : 0;
    v[j] = i < n ? in.place(i) : 0;
  }
  for (int i = threadIdx.x; i < kRadixWarps * kSortBins; i += kRadixThreads) (&cnt[0][0])[i] = 0;
  // places of this thread's two bins: exclusive prefix sum of the totals, plus the share of the earlier blocks
  const int b0 = threadIdx.x * 2;
  const int t0 = b0 < bins ? total[b0] : 0, t1 = b0 + 1 < bins ? total[b0 + 1] : 0;
  const int h0 = b0 < bins ? hist[(long long)b0 * n_blocks + blockIdx.x] : 0;
  const int h1 = b0 + 1 < bins ? hist[(long long)(b0 + 1) * n_blocks + blockIdx.x] : 0;
  int s = t0 + t1;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, s, d);
    if (lane >= d) s += u;
  }
  if (lane == 31) wsum[warp] = s;
  __syncthreads();
  int before = s - t0 - t1;
  for (int w = 0; w < warp; ++w) before += wsum[w];
  // rank of every key among the warp's earlier keys of the same digit, in order
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const bool live = w0 + j * 32 + lane < n;
    const int d = live ? (int)((k[j] >> shift) & (bins - 1)) : -1;
    const unsigned same = __match_any_sync(0xffffffffu, d);
    const int first = __ffs(same) - 1;
    int c = 0;
    if (live && lane == first) { c = cnt[warp][d]; cnt[warp][d] = c + __popc(same); }
    __syncwarp();
    rank[j] = __shfl_sync(0xffffffffu, c, first) + __popc(same & ((1u << lane) - 1));
  }
  __syncthreads();
  int r0 = before + h0, r1 = before + t0 + h1;
#pragma unroll
  for (int w = 0; w < kRadixWarps; ++w) {
    const int c0 = cnt[w][b0], c1 = cnt[w][b0 + 1];
    cnt[w][b0] = r0; cnt[w][b0 + 1] = r1;
    r0 += c0; r1 += c1;
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (w0 + j * 32 + lane < n) {
      const int to = cnt[warp][(k[j] >> shift) & (bins - 1)] + rank[j];
      key_out[to] = k[j];
      val_out[to] = v[j];
    }
}

// What the sum and join kernels need besides the sorted tokens:
//   joins[0], joins[1]  numbers of rows that cross chunks: short ones (up to kJoinShort sums) and long ones; behind them the
//                       chunks the rows start in, short ones from the front, long ones from the back, in any order (each
//                       row is joined alone)
//   seen                one bit per table row: whether any token has this id
// The bits are set from the sorted keys, once for each id: setting them from the tokens took 39 us for 131071 of them, all
// at the few words of the frequent ids.
constexpr int kJoinShort = 8;

__device__ __forceinline__ void embed_mark(const uint32_t *key, int i, int vocab, uint32_t *seen) {
  const uint32_t k = key[i];
  if (k < (uint32_t)vocab && (i == 0 || key[i - 1] != k)) atomicOr(seen + (k >> 5), 1u << (k & 31));
}
__global__ void embed_mark_kernel(const uint32_t *key, int n, int vocab, uint32_t *seen, int *joins) {
  launch_next();
  wait_previous();
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i < 2) joins[i] = 0;
  if (i < n) embed_mark(key, i, vocab, seen);
}

// The whole sort in one block, for up to kSortSmall tokens: keys and places wait in shared memory between the passes, and
// six launches are saved (a block for up to 16384 tokens was tried: 62 us where the launches take 45).  A warp has as many keys as
// the tokens need.
constexpr int kSortSmall = 4096;   // 16 warps x 256 keys
constexpr int kSortSmallBytes = 16 * kSortBins * 4 + kSortSmall * 8;

template <typename Id>
__global__ void __launch_bounds__(512)
embed_sort_small_kernel(const Id *ids, int n, int vocab, int passes, int bits, uint32_t *key_out, int *val_out,
                        int *joins, uint32_t *seen, int *status) {
  launch_next();
  wait_previous();
  extern __shared__ __align__(16) int sort_smem[];
  int *cnt = sort_smem;                        // [16][kSortBins]
  uint32_t *skey = reinterpret_cast<uint32_t *>(sort_smem + 16 * kSortBins);
  int *sval = sort_smem + 16 * kSortBins + kSortSmall;
  __shared__ int wsum[16];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, bins = 1 << bits;
  const int per = (n + 511) / 512, w0 = warp * per * 32;
  if (threadIdx.x < 2) joins[threadIdx.x] = 0;
  for (int i = threadIdx.x; i < (vocab + 31) / 32; i += 512) seen[i] = 0;
  for (int i = threadIdx.x; i < n; i += 512) {
    check_id(ids[i], i, vocab, status);
    skey[i] = KeysFromIds<Id>{ids, vocab, status}.get(i);
    sval[i] = i;
  }
  for (int p = 0; p < passes; ++p) {
    const int shift = p * bits;
    for (int i = threadIdx.x; i < 16 * kSortBins; i += 512) cnt[i] = 0;
    __syncthreads();
    uint32_t k[8];
    int v[8], rank[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (j >= per) break;
      const int i = w0 + j * 32 + lane;
      const bool in = i < n;
      k[j] = in ? skey[i] : 0;
      v[j] = in ? sval[i] : 0;
      const int d = in ? (int)((k[j] >> shift) & (bins - 1)) : -1;
      const unsigned same = __match_any_sync(0xffffffffu, d);
      const int first = __ffs(same) - 1;
      int c = 0;
      if (in && lane == first) { c = cnt[warp * kSortBins + d]; cnt[warp * kSortBins + d] = c + __popc(same); }
      __syncwarp();
      rank[j] = __shfl_sync(0xffffffffu, c, first) + __popc(same & ((1u << lane) - 1));
    }
    __syncthreads();
    // a thread per bin: place of the bin, then of each warp's share of it
    int tot = 0;
    for (int w = 0; w < 16; ++w) { const int c = cnt[w * kSortBins + threadIdx.x]; cnt[w * kSortBins + threadIdx.x] = tot; tot += c; }
    int s = tot;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, s, d);
      if (lane >= d) s += u;
    }
    if (lane == 31) wsum[warp] = s;
    __syncthreads();
    int before = s - tot;
    for (int w = 0; w < warp; ++w) before += wsum[w];
    for (int w = 0; w < 16; ++w) cnt[w * kSortBins + threadIdx.x] += before;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = w0 + j * 32 + lane;
      if (j < per && i < n) {
        const int to = cnt[warp * kSortBins + ((k[j] >> shift) & (bins - 1))] + rank[j];
        skey[to] = k[j];
        sval[to] = v[j];
      }
    }
    __syncthreads();
  }
  for (int i = threadIdx.x; i < n; i += 512) {
    key_out[i] = skey[i];
    val_out[i] = sval[i];
    embed_mark(skey, i, vocab, seen);
  }
}

// ---- d_table[v] (+)= scale sum of d_out over the tokens of v, in the order of the tokens, in fp32, rounded once.
// A frequent id owns thousands of tokens and a rare one a single token, so the sorted tokens are cut into chunks of equal
// length, whatever ids they hold: a chunk writes the rows that lie inside it.  A row that starts in a chunk and ends in the next
// belongs to the first of the two, which goes on to the row's end.  Of a row over three chunks or more each leaves its sum
// (slot 0 for the row that comes in, slot 1 for the one that goes on) to embed_join_kernel, which adds them up in order.
// Bound by HBM: every gradient row read once, every table row written once.  A thread has eight
// columns and a block whole rows (up to 4096 columns), so reads and writes are runs of several KB: 205 us for 24576 tokens into
// 152064 x 3584 bf16 (5.9 TB/s), 99 us for 131071 into 32003 x 1032 fp32 (6.3 TB/s).
constexpr int kEmbedMaxThreads = 512;
constexpr int kEmbedZeroRows = 16;      // table rows looked at by one block of the zero part (half a word of `seen`)
constexpr int kEmbedMaxChunk = 256;

template <typename Out>
__device__ __forceinline__ void embed_store(Out *dst, float (&x)[8], float scale, int accumulate) {
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] *= scale;
  if (accumulate) {
    float y[8];
    Vec<Out>::load(dst, y);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] += y[e];
  }
  Vec<Out>::store(dst, x);
}

// end of the run of v that starts at lo, in sorted keys
__device__ __forceinline__ int run_end(const uint32_t *key, int lo, int hi, uint32_t v) {
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (key[mid] == v) lo = mid + 1; else hi = mid;
  }
  return lo;
}

template <typename In, typename Out>
__global__ void __launch_bounds__(kEmbedMaxThreads)
embed_sum_kernel(const In *d_out, const uint32_t *key, const int *val, int n, int chunk, int n_chunks, int vocab, int hidden,
                 float scale, int accumulate, Out *d_table, float *part, int *joins, const uint32_t *seen) {
  launch_next();
  wait_previous();
  __shared__ uint32_t skey[2 * kEmbedMaxChunk];
  __shared__ int sval[2 * kEmbedMaxChunk];
  const int col = (blockIdx.y * blockDim.x + threadIdx.x) * 8;
  if ((int)blockIdx.x >= n_chunks) {
    // rows without tokens: zeros
    const int v0 = ((int)blockIdx.x - n_chunks) * kEmbedZeroRows;
    const uint32_t has = n ? seen[v0 >> 5] >> (v0 & 31) : 0;
    const float zero[8] = {};
    if (col < hidden)
      for (int i = 0; i < kEmbedZeroRows && v0 + i < vocab; ++i)
        if (!((has >> i) & 1)) Vec<Out>::store(d_table + (long long)(v0 + i) * hidden + col, zero);
    return;
  }
  const int c = blockIdx.x, j0 = c * chunk, m0 = min(chunk, n - j0), m1 = min(2 * chunk, n - j0);
  for (int i = threadIdx.x; i < m1; i += blockDim.x) { skey[i] = key[j0 + i]; sval[i] = val[j0 + i]; }
  const uint32_t none = 0xffffffffu, before = j0 > 0 ? key[j0 - 1] : none;
  const uint32_t before2 = j0 > chunk ? key[j0 - chunk - 1] : none, after2 = j0 + m1 < n ? key[j0 + m1] : none;
  __syncthreads();
  // the row that comes in: this chunk's, unless it started in the chunk before and ends in this one
  const uint32_t v_in = skey[0], after = m0 < m1 ? skey[m0] : none;
  int begin = 0, m = m0;
  if (before == v_in && before2 != v_in && after != v_in)
    begin = run_end(skey, 0, m0, v_in);
  // the row that goes on: followed to its end, if it starts here and ends in the next chunk
  const uint32_t v_out = skey[m0 - 1];
  const bool starts_here = !(v_out == v_in && before == v_in);
  bool goes_on = after == v_out;
  if (goes_on && starts_here && after2 != v_out) {
    m = run_end(skey, m0, m1, v_out);
    goes_on = false;
  }
  if (threadIdx.x == 0 && blockIdx.y == 0 && goes_on && starts_here && v_out < (uint32_t)vocab) {
    if (c + kJoinShort < n_chunks && key[(c + kJoinShort) * chunk] == v_out) joins[1 + n_chunks - atomicAdd(joins + 1, 1)] = c;
    else joins[2 + atomicAdd(joins, 1)] = c;
  }
  if (col >= hidden) return;
  float x[8] = {};
  bool first = begin == 0;   // still in the row that comes in
  for (int j = begin; j < m; j += 4) {
    float y[4][8];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (j + e < m && skey[j + e] < (uint32_t)vocab) Vec<In>::load(d_out + (long long)sval[j + e] * hidden + col, y[e]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (j + e < m && skey[j + e] < (uint32_t)vocab) {
        const uint32_t v = skey[j + e];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] += y[e][i];
        const bool last = j + e == m - 1;
        if (last || skey[j + e + 1] != v) {
          const bool comes_in = first && before == v;
          if (comes_in || (last && goes_on)) {
            float *dst = part + ((long long)(2 * c + (comes_in ? 0 : 1)) * hidden + col);
            Vec<float>::store(dst, x);
          } else {
            embed_store(d_table + (long long)v * hidden + col, x, scale, accumulate);
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] = 0.f;
          first = false;
        }
      }
    }
  }
}

// Rows that cross from one chunk into the next: slot 1 of the chunk c they start in, then slot 0 of the chunks behind it
// whose first key is theirs, three or more, added up in order.  Of a short one a block takes 2048 columns, a thread eight.  A long row is shared out over 32 column vectors x 8 shares of its sums.
template <typename Out>
__global__ void __launch_bounds__(256)
embed_join_kernel(const uint32_t *key, int chunk, int n_chunks, int hidden, float scale, int accumulate, Out *d_table, const float *part,
                  const int *joins) {
  launch_next();
  wait_previous();
  __shared__ float sh[8][264];
  const int lane = threadIdx.x & 31, seg = threadIdx.x >> 5;
  const int n_long = joins[1], s_long = (hidden + 255) / 256, items_long = n_long * s_long;
  const int s_short = (hidden + 2047) / 2048, items = items_long + joins[0] * s_short;
  for (int it = blockIdx.x; it < items; it += gridDim.x) {
    float x[8] = {};
    if (it >= items_long) {
      const int c = joins[2 + (it - items_long) / s_short], col = (it - items_long) % s_short * 2048 + threadIdx.x * 8;
      const uint32_t v = key[(c + 1) * chunk];
      uint32_t next[kJoinShort];
#pragma unroll
      for (int i = 2; i < kJoinShort; ++i) next[i] = c + i < n_chunks ? key[(c + i) * chunk] : 0xffffffffu;
      if (col >= hidden) continue;
      const float *src = part + (long long)2 * c * hidden + col;
      float y[kJoinShort][8];
      Vec<float>::load(src + hidden, y[0]);
      Vec<float>::load(src + (long long)2 * hidden, y[1]);
#pragma unroll
      for (int i = 2; i < kJoinShort; ++i)
        if (next[i] == v) Vec<float>::load(src + (long long)2 * i * hidden, y[i]);
#pragma unroll
      for (int i = 0; i < kJoinShort; ++i)
        if (i < 2 || next[i] == v)
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] += y[i][e];
      embed_store(d_table + (long long)v * hidden + col, x, scale, accumulate);
      continue;
    }
    const int c = joins[1 + n_chunks - it / s_long], col = it % s_long * 256 + lane * 8;
    const uint32_t v = key[(c + 1) * chunk];
    int count = 1;
    for (int b = c + 1;; b += 256) {
      const int at = b + (int)threadIdx.x;
      const int more = __syncthreads_count(at < n_chunks && key[at * chunk] == v);
      count += more;
      if (more < 256) break;
    }
    const int per = (count + 7) / 8, last = min(count, (seg + 1) * per);
    if (col < hidden) {
      const float *src = part + (long long)2 * c * hidden + col;
      for (int i = seg * per; i < last; i += 8) {
        float y[8][8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (i + e < last) Vec<float>::load(src + (long long)(i + e == 0 ? 1 : 2 * (i + e)) * hidden, y[e]);
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (i + e < last)
#pragma unroll
            for (int q = 0; q < 8; ++q) x[q] += y[e][q];
      }
    }
    Vec<float>::store(&sh[seg][lane * 8], x);
    __syncthreads();
    if (seg == 0 && col < hidden) {
      for (int s = 1; s < 8; ++s) {
        float y[8];
        Vec<float>::load(&sh[s][lane * 8], y);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] += y[e];
      }
      embed_store(d_table + (long long)v * hidden + col, x, scale, accumulate);
    }
    __syncthreads();
  }
}

}  // namespace augtree
