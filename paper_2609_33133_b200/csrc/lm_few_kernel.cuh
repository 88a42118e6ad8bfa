// The products of the vocabulary loss for few rows (up to 128): the work is reading W once, so the roles of the operands
// are turned round.  W's rows (or, for dH, its columns) fill the tensor core's M = 128 and the tokens its N, the next multiple of 16:
// the MMAs and the loads of H or G cost what the tokens need, and a persistent CTA per SM streams its share of W through a ring of
// as many stages as fit.  (N = 128 for 77 rows left 6 stages, 96 KB of W in flight an SM, and 220 us where 180 is the
// memory's; HBM's latency at its full rate wants more.)
//
//   STATS  x^T = W H^T, a tile of 128 vocabulary rows; a TMEM lane is a vocabulary row, a column a token.  Maxima and sums over
//          the vocabulary run across the lanes (halving exchanges: 31 shuffles leave lane j with column j's) and stay in
//          registers over all tiles of the CTA; one (m, l) pair a warp and token is left at the end.  The contraction is cut into
//          as many accumulators as fit, added up with rounding: the tensor core's own additions drop what does not fit, always
//          towards zero, in proportion to the length of the chain.  (One row at hidden 3584, worst relative error of the loss over
//          six inputs: 7.0e-7 with 16, 1.2e-6 with four, 8.0e-7 of the plain fp32 form; the time is the same, 186 us.)
//   GRAD   G, rounded to bf16 twice: G = hi + lo, lo = bf16(G - hi), so that the few rows' gradients, in which single elements of
//          G dominate, carry no rounding of G (2^-17 is left).  hi is row t of the scratch, lo row N + t.
//   DH     dH^T = W^T G^T, 256 hidden columns (two MMAs that share G's load) x [hi | lo] of the tokens, a share of the vocabulary each
// Bound by HBM: W is read once by each of the three.  152064 x 3584 (1.09 GB): STATS of one row 165-180 us (6.1-6.6 TB/s), of 77 rows 207,
// GRAD of 77 rows 195, DH 170.  (Tokens on M, with 256-row tiles of CTA pairs, took 189 and 204 us for STATS and GRAD of one
// row, 38 us more for the 1188 partial sums a row that they leave, and 1000 us for dH and dW of 77.)
//
// Roles (192 threads): warps 0-3 epilogue, warp 4 TMA loads, warp 5 MMAs; two accumulators of up to 256 columns.
#pragma once
#include <cuda.h>

#include "lm_tile_kernel.cuh"

namespace augtree {

enum : int { WAIT_FEW_FULL = 84, WAIT_FEW_EMPTY = 85, WAIT_FEW_ACC_FULL = 86, WAIT_FEW_ACC_EMPTY = 87 };

constexpr int kLmFew = 128;       // most rows
constexpr int kFewThreads = 192;

struct FewParams {
  const int *n_rows;              // GRAD, DH: packed rows (device)
  const void *ids;                // STATS: the targets themselves, [tokens]; the rows are not packed, a row is only its column
  int id_bytes, tokens;
  int v0, n, vocab, hidden;       // first vocabulary row of the piece, its rows; whole sizes
  int splits;                     // DH: shares of the piece
  float scale_log2;
  const int *target;              // GRAD: [N]
  const float *lse2, *gscale, *gtarget;  // GRAD: [N]
  float2 *part;                   // STATS: [N][4 gridDim.x]
  float *tlogit;                  // STATS: [N]
  __nv_bfloat16 *grad;            // GRAD: [2 N][ld_grad]
  long long ld_grad;
  float *dh_part;                 // DH: [splits][N][hidden]
  int dh_add;
  int mn_chunks;                  // DH: 64-column chunks in a box of the map of W
  int *status;
  long long wait_budget;
  int test_flags;
};

template <int KIND, int N>
struct FewSmem {
  static constexpr int kSub = KIND == LM_DH ? 2 : 1;          // tiles of 128 rows of A that share a load of B
  static constexpr int kBRows = KIND == LM_DH ? 2 * N : N;
  static constexpr int kABytes = kSub * 128 * 128, kBBytes = kBRows * 128;
  static constexpr int kStageBytes = kABytes + kBBytes;
  static constexpr int kStages = (220 * 1024) / kStageBytes;  // 3 (DH, N = 128) .. 12
  static constexpr int kOffRows = kStages * kStageBytes;      // target, lse2, gscale, gtarget
  static constexpr int kOffBar = kOffRows + 4 * kLmFew * 4;
  static constexpr int kBytes = kOffBar + 256;
  static_assert(kStages >= 3 && kStages <= 12 && kBytes <= 227 * 1024, "stage ring");
};

// Reduces W columns over the 32 lanes of a warp: lane j ends up with column j % W.  Halving exchanges: each step a lane gives
// away the half of its columns that belongs to its partner.
template <int W, class Op>
__device__ __forceinline__ float reduce_columns(float (&a)[W], int lane, Op op) {
#pragma unroll
  for (int h = W / 2; h >= 1; h /= 2) {
    const bool up = lane & h;
#pragma unroll
    for (int i = 0; i < h; ++i) {
      const float give = up ? a[i] : a[i + h], keep = up ? a[i + h] : a[i];
      a[i] = op(keep, __shfl_xor_sync(0xffffffffu, give, h));
    }
  }
  if constexpr (W == 16) a[0] = op(a[0], __shfl_xor_sync(0xffffffffu, a[0], 16));
  return a[0];
}

template <int W>
__device__ __forceinline__ void tmem_ld_cols(uint32_t taddr, uint32_t (&r)[W]) {
  if constexpr (W == 32) tmem_ld32(taddr, r);
  else tmem_ld16(taddr, r);
}

// Units of the kernel: vocabulary tiles (STATS, GRAD), or (share, hidden tile) pairs (DH).
template <int KIND>
__device__ __forceinline__ int few_units(const FewParams &p) {
  return KIND == LM_DH ? (p.hidden + 255) / 256 * p.splits : (p.n + 127) / 128;
}
template <int KIND>
__device__ __forceinline__ void few_unit(const FewParams &p, int u, int &tile, int &split, int &kb0, int &nkb) {
  if (KIND != LM_DH) { tile = u; split = 0; kb0 = 0; nkb = (p.hidden + 63) / 64; return; }
  const int tiles = (p.hidden + 255) / 256, kb = (p.n + 63) / 64;
  split = u / tiles;
  tile = u % tiles;
  kb0 = (int)((long long)kb * split / p.splits);
  nkb = (int)((long long)kb * (split + 1) / p.splits) - kb0;
}

// The accumulator that step kb of a contraction goes to.  With fewer steps than accumulators each step has its own, from 0 up.
__device__ __forceinline__ int few_part(int kb, int nkb, int n_acc) { return nkb <= n_acc ? kb : kb * n_acc / nkb; }

template <int KIND, int N>
__global__ void __launch_bounds__(kFewThreads, 1)
lm_few_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_b, const FewParams p) {
  using SM = FewSmem<KIND, N>;
  constexpr int NST = SM::kStages;
  constexpr int W = N % 32 ? 16 : 32, NG = N / W;   // columns of a group, groups
  constexpr int NACC = KIND == LM_STATS ? 256 / N : 1;  // accumulators of a tile, N columns each
  constexpr int NSUB = SM::kSub, NBUF = KIND == LM_DH ? 1 : 2;  // DH: two tiles of 2 N columns, a unit or two a CTA
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t base = smem_u32(smem_raw);
  launch_next();
  if (base & 1023u) {
    if (threadIdx.x == 0 && atomicCAS(p.status, 0, -6) == 0) p.status[1] = 5;
    return;
  }
  const uint32_t bars = base + SM::kOffBar;
  const uint32_t bar_full = bars, bar_empty = bars + 96;                  // [NST <= 12]
  const uint32_t bar_acc_full = bars + 192, bar_acc_empty = bars + 208;   // [2]
  volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(smem_raw + SM::kOffBar + 224);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(smem_raw + SM::kOffBar + 232);
  int *s_target = reinterpret_cast<int *>(smem_raw + SM::kOffRows);
  float *s_lse2 = reinterpret_cast<float *>(s_target + kLmFew), *s_gscale = s_lse2 + kLmFew, *s_gtarget = s_gscale + kLmFew;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < NST; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(bar_acc_full + 8 * s, 1); mbar_init(bar_acc_empty + 8 * s, 4); }
    *abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 5) { tmem_alloc(smem_u32((const void *)tmem_slot), 512); tmem_relinquish(); }
  if (warp == 4 && lane == 0) { tma_prefetch_desc(&tm_w); tma_prefetch_desc(&tm_b); }
  wait_previous();
  const int n_rows = KIND == LM_STATS ? p.tokens : *reinterpret_cast<const volatile int *>(p.n_rows);
  if (KIND != LM_DH && threadIdx.x < N) {
    const int t = threadIdx.x;
    const bool live = t < n_rows;
    if (KIND == LM_STATS) {
      const long long id = !live ? -1 : p.id_bytes == 8 ? static_cast<const long long *>(p.ids)[t] : static_cast<const int *>(p.ids)[t];
      s_target[t] = id >= 0 && id < p.vocab ? (int)id : -1;
    } else {
      s_target[t] = live ? p.target[t] : -1;
      s_lse2[t] = live ? p.lse2[t] : 0.f;
      s_gscale[t] = live ? p.gscale[t] : 0.f;
      s_gtarget[t] = live ? p.gtarget[t] : 0.f;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const AbortCtx ab{abort_flag, p.status, p.wait_budget};
  const int units = few_units<KIND>(p);
  int tile, split, kb0, nkb;

  if (warp == 4) {
    // ------------------------------------------------------------ TMA producer
    if (lane == 0) {
      uint32_t T = 0;
      bool ok = true;
      for (int u = blockIdx.x; ok && u < units; u += gridDim.x) {
        few_unit<KIND>(p, u, tile, split, kb0, nkb);
        for (int kb = kb0; kb < kb0 + nkb && ok; ++kb, ++T) {
          const uint32_t st = T % NST, bar = bar_full + 8 * st;
          ok = mbar_wait(bar_empty + 8 * st, ((T / NST) & 1) ^ 1, ab, WAIT_FEW_EMPTY);
          if (!ok) break;
          const uint32_t sA = base + st * SM::kStageBytes, sB = sA + SM::kABytes;
          if ((p.test_flags & TEST_SKIP_FWD_LOAD) && blockIdx.x == 0 && T == 0) continue;
          mbar_expect_tx(bar, SM::kStageBytes);
          if (KIND == LM_DH) {
            const int k0 = tile * 256, vr = p.v0 + kb * 64;
            if (p.mn_chunks == 2) for (int b = 0; b < 2; ++b) tma_load_3d(sA + b * 16384, &tm_w, bar, 0, vr, (k0 >> 6) + 2 * b);
            else for (int b = 0; b < 4; ++b) tma_load_3d(sA + b * 8192, &tm_w, bar, k0 + b * 64, vr, 0);
          } else {
            tma_load_2d(sA, &tm_w, bar, kb * 64, p.v0 + tile * 128);
          }
          tma_load_2d(sB, &tm_b, bar, kb * 64, 0);
        }
      }
    }
  } else if (warp == 5) {
    // -------------------------------------------------------------- MMA issuer
    constexpr int kAMn = KIND == LM_DH;
    constexpr uint32_t kIdesc = make_idesc(128, SM::kBRows, kAMn, 0);
    constexpr uint32_t kAStep = kAMn ? 2048 >> 4 : 32 >> 4;
    const bool elected = elect_one();
    uint32_t T = 0, ic = 0;
    bool ok = true;
    for (int u = blockIdx.x; ok && u < units; u += gridDim.x, ++ic) {
      few_unit<KIND>(p, u, tile, split, kb0, nkb);
      const uint32_t buf = ic % NBUF;
      if (ic >= NBUF) {
        ok = mbar_wait(bar_acc_empty + 8 * buf, (ic / NBUF - 1) & 1, ab, WAIT_FEW_ACC_EMPTY);
        if (!ok) break;
        tc_fence_after();
      }
      for (int kb = 0; kb < nkb && ok; ++kb, ++T) {
        const uint32_t st = T % NST;
        ok = mbar_wait(bar_full + 8 * st, (T / NST) & 1, ab, WAIT_FEW_FULL);
        if (!ok) break;
        tc_fence_after();
        const uint32_t sA = base + st * SM::kStageBytes;
        const uint32_t a_lo = sdesc_lo(sA, 8192), b_lo = sdesc_lo(sA + SM::kABytes, 8192);
        const int part = few_part(kb, nkb, NACC);
        const bool fresh = kb == 0 || few_part(kb - 1, nkb, NACC) != part;
        const uint32_t tD = tmem + buf * 256 + part * N;
        if (elected) {
#pragma unroll
          for (int s = 0; s < NSUB; ++s)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              mma_ss2(tD + s * 256, a_lo + s * (16384 >> 4) + k * kAStep, b_lo + k * 2, kIdesc, (uint32_t)(!fresh || k > 0));
          tc_commit(bar_empty + 8 * st);
        }
      }
      if (!ok) break;
      if (elected) tc_commit(bar_acc_full + 8 * buf);
    }
  } else {
    // ------------------------------------------------------------ epilogue warps 0-3
    const uint32_t lane_off = (uint32_t)(warp * 32) << 16;
    uint32_t ic = 0;
    bool ok = true;
    float m[NG], l[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) { m[g] = -INFINITY; l[g] = 0.f; }
    for (int u = blockIdx.x; ok && u < units; u += gridDim.x, ++ic) {
      few_unit<KIND>(p, u, tile, split, kb0, nkb);
      const uint32_t buf = ic % NBUF, tD = tmem + buf * 256 + lane_off;
      ok = mbar_wait(bar_acc_full + 8 * buf, (ic / NBUF) & 1, ab, WAIT_FEW_ACC_FULL);
      if (!ok) break;
      tc_fence_after();
      const int r = tile * (128 * NSUB) + warp * 32 + lane;   // vocabulary row of the piece, or (first) hidden column
      if (KIND == LM_STATS) {
        const int v = p.v0 + r;
        const bool exists = r < p.n;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          float x[W], a[W];
#pragma unroll
          for (int j = 0; j < W; ++j) x[j] = 0.f;
#pragma unroll
          for (int q = 0; q < NACC; ++q) {
            if (q >= nkb) break;   // (a short contraction fills fewer accumulators)
            uint32_t raw[W];
            tmem_ld_cols(tD + q * N + g * W, raw);
            tc_wait_ld();
#pragma unroll
            for (int j = 0; j < W; ++j) x[j] += __uint_as_float(raw[j]);
          }
#pragma unroll
          for (int j = 0; j < W; ++j) {
            if (exists && s_target[g * W + j] == v) p.tlogit[g * W + j] = x[j];
            x[j] = a[j] = exists ? __fmul_rn(x[j], p.scale_log2) : -INFINITY;  // (write_loss counts on this rounding)
          }
          const float top = reduce_columns(a, lane, [](float s, float t) { return fmaxf(s, t); });
          const float mn = fmaxf(m[g], top), ref = mn == -INFINITY ? 0.f : mn;
          l[g] *= ex2(m[g] - ref);
          m[g] = mn;
#pragma unroll
          for (int j = 0; j < W; ++j) a[j] = ex2(x[j] - __shfl_sync(0xffffffffu, ref, j));
          l[g] += reduce_columns(a, lane, [](float s, float t) { return s + t; });
        }
      } else if (KIND == LM_GRAD) {
        const int v = p.v0 + r;
        const bool exists = r < p.n;
        __nv_bfloat16 *dst = p.grad + r;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          uint32_t raw[W];
          tmem_ld_cols(tD + g * W, raw);
          tc_wait_ld();
#pragma unroll
          for (int j = 0; j < W; ++j) {
            const int t = g * W + j;
            const float pr = ex2(fmaf(__uint_as_float(raw[j]), p.scale_log2, -s_lse2[t]));
            const float d = !(exists && t < n_rows) ? 0.f : s_target[t] == v ? s_gtarget[t] : pr * s_gscale[t];
            const __nv_bfloat16 hi = __float2bfloat16_rn(d);
            dst[t * p.ld_grad] = hi;
            dst[(N + t) * p.ld_grad] = __float2bfloat16_rn(d - __bfloat162float(hi));
          }
        }
      } else {
#pragma unroll
        for (int s = 0; s < NSUB; ++s) {
          const int col = r + s * 128;
          float *dst = p.dh_part + (long long)split * N * p.hidden + col;
#pragma unroll
          for (int g = 0; g < N / 16; ++g) {
            uint32_t hi[16], lo[16];
            tmem_ld16(tD + s * 256 + g * 16, hi);
            tmem_ld16(tD + s * 256 + N + g * 16, lo);
            tc_wait_ld();
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              const int t = g * 16 + j;
              if (t < n_rows && col < p.hidden) {
                float x = nkb ? __uint_as_float(hi[j]) + __uint_as_float(lo[j]) : 0.f;
                if (p.dh_add) x += dst[(long long)t * p.hidden];
                dst[(long long)t * p.hidden] = x;
              }
            }
          }
        }
      }
      tc_fence_before();
      warp_arrive(bar_acc_empty + 8 * buf);
    }
    if (KIND == LM_STATS) {
      const int n_part = 4 * gridDim.x;
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const int t = g * W + lane % W;
        if (lane < W) p.part[(long long)t * n_part + 4 * blockIdx.x + warp] = make_float2(m[g], l[g]);
      }
    }
  }

  __syncwarp();
  if (*abort_flag) {
    const long long t0 = clock64();
    while (clock64() - t0 < 400000) {}
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 5) { tc_fence_after(); tmem_dealloc(tmem, 512); }
}

}  // namespace augtree
