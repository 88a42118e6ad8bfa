// Matrix products of the vocabulary loss, forward and backward: one persistent kernel, four kinds of product.
//
//   x_tv = h_t . W_v                       logits, never stored                          (c: logit scale)
//   STATS  per row t and 128 columns:  m = max of c log2(e) x,  l = sum 2^(c log2(e) x - m),  and x at the target
//   GRAD   G_tv = a_t c (2^(c log2(e) x - lse_t log2(e)) - [v = y_t])     stored in bf16, a piece of the vocabulary
//   DH     dH  = G W      [rows, hidden]   contraction over the piece, fp32 partial sums per share of it
//   DW     dW  = G^T H    [piece, hidden]  contraction over the rows, every row of dW has one owner
//
// All four are the same 256 x 256 output tile of a product C = A B^T with fp32 accumulators in TMEM; they differ in
// which operand has its contraction index contiguous in memory (the tensor core takes either order) and in the epilogue.
// G is rounded to bf16 because the two products that use it take bf16 operands: an error of at most half a step,
// 2^-8 of each element, independent between elements, so its sums stay as exact as the bf16 results they are
// delivered in; the sums themselves, the softmax statistics and the exponent are fp32.
//
// A tile belongs to a pair of CTAs (cluster of two, tcgen05.mma.cta_group::2): each loads 128 rows of A and 128 columns of
// B and gets 128 rows of the result, so 64 KB cross from L2 for every 64 steps of contraction of a 256 x 256 tile; single
// CTAs with 128 x 256 tiles need 96 KB for the same work and took 31.5 ms for loss and gradients of 8192 x 152064 x 3584.
//
// Roles (320 threads a CTA): warps 0-7 epilogue (warp w: TMEM lanes 32 (w % 4).., columns 128 (w / 4)..), warp 8 TMA loads
// (each CTA its own share, all counted on the first CTA's barrier), warp 9 of the first CTA issues the MMAs of both.
// TMEM: two accumulators of 256 columns, so a tile's epilogue runs under the next tile.
#pragma once
#include <cuda.h>

#include "ptx.cuh"

namespace augtree {

enum : int { LM_STATS = 0, LM_GRAD = 1, LM_DH = 2, LM_DW = 3 };
enum : int { WAIT_LM_FULL = 80, WAIT_LM_EMPTY = 81, WAIT_LM_ACC_FULL = 82, WAIT_LM_ACC_EMPTY = 83 };

constexpr int kLmTile = 256;     // tile rows and columns of a CTA pair
constexpr int kLmThreads = 320;
constexpr int kLmMaxJobs = 2;

// One product.  Rows of the compacted token block (their number is known on the device only) take part in every
// kind: as M (STATS, GRAD, DH) or as the contraction (DW).
struct LmJob {
  int kind;
  int m_fixed;     // DW: rows of the piece; other kinds: 0 (M = the token rows)
  int n;           // columns: vocabulary columns of the piece (STATS, GRAD) or hidden (DH, DW)
  int k_fixed;     // contraction length; 0 = the token rows (DW)
  int splits;      // shares of the contraction (DH), 1 otherwise
};

struct LmParams {
  LmJob job[kLmMaxJobs];
  int n_jobs;
  const int *n_rows;        // device: rows that are scored
  int v0, vocab, hidden;    // first vocabulary row of the piece; whole sizes
  int mn_chunks;            // 64-column chunks in a box of tm_h_mn and tm_w_mn: 2, or 1 (hidden not a multiple of 64)
  long long rows_pad;       // leading size of per-row arrays and of the partial sums
  float scale_log2;         // c log2(e)
  const int *target;        // [rows_pad]
  const float *lse2;        // [rows_pad] lse log2(e)
  const float *gscale;      // [rows_pad] a_t c; 0 behind the last row
  float2 *part;             // STATS: [2 x vocabulary tiles][rows_pad] (m, l)
  float *tlogit;            // STATS: [rows_pad] x at the target
  __nv_bfloat16 *grad;      // GRAD out: [rows_pad][ld_grad]
  long long ld_grad;
  float *dh_part;           // DH out: [splits][rows_pad][hidden]
  int dh_add;               // DH: add to what an earlier piece left
  void *dw;                 // DW out: rows v0.. of [vocab, hidden]
  int dw_f32, dw_add;
  int *status;
  long long wait_budget;
  int test_flags;
};

struct LmSmem {
  static constexpr int kABytes = 128 * 128, kBBytes = 128 * 128;  // this CTA's share of a stage
  static constexpr int kStageBytes = kABytes + kBBytes;
  static constexpr int kStages = 7;
  static constexpr int kOffBar = kStages * kStageBytes;
  static constexpr int kBytes = kOffBar + 256;
};

struct LmTileCoord {
  int job, m, n, split, kb0, nkb;
};

// Tile number -> job, tile coordinates and contraction range.  The index that runs fastest is the one whose operand
// is the smaller: the tiles in flight then share the large operand's rows while the small one stays in L2.
__device__ __forceinline__ bool lm_tile(const LmParams &p, int n_rows, int t, LmTileCoord &c) {
  for (int j = 0; j < p.n_jobs; ++j) {
    const LmJob &J = p.job[j];
    const int mt = ((J.m_fixed ? J.m_fixed : n_rows) + kLmTile - 1) / kLmTile;
    const int nt = (J.n + kLmTile - 1) / kLmTile;
    const int kb = ((J.k_fixed ? J.k_fixed : n_rows) + 63) / 64;
    const int count = mt * nt * J.splits;
    if (t < count) {
      c.job = j;
      const int per = (kb + J.splits - 1) / J.splits;
      if (J.kind <= LM_GRAD) { c.m = t % mt; c.n = t / mt; c.split = 0; }
      else { c.split = t / (mt * nt); const int r = t % (mt * nt); c.n = r % nt; c.m = r / nt;
      }
      c.kb0 = min(c.split * per, kb);
      c.nkb = min(per, kb - c.kb0);
      return true;
    }
    t -= count;
  }
  return false;
}

// Tensor maps: H and W with a box of 64 contiguous hidden columns x 128 rows (contraction contiguous) or (_mn, contraction
// along the rows) of two such columns x 64 rows, one box for the 128 rows or columns of a stage: two boxes of half the size
// come in more slowly than the tensor core takes them (530 cycles a stage of 512, one box 453).  G likewise.
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kLmThreads, 1)
lm_tile_kernel(const __grid_constant__ CUtensorMap tm_h, const __grid_constant__ CUtensorMap tm_w,
               const __grid_constant__ CUtensorMap tm_g, const __grid_constant__ CUtensorMap tm_h_mn,
               const __grid_constant__ CUtensorMap tm_w_mn, const __grid_constant__ CUtensorMap tm_g_mn, const LmParams p) {
  using SM = LmSmem;
  constexpr int NST = SM::kStages;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t base = smem_u32(smem_raw);
  if (base & 1023u) {  // the same in both CTAs of a pair
    if (threadIdx.x == 0 && atomicCAS(p.status, 0, -6) == 0) p.status[1] = 4;
    return;
  }
  const uint32_t bars = base + SM::kOffBar;
  const uint32_t bar_full = bars, bar_empty = bars + 64;                  // [NST <= 8]
  const uint32_t bar_acc_full = bars + 128, bar_acc_empty = bars + 144;   // [2]
  volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(smem_raw + SM::kOffBar + 192);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(smem_raw + SM::kOffBar + 200);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < NST; ++s) { mbar_init(bar_full + 8 * s, 1); mbar_init(bar_empty + 8 * s, 1); }
    for (int s = 0; s < 2; ++s) { mbar_init(bar_acc_full + 8 * s, 1); mbar_init(bar_acc_empty + 8 * s, 16); }
    *abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 9) { tmem_alloc_pair(smem_u32((const void *)tmem_slot), 512); tmem_relinquish_pair(); }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t rank = cluster_ctarank();
  const uint32_t tmem = *tmem_slot;
  const AbortCtx ab{abort_flag, p.status, p.wait_budget};
  const int n_rows = __ldg(p.n_rows);
  const int t0 = blockIdx.x >> 1, tstep = gridDim.x >> 1;
  LmTileCoord c;

  if (warp == 8) {
    // ------------------------------------------------------------ TMA producer
    if (lane == 0) {
      uint32_t T = 0;
      bool ok = true;
      for (int t = t0; ok && lm_tile(p, n_rows, t, c); t += tstep) {
        const int kind = p.job[c.job].kind;
        const int m0 = c.m * kLmTile + rank * 128, n0 = c.n * kLmTile + rank * 128;  // this CTA's rows of A, columns of B
        for (int kb = c.kb0; kb < c.kb0 + c.nkb && ok; ++kb, ++T) {
          const uint32_t st = T % NST, bar = map_to_rank(bar_full + 8 * st, 0);
          ok = mbar_wait(bar_empty + 8 * st, ((T / NST) & 1) ^ 1, ab, WAIT_LM_EMPTY);
          if (!ok) break;
          const uint32_t sA = base + st * SM::kStageBytes, sB = sA + SM::kABytes;
          const int k0 = kb * 64;
          if ((p.test_flags & TEST_SKIP_FWD_LOAD) && blockIdx.x == 0 && T == 0) continue;
          if (rank == 0) mbar_expect_tx(bar_full + 8 * st, 2 * SM::kStageBytes);
          if (kind <= LM_GRAD) {
            tma_load_2d_pair(sA, &tm_h, bar, k0, m0);
            tma_load_2d_pair(sB, &tm_w, bar, k0, p.v0 + n0);
          } else {
            const bool dh = kind == LM_DH;
            if (dh) tma_load_2d_pair(sA, &tm_g, bar, k0, m0);
            else tma_load_3d_pair(sA, &tm_g_mn, bar, 0, k0, m0 >> 6);
            const CUtensorMap *tm_b = dh ? &tm_w_mn : &tm_h_mn;
            const int kr = dh ? p.v0 + k0 : k0;
            if (p.mn_chunks == 2) tma_load_3d_pair(sB, tm_b, bar, 0, kr, n0 >> 6);
            else for (int b = 0; b < 2; ++b) tma_load_3d_pair(sB + b * 8192, tm_b, bar, n0 + b * 64, kr, 0);
          }
        }
      }
    }
  } else if (warp == 9) {
   if (rank == 0) {
    // -------------------------------------------------------------- MMA issuer
    const bool elected = elect_one();
    uint32_t T = 0, ic = 0;
    bool ok = true;
    for (int t = t0; ok && lm_tile(p, n_rows, t, c); t += tstep, ++ic) {
      const int kind = p.job[c.job].kind;
      const int a_mn = kind == LM_DW, b_mn = kind >= LM_DH;
      const uint32_t idesc = make_idesc(256, kLmTile, a_mn, b_mn);
      const uint32_t a_step = a_mn ? 2048 >> 4 : 32 >> 4, b_step = b_mn ? 2048 >> 4 : 32 >> 4;
      const uint32_t buf = ic & 1;
      if (ic >= 2) {
        ok = mbar_wait(bar_acc_empty + 8 * buf, ((ic >> 1) - 1) & 1, ab, WAIT_LM_ACC_EMPTY);
        if (!ok) break;
        tc_fence_after();
      }
      const uint32_t tD = tmem + buf * kLmTile;
      for (int kb = 0; kb < c.nkb && ok; ++kb, ++T) {
        const uint32_t st = T % NST;
        ok = mbar_wait(bar_full + 8 * st, (T / NST) & 1, ab, WAIT_LM_FULL);
        if (!ok) break;
        tc_fence_after();
        const uint32_t sA = base + st * SM::kStageBytes;
        const uint32_t a_lo = sdesc_lo(sA, 8192), b_lo = sdesc_lo(sA + SM::kABytes, 8192);
        if (elected) {
#pragma unroll
          for (int k = 0; k < 4; ++k) mma_ss2_pair(tD, a_lo + k * a_step, b_lo + k * b_step, idesc, (uint32_t)(kb > 0 || k > 0));
          tc_commit_pair(bar_empty + 8 * st);
        }
      }
      if (!ok) break;
      if (elected) tc_commit_pair(bar_acc_full + 8 * buf);
    }
   }
  } else {
    // ------------------------------------------------------------ epilogue warps 0-7
    const int r = (warp & 3) * 32 + lane;
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
    const int half = warp >> 2, col0 = half * 128;
    uint32_t ic = 0;
    bool ok = true;
    for (int t = t0; ok && lm_tile(p, n_rows, t, c); t += tstep, ++ic) {
      const LmJob &J = p.job[c.job];
      const uint32_t buf = ic & 1;
      ok = mbar_wait(bar_acc_full + 8 * buf, (ic >> 1) & 1, ab, WAIT_LM_ACC_FULL);
      if (!ok) break;
      tc_fence_after();
      const uint32_t tD = tmem + buf * kLmTile + lane_off + col0;
      const int row = c.m * kLmTile + rank * 128 + r, n0 = c.n * kLmTile + col0;  // tile row, first column of this warp
      if (J.kind == LM_STATS) {
        const int tgt = row < n_rows ? p.target[row] - p.v0 - n0 : -1;  // column of the target, relative
        float m = -INFINITY, l = 0.f, xt = 0.f;
        bool hit = false;
        for (int q = 0; q < 4; ++q) {
          uint32_t v[32];
          tmem_ld32(tD + q * 32, v);
          tc_wait_ld();
          const int left = J.n - (n0 + q * 32);  // columns that exist
          if ((unsigned)(tgt - q * 32) < 32u) {
            hit = true;
#pragma unroll
            for (int e = 0; e < 32; ++e) if (tgt - q * 32 == e) xt = __uint_as_float(v[e]);
          }
          float cm = -INFINITY;
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            const float x = e < left ? __uint_as_float(v[e]) * p.scale_log2 : -INFINITY;
            v[e] = __float_as_uint(x);
            cm = fmaxf(cm, x);
          }
          const float mn = fmaxf(m, cm), ref = mn == -INFINITY ? 0.f : mn;
          l *= ex2(m - ref);
#pragma unroll
          for (int e = 0; e < 32; ++e) l += ex2(__uint_as_float(v[e]) - ref);
          m = mn;
        }
        if (row < n_rows) {
          p.part[(long long)(2 * ((p.v0 / kLmTile) + c.n) + half) * p.rows_pad + row] = make_float2(m, l);
          if (hit) p.tlogit[row] = xt;
        }
      } else if (J.kind == LM_GRAD) {
        const bool live = row < n_rows;
        const int tgt = live ? p.target[row] - p.v0 - n0 : -1;
        const float lse2 = live ? p.lse2[row] : 0.f, gs = live ? p.gscale[row] : 0.f;
        __nv_bfloat16 *dst = p.grad + (long long)row * p.ld_grad + n0;
        for (int q = 0; q < 4; ++q) {
          uint32_t v[32];
          tmem_ld32(tD + q * 32, v);
          tc_wait_ld();
          const int left = J.n - (n0 + q * 32);
          float g[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            const float pr = ex2(fmaf(__uint_as_float(v[e]), p.scale_log2, -lse2)) - (tgt - q * 32 == e ? 1.f : 0.f);
            g[e] = live && e < left ? pr * gs : 0.f;
          }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = pack_bf16(g[16 * e + 2 * i], g[16 * e + 2 * i + 1]);
            st_global_v8(dst + q * 32 + 16 * e, w);
          }
        }
      } else {
        const bool dh = J.kind == LM_DH;
        const bool live = dh ? row < n_rows : row < J.m_fixed;
        const bool f32 = dh || p.dw_f32, add = dh ? p.dh_add : p.dw_add;
        const bool zero = c.nkb == 0;   // an empty contraction: nothing was accumulated
        const long long off = dh ? ((long long)c.split * p.rows_pad + row) * p.hidden + n0
                                 : ((long long)p.v0 + row) * p.hidden + n0;
        for (int q = 0; q < 4; ++q) {
          uint32_t v[32];
          tmem_ld32(tD + q * 32, v);
          tc_wait_ld();
          if (live) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int col = q * 32 + e * 8;
              if (n0 + col < p.hidden) {   // hidden is a multiple of 8
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = zero ? 0.f : __uint_as_float(v[e * 8 + i]);
                if (f32) {
                  float4 *d = reinterpret_cast<float4 *>((dh ? p.dh_part : static_cast<float *>(p.dw)) + off + col);
                  if (add) {
                    const float4 a = d[0], b = d[1];
                    x[0] += a.x; x[1] += a.y; x[2] += a.z; x[3] += a.w; x[4] += b.x; x[5] += b.y; x[6] += b.z; x[7] += b.w;
                  }
                  d[0] = make_float4(x[0], x[1], x[2], x[3]);
                  d[1] = make_float4(x[4], x[5], x[6], x[7]);
                } else {
                  *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p.dw) + off + col) =
                      make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
                }
              }
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(map_to_rank(bar_acc_empty + 8 * buf, 0));
    }
  }

  __syncwarp();
  if (*abort_flag) {
    const long long t0c = clock64();
    while (clock64() - t0c < 400000) {}
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();  // neither CTA leaves, or gives up its half of TMEM, while the other's loads, MMAs or arrivals may reach it
  if (warp == 9) { tc_fence_after(); tmem_dealloc_pair(tmem, 512); }
}

}  // namespace augtree
