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
// G is rounded to bf16 because the two products that use it take bf16 operands: at most half a step, 2^-8 of each element,
// independent between elements.  In the sums that is an error of the size of their own delivery in bf16, which comes on top of it:
// 2.3e-3 to 2.4e-3 of dH and dW (relative L2) where delivery alone leaves 1.66e-3.  The sums themselves, the softmax statistics and
// the exponent are fp32.  With up to 256 rows single elements (the targets') dominate a result and their roundings with it; there G
// is kept in two halves, hi = bf16(G) and lo = bf16(G - hi), and the contractions of dH and dW run over both, which few rows can
// afford (W and dW pass through memory just the same) and leaves 1.66e-3.  With many rows it would double the time of both products.
//
// A tile belongs to a pair of CTAs (cluster of two, tcgen05.mma.cta_group::2): each loads 128 rows of A and 128 columns of
// B and gets 128 rows of the result, so 64 KB cross from L2 for every 64 steps of contraction of a 256 x 256 tile; single
// CTAs with 128 x 256 tiles need 96 KB for the same work and took 31.5 ms for loss and gradients of 8192 x 152064 x 3584.
//
// Roles (320 threads a CTA): warps 0-7 epilogue (warp w: TMEM lanes 32 (w % 4).., columns 128 (w / 4)..), warp 8 TMA loads
// (each CTA its own share, all counted on the first CTA's barrier), warp 9 of the first CTA issues the MMAs of both.
// TMEM: two accumulators of 256 columns, so a tile's epilogue runs under the next tile.  Results leave through shared memory
// and the copy engine, 32 rows x 128 bytes a warp at a time, whole lines: with 16-byte stores, a row per thread, dW of 77
// rows under 152064 x 3584 was bound by the store unit (680 us for 1.1 GB).
//
// Bound by the tensor pipe at the clock that the power cap leaves: 8192 x 30464 x 3584, single launches: STATS 1.08 ms (1658 TFLOP/s,
// 95.5 % tensor-active), GRAD 1.12 ms (93.4 %), DH + DW 2.46 ms (93.8 %); a whole step in a loop 1315 TFLOP/s.
#pragma once
#include <cuda.h>

#include <type_traits>

#include "pair_tile.cuh"

namespace augtree {

enum : int { LM_STATS = 0, LM_GRAD = 1, LM_DH = 2, LM_DW = 3 };
enum : int { WAIT_LM_FULL = 80, WAIT_LM_EMPTY = 81, WAIT_LM_ACC_FULL = 82, WAIT_LM_ACC_EMPTY = 83 };

constexpr int kLmThreads = 320;
constexpr int kLmMaxJobs = 2;

// One product.  Rows of the compacted token block (their number is known on the device only) take part in every
// kind: as M (STATS, GRAD, DH) or as the contraction (DW).
struct LmJob {
  int kind;
  int m_fixed;     // DW: rows of the piece; other kinds: 0 (M = the token rows)
  int n;           // columns: vocabulary columns of the piece (STATS, GRAD) or hidden (DH, DW)
  int k_fixed;     // contraction length; 0 = the token rows (DW).  Empty in any case when no row is scored
  int splits;      // shares of the contraction (DH), 1 otherwise
  int group;       // STATS, GRAD: row tiles that are taken over all columns before the next ones
};

struct LmParams {
  LmJob job[kLmMaxJobs];
  int n_jobs;
  const int *n_rows;        // device: rows that are scored
  int v0, vocab, hidden;    // first vocabulary row of the piece; whole sizes
  int mn_chunks;            // 64-column chunks in a box of tm_w_mn: 2, or 1 (hidden not a multiple of 64)
  long long rows_pad;       // leading size of per-row arrays and of the partial sums
  float scale_log2;         // c log2(e)
  const int *target;        // [rows_pad]
  const float *lse2;        // [rows_pad] lse log2(e)
  const float *gscale;      // [rows_pad] a_t c; like the other arrays of a number per row not set behind the last one
  const float *gtarget;     // [rows_pad] G at the target, from an fp32 logit
  float2 *part;             // STATS: [2 x vocabulary tiles][rows_pad] (m, l)
  float *tlogit;            // STATS: [rows_pad] x at the target
  int halves;               // 2: G is hi in rows 0 .. rows_pad, lo in the rows behind them; 1: hi alone
  __nv_bfloat16 *grad_lo;   // GRAD with two halves: [rows_pad][ld_grad], where lo goes
  long long ld_grad;
  int half_k;               // DH: contraction steps x 64 of one half
  int dh_add;               // DH: add to what an earlier piece left in the partial sums
  int dw_f32, dw_add;       // DW: type of dW, add to what is there
  int *status;
  long long wait_budget;
  int test_flags;
};

struct LmSmem {
  static constexpr int kABytes = 128 * 128, kBBytes = 128 * 128;  // this CTA's share of a stage
  static constexpr int kStageBytes = kABytes + kBBytes;
  static constexpr int kStages = 6;
  static constexpr int kOffOut = kStages * kStageBytes;   // 4 KB a warp on their way out
  static constexpr int kOffBar = kOffOut + 8 * 4096;
  static constexpr int kBytes = kOffBar + 256;
};

// Walks the tiles of one CTA pair: tile t0, t0 + step, .. of all jobs in a row.
//   STATS, GRAD  row tiles run fastest, within a group whose hidden states stay in L2 while W streams past, once a group.  (With
//                all rows of 16384 x 3584 in one group, 117 MB, they come from HBM again for every column of tiles.)
//   DH, DW       hidden columns run fastest: a row of tiles shares its G, which then passes once
// From tile to tile the coordinates move on by additions; divisions are left to the start of a job or group (with them in every
// step each role spent 2400 cycles a tile on finding it, more than a tile of 64 rows takes).
struct LmTile {
  int kind, m, n, split, kb0, nkb;   // product, tile coordinates, share of the contraction: first step, steps
  int cols, m_fixed;                 // of the job
  int t, job, first, end, step;      // tile number, its job, the numbers of the job's or group's tiles
  int m0, rows, mt, nt, kb, per, d_fast, d_slow;

  __device__ __forceinline__ bool start(const LmParams &p, int n_rows, int t0, int tile_step) {
    t = t0; step = tile_step; job = 0; first = 0;
    return enter(p, n_rows);
  }
  // the job and group that hold tile t; `first` is the first tile of `job`
  __device__ __forceinline__ bool enter(const LmParams &p, int n_rows) {
    for (; job < p.n_jobs; ++job) {
      const LmJob J = job == 0 ? p.job[0] : p.job[1];
      kind = J.kind; cols = J.n; m_fixed = J.m_fixed;
      mt = ((J.m_fixed ? J.m_fixed : n_rows) + kLmTile - 1) / kLmTile;
      nt = (J.n + kLmTile - 1) / kLmTile;
      // Without scored rows GRAD has no tiles and G is not written: nothing of it may be read, whatever length the host knows.
      kb = n_rows == 0 ? 0 : ((J.k_fixed ? J.k_fixed : n_rows) + 63) / 64;
      const int count = mt * nt * J.splits;
      if (t < first + count) {
        int r = t - first;
        per = (kb + J.splits - 1) / J.splits;
        if (kind <= LM_GRAD) {
          const int g = r / (J.group * nt);
          m0 = g * J.group;
          rows = min(J.group, mt - m0);
          r -= m0 * nt;
          m = m0 + r % rows; n = r / rows; split = 0;
          end = first + (m0 + rows) * nt;
        } else {
          m0 = 0; rows = nt;
          n = r % nt; m = r / nt; split = m / mt; m -= split * mt;
          end = first + count;
        }
        d_fast = step % rows; d_slow = step / rows;
        range();
        return true;
      }
      first += count;
    }
    return false;
  }
  __device__ __forceinline__ void range() {
    kb0 = min(split * per, kb);
    nkb = min(per, kb - kb0);
  }
  __device__ __forceinline__ bool next(const LmParams &p, int n_rows) {
    t += step;
    if (t >= end) return enter(p, n_rows);
    if (kind <= LM_GRAD) {
      m += d_fast; n += d_slow;
      if (m >= m0 + rows) { m -= rows; ++n; }
    } else {
      n += d_fast; m += d_slow;
      if (n >= nt) { n -= nt; ++m; }
      while (m >= mt) { m -= mt; ++split; }
      range();
    }
    return true;
  }
};

// Tensor maps: H and W with a box of 64 contiguous hidden columns x 128 rows (contraction contiguous) or (_mn, contraction
// along the rows) of two such columns x 64 rows, one box for the 128 rows or columns of a stage: two boxes of half the size
// come in more slowly than the tensor core takes them (530 cycles a stage of 512, one box 453).  G likewise.  tm_out: G (GRAD)
// or dW (DW), tm_dh: the partial sums [splits x rows_pad][hidden]; boxes of 128 bytes x 32 rows.
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kLmThreads, 1)
lm_tile_kernel(const __grid_constant__ CUtensorMap tm_h, const __grid_constant__ CUtensorMap tm_w,
               const __grid_constant__ CUtensorMap tm_g, const __grid_constant__ CUtensorMap tm_h_mn,
               const __grid_constant__ CUtensorMap tm_w_mn, const __grid_constant__ CUtensorMap tm_g_mn,
               const __grid_constant__ CUtensorMap tm_out, const __grid_constant__ CUtensorMap tm_dh, const LmParams p) {
  using SM = LmSmem;
  constexpr int NST = SM::kStages;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t base = smem_u32(smem_raw);
  launch_next();
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
  if (warp == 8 && lane == 0) {
    for (int j = 0; j < p.n_jobs; ++j) {
      const int kind = p.job[j].kind;
      if (kind <= LM_GRAD) { tma_prefetch_desc(&tm_h); tma_prefetch_desc(&tm_w); }
      if (kind == LM_DH) { tma_prefetch_desc(&tm_g); tma_prefetch_desc(&tm_w_mn); tma_prefetch_desc(&tm_dh); }
      if (kind == LM_DW) { tma_prefetch_desc(&tm_g_mn); tma_prefetch_desc(&tm_h_mn); }
      if (kind == LM_GRAD || kind == LM_DW) tma_prefetch_desc(&tm_out);
    }
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t rank = cluster_ctarank();
  wait_previous();
  const uint32_t tmem = *tmem_slot;
  const AbortCtx ab{abort_flag, p.status, p.wait_budget};
  const int n_rows = *reinterpret_cast<const volatile int *>(p.n_rows);
  const int t0 = blockIdx.x >> 1, tstep = gridDim.x >> 1;
  LmTile c = {};
  bool more = c.start(p, n_rows, t0, tstep);

  if (warp == 8) {
    // ------------------------------------------------------------ TMA producer
    // One thread issues every load, so its own instructions are on the path of a stage: the loop is compiled for each kind,
    // with the maps as constants and nothing left to compute but coordinates.
    if (lane == 0) {
      const uint32_t full_leader = map_to_rank(bar_full, 0);
      uint32_t st = 0, phase = 1;
      bool ok = true, skip = (p.test_flags & TEST_SKIP_FWD_LOAD) && blockIdx.x == 0;
      auto produce = [&](auto kind_tag) {
        constexpr int kKind = decltype(kind_tag)::value;
        const int m0 = c.m * kLmTile + rank * 128, n0 = c.n * kLmTile + rank * 128;  // this CTA's rows of A, columns of B
        const int mc = m0 >> 6, nc = n0 >> 6, w0 = p.v0 + n0;
        const bool one_box = p.mn_chunks == 2;
        int k0 = c.kb0 * 64;
        for (int left = c.nkb; left > 0; --left, k0 += 64) {
          if (!mbar_wait(bar_empty + 8 * st, phase, ab, WAIT_LM_EMPTY)) { ok = false; break; }
          const uint32_t sA = base + st * SM::kStageBytes, sB = sA + SM::kABytes, bar = full_leader + 8 * st;
          if (!skip) {
            if (rank == 0) mbar_expect_tx(bar_full + 8 * st, 2 * SM::kStageBytes);
            if constexpr (kKind <= LM_GRAD) {
              tma_load_2d_pair(sA, &tm_h, bar, k0, m0);
              tma_load_2d_pair(sB, &tm_w, bar, k0, w0);
            } else if constexpr (kKind == LM_DH) {
              const bool lo = k0 >= p.half_k;
              const int kc = lo ? k0 - p.half_k : k0, vr = p.v0 + kc;
              tma_load_2d_pair(sA, &tm_g, bar, kc, lo ? m0 + (int)p.rows_pad : m0);
              if (one_box) tma_load_3d_pair(sB, &tm_w_mn, bar, 0, vr, nc);
              else for (int b = 0; b < 2; ++b) tma_load_3d_pair(sB + b * 8192, &tm_w_mn, bar, n0 + b * 64, vr, 0);
            } else {
              tma_load_3d_pair(sA, &tm_g_mn, bar, 0, k0, mc);
              tma_load_3d_pair(sB, &tm_h_mn, bar, 0, k0, nc);
            }
          }
          skip = false;
          if (++st == NST) { st = 0; phase ^= 1; }
        }
      };
      for (; ok && more; more = c.next(p, n_rows)) {
        if (c.kind <= LM_GRAD) produce(std::integral_constant<int, LM_GRAD>{});
        else if (c.kind == LM_DH) produce(std::integral_constant<int, LM_DH>{});
        else produce(std::integral_constant<int, LM_DW>{});
      }
    }
  } else if (warp == 9) {
   if (rank == 0) {
    // -------------------------------------------------------------- MMA issuer
    const bool elected = elect_one();
    uint32_t T = 0, ic = 0;
    bool ok = true;
    for (; ok && more; more = c.next(p, n_rows), ++ic) {
      const int a_mn = c.kind == LM_DW, b_mn = c.kind >= LM_DH;
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
    const uint32_t s_out = base + SM::kOffOut + warp * 4096;
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
    const int half = warp >> 2, col0 = half * 128;
    uint32_t ic = 0;
    bool ok = true;
    for (; ok && more; more = c.next(p, n_rows), ++ic) {
      const uint32_t buf = ic & 1;
      ok = mbar_wait(bar_acc_full + 8 * buf, (ic >> 1) & 1, ab, WAIT_LM_ACC_FULL);
      if (!ok) break;
      tc_fence_after();
      const uint32_t tD = tmem + buf * kLmTile + lane_off + col0;
      const int row0 = c.m * kLmTile + rank * 128 + (warp & 3) * 32, row = row0 + lane, n0 = c.n * kLmTile + col0;  // tile row, first column of this warp
      if (c.kind == LM_STATS) {
        const int tgt = row < n_rows ? p.target[row] - p.v0 - n0 : -1;  // column of the target, relative
        float m = -INFINITY, l = 0.f, xt = 0.f;
        bool hit = false;
        for (int q = 0; q < 4; ++q) {
          uint32_t v[32];
          tmem_ld32(tD + q * 32, v);
          tc_wait_ld();
          const int left = c.cols - (n0 + q * 32);  // columns that exist
          if ((unsigned)(tgt - q * 32) < 32u) {
            hit = true;
#pragma unroll
            for (int e = 0; e < 32; ++e) if (tgt - q * 32 == e) xt = __uint_as_float(v[e]);
          }
          float cm = -INFINITY;
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            const float x = e < left ? __fmul_rn(__uint_as_float(v[e]), p.scale_log2) : -INFINITY;  // (write_loss counts on this rounding)
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
      } else if (c.kind == LM_GRAD) {
        const bool live = row < n_rows;
        const int tgt = live ? p.target[row] - p.v0 - n0 : -1;
        const float lse2 = live ? p.lse2[row] : 0.f, gs = live ? p.gscale[row] : 0.f, gt = live ? p.gtarget[row] : 0.f;
        for (int q = 0; q < 4; ++q) {
          uint32_t v[32];
          tmem_ld32(tD + q * 32, v);
          tc_wait_ld();
          const int left = c.cols - (n0 + q * 32);
          float g[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            const float pr = ex2(fmaf(__uint_as_float(v[e]), p.scale_log2, -lse2));
            g[e] = tgt - q * 32 == e ? gt : live && e < left ? pr * gs : 0.f;
          }
          if (!(q & 1)) { if (lane == 0) bulk_wait_read(); __syncwarp(); }
          stage_bf16(s_out, lane, (q & 1) * 4, g);
          if (p.halves == 2) {  // few rows: lo by plain stores, there is no second block to stage it in
            __nv_bfloat16 *lo = p.grad_lo + (long long)row * p.ld_grad + n0 + q * 32;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint32_t w[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const float a = g[8 * e + 2 * j], b = g[8 * e + 2 * j + 1];
                w[j] = pack_bf16(a - __bfloat162float(__float2bfloat16_rn(a)), b - __bfloat162float(__float2bfloat16_rn(b)));
              }
              *reinterpret_cast<uint4 *>(lo + 8 * e) = make_uint4(w[0], w[1], w[2], w[3]);  // (the scratch is aligned to 16 bytes)
            }
          }
          if (q & 1) {
            fence_async_shared();
            __syncwarp();
            if (lane == 0) { tma_store_2d(&tm_out, s_out, n0 + (q - 1) * 32, row0); bulk_commit(); }
          }
        }
      } else {
        const bool dh = c.kind == LM_DH, f32 = dh || p.dw_f32, add = dh ? p.dh_add : p.dw_add;
        const bool zero = c.nkb == 0;   // an empty contraction: nothing was accumulated
        const CUtensorMap *map = dh ? &tm_dh : &tm_out;
        // (a box that begins outside is left out; one that only ends outside is cut off by the map)
        const bool inside = row0 < (dh ? n_rows : c.m_fixed);
        const long long out_row = dh ? c.split * p.rows_pad + row0 : p.v0 + row0;
        for (int q = 0; q < 4; ++q) {
          uint32_t v[32];
          tmem_ld32(tD + q * 32, v);
          tc_wait_ld();
          float x[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] = zero ? 0.f : __uint_as_float(v[e]);
          const int col = n0 + q * 32;
          if (f32) {
            if (lane == 0) bulk_wait_read();
            __syncwarp();
            stage_f32(s_out, lane, x);
            fence_async_shared();
            __syncwarp();
            if (lane == 0 && inside && col < p.hidden) {
              if (add) tma_add_2d(map, s_out, col, (int)out_row); else tma_store_2d(map, s_out, col, (int)out_row);
              bulk_commit();
            }
          } else {
            if (!(q & 1)) { if (lane == 0) bulk_wait_read(); __syncwarp(); }
            stage_bf16(s_out, lane, (q & 1) * 4, x);
            if (q & 1) {
              fence_async_shared();
              __syncwarp();
              if (lane == 0 && inside && col - 32 < p.hidden) { tma_store_2d(map, s_out, col - 32, (int)out_row); bulk_commit(); }
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(map_to_rank(bar_acc_empty + 8 * buf, 0));
    }
    if (lane == 0) bulk_wait();
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
