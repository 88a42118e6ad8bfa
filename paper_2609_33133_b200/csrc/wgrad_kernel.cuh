// Gradient of a product's weight from the 8-bit checkpoint of its input: dW = dY^T X, [out, cols], contraction over the tokens.
//
// 256 x 256 tiles of CTA pairs (tcgen05.mma.cta_group::2, fp32 accumulators in TMEM): each CTA loads 128 columns of dY and of X for 64 tokens
// a stage, both with their contraction along the rows (the tensor core takes either order).  X is the bf16 form of what the
// checkpoint stands for, times a token's factor where there is one; without the factor that form is exact (an 8-bit integer times a power of
// two), with it the product is rounded once, as the norm's output is in the forward pass.  A factor of a channel goes into the result in fp32.
//
// The tensor core's adder drops what does not fit, always towards zero, 2^-24 to 2^-23 of the accumulator for every 16 tokens: over
// 16384 tokens that would be 3e-5 of a result.  So a tile's contraction is cut into pieces of kWgChunk stages, the two halves of TMEM take
// them in turn, and the epilogue adds the pieces in registers, rounded to nearest, under the next piece's products.
//
// Few tiles share their contraction out further (`splits`), each share into fp32 scratch, and wgrad_join_kernel adds them in order.
//
// Roles (320 threads a CTA): warps 0-7 epilogue (warp w: TMEM lanes 32 (w % 4).., columns 128 (w / 4)..), warp 8 TMA loads
// (each CTA its own share, all counted on the first CTA's barrier), warp 9 of the first CTA issues the MMAs of both.
#pragma once
#include <cuda.h>

#include "block_kernels.cuh"
#include "pair_tile.cuh"

namespace augtree {

constexpr int kWgChunk = 32;   // stages (of 64 tokens) between additions in registers
enum : int { WAIT_WG_FULL = 100, WAIT_WG_EMPTY = 101, WAIT_WG_ACC_FULL = 102, WAIT_WG_ACC_EMPTY = 103 };

struct WgradParams {
  int out, cols, steps;        // rows and columns of dW; stages of the contraction
  int mt, nt, splits, share;   // tiles; shares of the contraction, stages of a share
  int a_chunks;                // 64-column chunks in a box of dY: 2, or 1 (out not a multiple of 64)
  long long part_rows;         // rows of a share's partial sums
  int f32, add;                // type of what is written, add to what is there (splits == 1)
  const void *col;             // factor of a column of dW, or null
  int col_type;
  int *status;
  long long wait_budget;
  int test_flags;
};

struct WgradTile {
  int m, n, split, k0, steps;
  __device__ __forceinline__ WgradTile(const WgradParams &p, int t) {
    n = t % p.nt;              // hidden columns fastest: neighbours share their columns of dY
    const int rest = t / p.nt;
    split = rest / p.mt;
    m = rest - split * p.mt;
    k0 = min(split * p.share, p.steps);
    steps = min(p.share, p.steps - k0);
  }
};

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kLmThreads, 1)
wgrad_kernel(const __grid_constant__ CUtensorMap tm_dy, const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_out,
             const WgradParams p) {
  using SM = LmSmem;
  constexpr int NST = SM::kStages;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t base = smem_u32(smem_raw);
  launch_next();
  if (base & 1023u) {  // the same in both CTAs of a pair
    if (threadIdx.x == 0 && atomicCAS(p.status, 0, -6) == 0) p.status[1] = 5;
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
  if (warp == 8 && lane == 0) { tma_prefetch_desc(&tm_dy); tma_prefetch_desc(&tm_x); tma_prefetch_desc(&tm_out); }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t rank = cluster_ctarank();
  wait_previous();
  const uint32_t tmem = *tmem_slot;
  const AbortCtx ab{abort_flag, p.status, p.wait_budget};
  const int tiles = p.mt * p.nt * p.splits, t0 = blockIdx.x >> 1, tstep = gridDim.x >> 1;

  if (warp == 8) {
    // ------------------------------------------------------------ TMA producer
    if (lane == 0) {
      const uint32_t full_leader = map_to_rank(bar_full, 0);
      uint32_t st = 0, phase = 1;
      bool ok = true, skip = (p.test_flags & TEST_SKIP_FWD_LOAD) && blockIdx.x == 0;
      for (int t = t0; ok && t < tiles; t += tstep) {
        const WgradTile c(p, t);
        const int m0 = c.m * kLmTile + rank * 128, n0 = c.n * kLmTile + rank * 128;
        int k0 = c.k0 * 64;
        for (int left = c.steps; left > 0; --left, k0 += 64) {
          if (!mbar_wait(bar_empty + 8 * st, phase, ab, WAIT_WG_EMPTY)) { ok = false; break; }
          const uint32_t sA = base + st * SM::kStageBytes, sB = sA + SM::kABytes, bar = full_leader + 8 * st;
          if (!skip) {
            if (rank == 0) mbar_expect_tx(bar_full + 8 * st, 2 * SM::kStageBytes);
            if (p.a_chunks == 2) tma_load_3d_pair(sA, &tm_dy, bar, 0, k0, m0 >> 6);
            else for (int b = 0; b < 2; ++b) tma_load_3d_pair(sA + b * 8192, &tm_dy, bar, m0 + b * 64, k0, 0);
            tma_load_3d_pair(sB, &tm_x, bar, 0, k0, n0 >> 6);
          }
          skip = false;
          if (++st == NST) { st = 0; phase ^= 1; }
        }
      }
    }
  } else if (warp == 9) {
    if (rank == 0) {
      // ------------------------------------------------------------ MMA issuer
      const bool elected = elect_one();
      const uint32_t idesc = make_idesc(256, kLmTile, 1, 1);
      uint32_t T = 0, ic = 0;
      bool ok = true;
      for (int t = t0; ok && t < tiles; t += tstep) {
        const WgradTile c(p, t);
        for (int kb = 0; kb < c.steps && ok; ++ic) {
          const uint32_t buf = ic & 1, tD = tmem + buf * kLmTile;
          if (ic >= 2) {
            ok = mbar_wait(bar_acc_empty + 8 * buf, ((ic >> 1) - 1) & 1, ab, WAIT_WG_ACC_EMPTY);
            if (!ok) break;
            tc_fence_after();
          }
          const int end = min(kb + kWgChunk, c.steps);
          for (bool first = true; kb < end; ++kb, ++T, first = false) {
            const uint32_t st = T % NST;
            ok = mbar_wait(bar_full + 8 * st, (T / NST) & 1, ab, WAIT_WG_FULL);
            if (!ok) break;
            tc_fence_after();
            const uint32_t sA = base + st * SM::kStageBytes;
            const uint32_t a_lo = sdesc_lo(sA, 8192), b_lo = sdesc_lo(sA + SM::kABytes, 8192);
            if (elected) {
#pragma unroll
              for (int k = 0; k < 4; ++k) mma_ss2_pair(tD, a_lo + k * (2048 >> 4), b_lo + k * (2048 >> 4), idesc, (uint32_t)(!first || k > 0));
              tc_commit_pair(bar_empty + 8 * st);
            }
          }
          if (!ok) break;
          if (elected) tc_commit_pair(bar_acc_full + 8 * buf);
        }
      }
    }
  } else {
    // ------------------------------------------------------------ epilogue warps 0-7
    const uint32_t s_out = base + SM::kOffOut + warp * 4096;
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
    const int col0 = (warp >> 2) * 128;
    uint32_t ic = 0;
    bool ok = true;
    for (int t = t0; ok && t < tiles; t += tstep) {
      const WgradTile c(p, t);
      float acc[4][32];
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int e = 0; e < 32; ++e) acc[q][e] = 0.f;
      for (int kb = 0; kb < c.steps; kb += kWgChunk, ++ic) {
        const uint32_t buf = ic & 1;
        ok = mbar_wait(bar_acc_full + 8 * buf, (ic >> 1) & 1, ab, WAIT_WG_ACC_FULL);
        if (!ok) break;
        tc_fence_after();
        const uint32_t tD = tmem + buf * kLmTile + lane_off + col0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          uint32_t v[32];
          tmem_ld32(tD + q * 32, v);
          tc_wait_ld();
#pragma unroll
          for (int e = 0; e < 32; ++e) acc[q][e] += __uint_as_float(v[e]);
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(map_to_rank(bar_acc_empty + 8 * buf, 0));
      }
      if (!ok) break;
      const int row0 = c.m * kLmTile + rank * 128 + (warp & 3) * 32, n0 = c.n * kLmTile + col0;
      // (a box that begins outside is left out; one that only ends outside is cut off by the map)
      const bool inside = row0 < p.out;
      const int out_row = (int)(c.split * p.part_rows) + row0;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int col = n0 + q * 32;
        if (p.col) {
          const float f = col + lane < p.cols ? block_scalar(p.col, col + lane, p.col_type) : 0.f;
#pragma unroll
          for (int e = 0; e < 32; ++e) acc[q][e] *= __shfl_sync(0xffffffffu, f, e);
        }
        if (p.f32) {
          if (lane == 0) bulk_wait_read();
          __syncwarp();
          stage_f32(s_out, lane, acc[q]);
          fence_async_shared();
          __syncwarp();
          if (lane == 0 && inside && col < p.cols) {
            if (p.add) tma_add_2d(&tm_out, s_out, col, out_row); else tma_store_2d(&tm_out, s_out, col, out_row);
            bulk_commit();
          }
        } else {
          if (!(q & 1)) { if (lane == 0) bulk_wait_read(); __syncwarp(); }
          stage_bf16(s_out, lane, (q & 1) * 4, acc[q]);
          if (q & 1) {
            fence_async_shared();
            __syncwarp();
            if (lane == 0 && inside && col - 32 < p.cols) { tma_store_2d(&tm_out, s_out, col - 32, out_row); bulk_commit(); }
          }
        }
      }
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

// Shares' partial sums into dW, in the order of the shares.
__global__ void __launch_bounds__(256)
wgrad_join_kernel(const float *part, int splits, long long part_rows, int out, int cols, const void *col, int col_type, void *dw, int type, int add) {
  launch_next();
  wait_previous();
  const long long vecs = cols / 8, total = out * vecs, stride = part_rows * cols;
  for (long long i = blockIdx.x * 256ll + threadIdx.x; i < total; i += gridDim.x * 256ll) {
    V8 x = Row8<float>::load(part + i * 8);
    for (int s = 1; s < splits; ++s) x = x + Row8<float>::load(part + s * stride + i * 8);
    if (col) {
      const long long c0 = i % vecs * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] *= block_scalar(col, c0 + e, col_type);
    }
    if (add) x = x + Row8<float>::load(static_cast<const float *>(dw) + i * 8);
    block_store8<kAny>(static_cast<uint8_t *>(dw) + i * 8 * type_bytes(type), 0, type, x);
  }
}

}  // namespace augtree
