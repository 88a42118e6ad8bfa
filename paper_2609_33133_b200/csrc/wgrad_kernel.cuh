// Gradient of a product's weight from the 8-bit checkpoint of its input: dW = dY^T X, [out, cols], contraction over the tokens.
//
// 256 x 256 tiles of CTA pairs (tcgen05.mma.cta_group::2, fp32 accumulators in TMEM): each CTA brings 128 columns of dY and of X for 64 tokens
// a stage, both with their contraction along the rows (the tensor core takes either order).  X as a bf16 operand is
// exact (an 8-bit integer times a power of two) but where a token's factor goes in: that product is rounded once, as the norm's
// output is in the forward pass.  A factor of a channel goes into the result in fp32.  There are two ways to that operand:
//   kBits   the kernel loads the 8 bits and turns them into bf16 in shared memory, by warps of its own, in the layout that the copy engine would have
//           written.  No launch and no memory beside it, but every row of tiles does it again, and with 92 instructions for 16 values it
//           keeps the tensor core waiting: 740 cycles a stage instead of 512.
//   other   ckpt_unpack_kernel has left X in bf16 in scratch, from where the copy engine loads it.
// Measured (us, kBits against other): 129 tokens x 256 -> 256 6.9 against 8.2; 4096 x 3584 -> 512 24 against 27; 4096 x 3584 -> 3584 91 against 84;
// 16384 x 3584 -> 18944 1705 against 1450 to 1540.  wgrad_way (block.cu) chooses.
// Without kBits the tensor pipe is 95.9 % active (4096 x 3584 -> 18944: 343 us, 1621 TFLOP/s); in a long run the board's power decides: 16384 x 3584 -> 18944 takes
// 1770 us, 1257 TFLOP/s, and the library's product of the same sizes 1610.
//
// The tensor core's adder drops what does not fit, always towards zero, 2^-24 to 2^-23 of the accumulator for every 16 tokens: over
// 16384 tokens of one sign 1e-4 of a result, far under a bf16 result's rounding but not under an fp32 one's.  So for fp32 a tile's contraction is cut into
// pieces of kWgChunk stages; the two halves of TMEM take them in turn, and the pieces are added in memory by the copy engine, rounded to
// nearest, one behind the other (each warp waits for its own addition to be done before it starts the next).  A bf16 result goes that way through fp32
// scratch, too, from more than kWgLong stages on: in one accumulator a million tokens of one sign lost 6.6e-3 of it, twice its rounding.
//
// Few tiles share their contraction out further (`splits`), each share into fp32 scratch, and wgrad_join_kernel adds them in order.
//
// Roles: warps 0-7 epilogue (warp w: TMEM lanes 32 (w % 4).., columns 128 (w / 4)..), warp 8 loads dY and a bf16 X (each CTA its own
// share, all counted on the first CTA's barrier), warp 9 of the first CTA issues the MMAs of both; with kBits also warp 10, which loads X in 8 bits,
// warp 11, which brings the tokens' factors, and warps 12-19, which turn X into bf16 and tell the first CTA: what they have written is handed over at cluster scope, since an
// MMA that the first CTA issues reads the second one's as well.
#pragma once
#include <cuda.h>

#include "block_kernels.cuh"
#include "pair_tile.cuh"

namespace augtree {

constexpr int kWgChunk = 32;   // stages (of 64 tokens) between additions of an fp32 result
constexpr int kWgLong = 512;   // stages that a bf16 result may take in one accumulator: 2048 additions, which lose 2.4e-4 of it at most, an eighth of its rounding's half step or less
constexpr int kWgTeams = 2, kWgTeam = 4;    // teams of warps that turn X into bf16, stage by stage in turn; warps of a team
template <bool kBits> constexpr int kWgThreads = kBits ? (12 + kWgTeams * kWgTeam) * 32 : 320;
enum : int { WAIT_WG_FULL = 100, WAIT_WG_EMPTY = 101, WAIT_WG_ACC_FULL = 102, WAIT_WG_ACC_EMPTY = 103, WAIT_WG_RAW_FULL = 104, WAIT_WG_RAW_EMPTY = 105,
             WAIT_WG_X_FULL = 106, WAIT_WG_X_EMPTY = 107 };

template <bool kBits> struct WgSmem {
  static constexpr int kABytes = 128 * 128, kXBytes = 128 * 128;    // this CTA's 128 columns of 64 tokens in bf16
  static constexpr int kRawBytes = 64 * 128, kScaleBytes = 64 * 16; // the same in 8 bits; 16 exponent bytes of a token, four of them its columns'
  static constexpr int kA = kBits ? 5 : 6, kX = kBits ? 4 : 6, kRaw = kBits ? 4 : 1;    // stages of each (kRaw: with kBits)
  static constexpr int kOffX = kA * kABytes, kOffRaw = kOffX + kX * kXBytes, kOffScale = kOffRaw + (kBits ? kRaw * kRawBytes : 0);
  static constexpr int kOffRow = kOffScale + (kBits ? kRaw * kScaleBytes : 0);    // 64 factors a stage, in 1 KB for all
  static constexpr int kOffOut = kOffRow + (kBits ? 1024 : 0);      // 4 KB a warp on their way out
  static constexpr int kOffBar = kOffOut + 8 * 4096;
  static constexpr int kBytes = kOffBar + 512;
  // A stage of X is one team's for good: a team that took over another's could wait for a phase whose predecessor has not ended yet, and such a
  // wait returns at once.
  static_assert(!kBits || (kX % kWgTeams == 0 && kRaw % kWgTeams == 0 && kRaw <= 4), "stages of a team");
  static_assert(kOffOut % 1024 == 0 && kBytes <= 227 * 1024, "shared memory");
};

struct WgradParams {
  int out, cols, steps;        // rows and columns of dW; stages of the contraction
  int mt, nt, splits, share;   // tiles; shares of the contraction, stages of a share
  int a_chunks;                // 64-column chunks in a box of dY: 2, or 1 (out not a multiple of 64)
  int scales;                  // where a checkpoint row's exponents begin
  int rows;                    // tokens
  const float *row;            // factor of a token, or null
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

// tm_x: X in bf16.  tm_raw: the checkpoint as bytes, boxes of 128 columns x 64 tokens; tm_scale: the same memory, boxes of 16 bytes x 64 tokens (the four
// exponents that are wanted lie somewhere in them: a copy has to start on 16 bytes).
template <bool kBits>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kWgThreads<kBits>, 1)
wgrad_kernel(const __grid_constant__ CUtensorMap tm_dy, const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_raw,
             const __grid_constant__ CUtensorMap tm_scale, const __grid_constant__ CUtensorMap tm_out, const WgradParams p) {
  using SM = WgSmem<kBits>;
  extern __shared__ __align__(1024) uint8_t smem_raw[];
  const uint32_t base = smem_u32(smem_raw);
  launch_next();
  if (base & 1023u) {  // the same in both CTAs of a pair
    if (threadIdx.x == 0 && atomicCAS(p.status, 0, -6) == 0) p.status[1] = 5;
    return;
  }
  // barriers: eight bytes each
  const uint32_t bars = base + SM::kOffBar;
  const uint32_t a_full = bars, a_empty = bars + 64, x_full = bars + 128, x_empty = bars + 160, raw_full = bars + 192, raw_empty = bars + 240;
  const uint32_t acc_full = bars + 288, acc_empty = bars + 304;
  volatile uint32_t *tmem_slot = reinterpret_cast<volatile uint32_t *>(smem_raw + SM::kOffBar + 384);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(smem_raw + SM::kOffBar + 392);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int s = 0; s < SM::kA; ++s) { mbar_init(a_full + 8 * s, 1); mbar_init(a_empty + 8 * s, 1); }
    if (kBits) for (int s = 0; s < SM::kX; ++s) { mbar_init(x_full + 8 * s, 2 * kWgTeam); mbar_init(x_empty + 8 * s, 1); }
    for (int s = 0; s < SM::kRaw; ++s) { mbar_init(raw_full + 8 * s, p.row ? 2 : 1); mbar_init(raw_empty + 8 * s, kWgTeam); }
    for (int s = 0; s < 2; ++s) { mbar_init(acc_full + 8 * s, 1); mbar_init(acc_empty + 8 * s, 16); }
    *abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 9) { tmem_alloc_pair(smem_u32((const void *)tmem_slot), 512); tmem_relinquish_pair(); }
  if (warp == 8 && lane == 0) {
    tma_prefetch_desc(&tm_dy); tma_prefetch_desc(&tm_out);
    if (kBits) { tma_prefetch_desc(&tm_raw); tma_prefetch_desc(&tm_scale); } else tma_prefetch_desc(&tm_x);
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t rank = cluster_ctarank();
  wait_previous();
  const uint32_t tmem = *tmem_slot;
  const AbortCtx ab{abort_flag, p.status, p.wait_budget};
  const int tiles = p.mt * p.nt * p.splits, t0 = blockIdx.x >> 1, tstep = gridDim.x >> 1;
  const bool skip_first = (p.test_flags & TEST_SKIP_FWD_LOAD) && blockIdx.x == 0;

  if (warp == 8) {
    // ------------------------------------------------------------ dY, X in bf16
    if (lane == 0) {
      const uint32_t full_leader = map_to_rank(a_full, 0);
      uint32_t st = 0, phase = 1;
      bool ok = true, skip = !kBits && skip_first;
      for (int t = t0; ok && t < tiles; t += tstep) {
        const WgradTile c(p, t);
        const int m0 = c.m * kLmTile + rank * 128, n0 = c.n * kLmTile + rank * 128;
        int k0 = c.k0 * 64;
        for (int left = c.steps; left > 0; --left, k0 += 64) {
          if (!mbar_wait(a_empty + 8 * st, phase, ab, WAIT_WG_EMPTY)) { ok = false; break; }
          const uint32_t sA = base + st * SM::kABytes, bar = full_leader + 8 * st;
          if (!skip) {
            if (rank == 0) mbar_expect_tx(a_full + 8 * st, 2 * (kBits ? SM::kABytes : SM::kABytes + SM::kXBytes));
            if (p.a_chunks == 2) tma_load_3d_pair(sA, &tm_dy, bar, 0, k0, m0 >> 6);
            else for (int b = 0; b < 2; ++b) tma_load_3d_pair(sA + b * 8192, &tm_dy, bar, m0 + b * 64, k0, 0);
            if constexpr (!kBits) tma_load_3d_pair(base + SM::kOffX + st * SM::kXBytes, &tm_x, bar, 0, k0, n0 >> 6);
          }
          skip = false;
          if (++st == SM::kA) { st = 0; phase ^= 1; }
        }
      }
    }
  } else if (kBits && warp == 10) {
    // ------------------------------------------------------------ X in 8 bits, into this CTA alone
    if (lane == 0) {
      uint32_t st = 0, phase = 1;
      bool ok = true, skip = skip_first;
      for (int t = t0; ok && t < tiles; t += tstep) {
        const WgradTile c(p, t);
        const int n0 = c.n * kLmTile + rank * 128, s0 = p.scales + ((n0 >> 5) & ~15);
        int k0 = c.k0 * 64;
        for (int left = c.steps; left > 0; --left, k0 += 64) {
          if (!mbar_wait(raw_empty + 8 * st, phase, ab, WAIT_WG_RAW_EMPTY)) { ok = false; break; }
          const uint32_t bar = raw_full + 8 * st;
          if (!skip) {
            mbar_expect_tx(bar, SM::kRawBytes + SM::kScaleBytes);
            tma_load_2d(base + SM::kOffRaw + st * SM::kRawBytes, &tm_raw, bar, n0, k0);
            tma_load_2d(base + SM::kOffScale + st * SM::kScaleBytes, &tm_scale, bar, s0, k0);
          }
          skip = false;
          if (++st == SM::kRaw) { st = 0; phase ^= 1; }
        }
      }
    }
  } else if (kBits && warp == 11) {
    // ------------------------------------------------------------ factors of the tokens, read three stages ahead of their place
    if (p.row) {
      float *row = reinterpret_cast<float *>(smem_raw + SM::kOffRow);
      constexpr int kFar = 3;
      uint32_t st = 0, phase = 1;
      bool ok = true;
      for (int t = t0; ok && t < tiles; t += tstep) {
        const WgradTile c(p, t);
        float f[kFar][2];
        auto fetch = [&](int stage, float (&v)[2]) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int token = (c.k0 + stage) * 64 + lane + 32 * h;
            v[h] = stage < c.steps && token < p.rows ? p.row[token] : 0.f;
          }
        };
#pragma unroll
        for (int i = 0; i < kFar; ++i) fetch(i, f[i]);
        for (int stage = 0; ok && stage < c.steps; stage += kFar) {
#pragma unroll
          for (int i = 0; i < kFar; ++i) {
            if (stage + i >= c.steps) break;
            if (!mbar_wait(raw_empty + 8 * st, phase, ab, WAIT_WG_RAW_EMPTY)) { ok = false; break; }
            row[st * 64 + lane] = f[i][0];
            row[st * 64 + lane + 32] = f[i][1];
            __syncwarp();
            if (lane == 0) { mbar_arrive(raw_full + 8 * st); }
            fetch(stage + i + kFar, f[i]);
            if (++st == SM::kRaw) { st = 0; phase ^= 1; }
          }
        }
      }
    }
  } else if (kBits && warp >= 12) {
    // ------------------------------------------------------------ from 8 bits to bf16
    // One warp's way through a stage (wait, read, arithmetic, write, fence, arrival) takes twice as long as the tensor core's, so two teams take
    // the stages in turn.  A thread has 16 columns of tokens k, k + 16, k + 32, k + 48.  Its two 16-byte pieces go to places 2 c and 2 c + 1 of the token's
    // 128 bytes (swizzled with the token's number); the second chunk's threads write them in the other order, so that the eight threads of a token
    // never meet in a bank.
    const int team = (warp - 12) / kWgTeam, k = (threadIdx.x - (12 + team * kWgTeam) * 32) >> 3, c16 = threadIdx.x & 7, flip = c16 >> 2;
    const uint32_t put0 = (c16 >> 2) * 8192 + k * 128 + (((((c16 & 3) * 2) | flip) ^ (k & 7)) << 4);      // (k + 16 has the same low bits)
    const uint32_t put1 = put0 ^ 16;
    const float *row = reinterpret_cast<const float *>(smem_raw + SM::kOffRow);
    uint32_t sr = team, pr = 0, sx = team, px = 1;
    int turn = 0;        // of the stage, counted over all tiles
    bool ok = true;
    for (int t = t0; ok && t < tiles; t += tstep) {
      const WgradTile c(p, t);
      const int n0 = c.n * kLmTile + rank * 128;
      const uint32_t scale_at = ((n0 >> 5) & 15) + (c16 >> 1);
      const int first = (team - turn % kWgTeams + kWgTeams) % kWgTeams;       // this team's first stage of the tile
      turn += c.steps;
      for (int stage = first; stage < c.steps; stage += kWgTeams) {
        if (!mbar_wait(raw_full + 8 * sr, pr, ab, WAIT_WG_RAW_FULL)) { ok = false; break; }
        const uint8_t *raw = smem_raw + SM::kOffRaw + sr * SM::kRawBytes + k * 128 + c16 * 16;
        const uint8_t *sc = smem_raw + SM::kOffScale + sr * SM::kScaleBytes + k * 16 + scale_at;
        const uint32_t sX = base + SM::kOffX + sx * SM::kXBytes;
        uint4 q[4];
        float unit[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          q[h] = *reinterpret_cast<const uint4 *>(raw + h * 16 * 128);
          unit[h] = ckpt_unit(sc[h * 16 * 16]);
          if (p.row) unit[h] *= row[sr * 64 + k + 16 * h];
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(raw_empty + 8 * sr);      // (all of the warp's reads have come back: their values went into what follows)
        if (!mbar_wait(x_empty + 8 * sx, px, ab, WAIT_WG_X_EMPTY)) { ok = false; break; }
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          const uint2 a = make_uint2(q[h].x, q[h].y), b = make_uint2(q[h].z, q[h].w);
          const V8 lo = ckpt_decode(flip ? b : a, unit[h]), hi = ckpt_decode(flip ? a : b, unit[h]);
          st_shared_v4(sX + put0 + h * 16 * 128, pack_bf16(lo.p[0].x, lo.p[0].y), pack_bf16(lo.p[1].x, lo.p[1].y), pack_bf16(lo.p[2].x, lo.p[2].y), pack_bf16(lo.p[3].x, lo.p[3].y));
          st_shared_v4(sX + put1 + h * 16 * 128, pack_bf16(hi.p[0].x, hi.p[0].y), pack_bf16(hi.p[1].x, hi.p[1].y), pack_bf16(hi.p[2].x, hi.p[2].y), pack_bf16(hi.p[3].x, hi.p[3].y));
        }
        fence_async_shared();      // the tensor core reads what was written here
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster_release(map_to_rank(x_full + 8 * sx, 0));
        sr += kWgTeams;
        if (sr >= SM::kRaw) { sr -= SM::kRaw; pr ^= 1; }
        sx += kWgTeams;
        if (sx >= SM::kX) { sx -= SM::kX; px ^= 1; }
      }
    }
  } else if (warp == 9) {
    if (rank == 0) {
      // ------------------------------------------------------------ MMA issuer
      const bool elected = elect_one();
      const uint32_t idesc = make_idesc(256, kLmTile, 1, 1);
      uint32_t sa = 0, pa = 0, sx = 0, px = 0, ic = 0;
      bool ok = true;
      for (int t = t0; ok && t < tiles; t += tstep) {
        const WgradTile c(p, t);
        const int chunk = p.f32 ? kWgChunk : c.steps;
        for (int kb = 0; kb < c.steps && ok; ++ic) {
          const uint32_t buf = ic & 1, tD = tmem + buf * kLmTile;
          if (ic >= 2) {
            ok = mbar_wait(acc_empty + 8 * buf, ((ic >> 1) - 1) & 1, ab, WAIT_WG_ACC_EMPTY);
            if (!ok) break;
            tc_fence_after();
          }
          const int end = min(kb + chunk, c.steps);
          for (bool first = true; kb < end; ++kb, first = false) {
            ok = mbar_wait(a_full + 8 * sa, pa, ab, WAIT_WG_FULL) && (!kBits || mbar_wait_cluster(x_full + 8 * sx, px, ab, WAIT_WG_X_FULL));
            if (!ok) break;
            tc_fence_after();
            const uint32_t a_lo = sdesc_lo(base + sa * SM::kABytes, 8192), b_lo = sdesc_lo(base + SM::kOffX + sx * SM::kXBytes, 8192);
            if (elected) {
#pragma unroll
              for (int k = 0; k < 4; ++k) mma_ss2_pair(tD, a_lo + k * (2048 >> 4), b_lo + k * (2048 >> 4), idesc, (uint32_t)(!first || k > 0));
              tc_commit_pair(a_empty + 8 * sa);
              if constexpr (kBits) tc_commit_pair(x_empty + 8 * sx);
            }
            if (++sa == SM::kA) { sa = 0; pa ^= 1; }
            if (++sx == SM::kX) { sx = 0; px ^= 1; }
          }
          if (!ok) break;
          if (elected) tc_commit_pair(acc_full + 8 * buf);
        }
      }
    }
  } else if (warp < 8) {
    // ------------------------------------------------------------ epilogue
    const uint32_t s_out = base + SM::kOffOut + warp * 4096;
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
    const int col0 = (warp >> 2) * 128;
    uint32_t ic = 0;
    bool ok = true;
    for (int t = t0; ok && t < tiles; t += tstep) {
      const WgradTile c(p, t);
      const int row0 = c.m * kLmTile + rank * 128 + (warp & 3) * 32, n0 = c.n * kLmTile + col0, chunk = p.f32 ? kWgChunk : c.steps;
      // (a box that begins outside is left out; one that only ends outside is cut off by the map)
      const bool inside = row0 < p.out;
      const int out_row = (int)(c.split * p.part_rows) + row0;
      float f[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) f[q] = p.col && n0 + q * 32 + lane < p.cols ? block_scalar(p.col, n0 + q * 32 + lane, p.col_type) : 1.f;
      for (int kb = 0; kb < c.steps; kb += chunk, ++ic) {
        const uint32_t buf = ic & 1;
        ok = mbar_wait(acc_full + 8 * buf, (ic >> 1) & 1, ab, WAIT_WG_ACC_FULL);
        if (!ok) break;
        tc_fence_after();
        const uint32_t tD = tmem + buf * kLmTile + lane_off + col0;
        const bool add = kb > 0 || p.add;
        if (kb > 0 && lane == 0) bulk_wait();       // the piece before is in memory
        __syncwarp();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int col = n0 + q * 32;
          uint32_t v[32];
          tmem_ld32(tD + q * 32, v);
          tc_wait_ld();
          float x[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] = __uint_as_float(v[e]) * __shfl_sync(0xffffffffu, f[q], e);
          if (p.f32) {
            if (lane == 0) bulk_wait_read();
            __syncwarp();
            stage_f32(s_out, lane, x);
            fence_async_shared();
            __syncwarp();
            if (lane == 0 && inside && col < p.cols) {
              if (add) tma_add_2d(&tm_out, s_out, col, out_row); else tma_store_2d(&tm_out, s_out, col, out_row);
              bulk_commit();
            }
          } else {
            if (!(q & 1)) { if (lane == 0) bulk_wait_read(); __syncwarp(); }
            stage_bf16(s_out, lane, (q & 1) * 4, x);
            if (q & 1) {
              fence_async_shared();
              __syncwarp();
              if (lane == 0 && inside && col - 32 < p.cols) { tma_store_2d(&tm_out, s_out, col - 32, out_row); bulk_commit(); }
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(map_to_rank(acc_empty + 8 * buf, 0));
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

// Shares' partial sums (or a long bf16 result's only one) into dW, in the order of the shares.
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
