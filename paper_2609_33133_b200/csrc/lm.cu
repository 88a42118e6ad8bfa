// C-ABI entry points of a model's vocabulary ends: embedding lookup and vocabulary cross entropy, with their gradients.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <new>
#include <type_traits>

#include "handle.h"
#include "lm_few_kernel.cuh"
#include "lm_kernels.cuh"
#include "lm_tile_kernel.cuh"
#include "../../include/augtree.h"

using namespace augtree;

struct augtree_lm {
  int32_t vocab = 0, hidden = 0;
  float embed_scale = 1.f, logit_scale = 1.f;
  uint32_t flags = 0;
  int32_t n_lanes = 0;
  int64_t piece_bytes = 0;
  int device = -1;
  int *d_status = nullptr;  // status, detail
};

namespace {

struct LossWs {
  LmRows rows;
  __nv_bfloat16 *h;       // [rows_pad][pad_cols] scored rows
  float *tlogit;          // forward
  float2 *part;           // forward: [n_part][rows_pad]
  __nv_bfloat16 *grad;    // backward: [rows_pad][piece]
  float *dh_part;         // backward: [splits][rows_pad][hidden]
};

int n_part(const augtree_lm *lm) { return 2 * (int)((lm->vocab + kLmTile - 1) / kLmTile); }

// Few rows take kernels of their own (lm_few_kernel.cuh): the MMAs' N, 0 for many rows.
int few_rows(int64_t tokens) { return tokens <= kLmFew ? (int)up(std::max<int64_t>(tokens, 1), 16) : 0; }
// Rows of the call as the kernels see them, and whether G is kept in two halves (lm_tile_kernel.cuh).
int64_t tile_rows(int64_t tokens) { return few_rows(tokens) ? few_rows(tokens) : up(tokens, kLmTile); }
int halves(int64_t tokens) { return tokens <= kLmTile ? 2 : 1; }
constexpr int kRowsOneLaunch = 256;  // up to here the scored rows are found and packed in one launch

int64_t pad_cols(const augtree_lm *lm) { return up(lm->hidden, 64); }

// Columns of a piece of the vocabulary in the backward pass: as many as fit the scratch bound for G, in equal pieces.
// With the default bound a piece has 4096 columns at least, so that the additions into dH's partial sums, one per
// piece, stay a small part of the piece's products however many rows there are.
int64_t piece_bound(const augtree_lm *lm) { return lm->piece_bytes > 0 ? lm->piece_bytes : (int64_t)512 << 20; }
int64_t piece_least(const augtree_lm *lm) { return lm->piece_bytes > 0 ? kLmTile : 4096; }
int64_t piece_cols(const augtree_lm *lm, int64_t rows_pad) {
  const int64_t cols = std::max<int64_t>(piece_bound(lm) / (rows_pad * 2) / kLmTile * kLmTile, piece_least(lm));
  const int64_t pieces = (lm->vocab + cols - 1) / cols;
  return up((lm->vocab + pieces - 1) / pieces, kLmTile);
}

// Shares of dH's contraction.  A launch holds dH's tiles (each a contraction over the piece, `kb` steps) and dW's (over the rows,
// `kr` steps), dealt out to the CTA pairs in turn; the longest pair is waited for.  More shares even the pairs out (and let
// few rows fill the GPU) but each costs a pass over the partial sums: the fewest within 2 % of the best.
int64_t most_splits(int64_t rows) { return std::min<int64_t>(std::max<int64_t>(16384 / rows, 2), 32); }
int dh_splits(const augtree_lm *lm, int64_t rows_pad, int halves, int64_t cols) {
  const int64_t pairs = std::max(lm->n_lanes / 2, 1), nt = (lm->hidden + kLmTile - 1) / kLmTile;
  const int64_t kb = halves * ((cols + 63) / 64), kr = halves * ((rows_pad + 63) / 64);
  const int64_t dh_tiles = rows_pad / kLmTile * nt, dw_tiles = (cols + kLmTile - 1) / kLmTile * nt;
  auto longest = [&](int64_t s) {
    // pair i has every pairs-th tile from i on: the longest is pair 0 or the first one with a dH tile less
    auto load = [&](int64_t i) {
      const int64_t dh = (dh_tiles * s - i + pairs - 1) / pairs, all = (dh_tiles * s + dw_tiles - i + pairs - 1) / pairs;
      return dh * ((kb + s - 1) / s) + (all - dh) * kr;
    };
    return std::max(load(0), load(dh_tiles * s % pairs));
  };
  const int64_t most = std::min<int64_t>(kb, most_splits(rows_pad));
  int64_t best = longest(1), pick = 1;
  for (int64_t s = 2; s <= most; ++s) best = std::min(best, longest(s));
  while (pick < most && longest(pick) * 100 > best * 102) ++pick;
  return (int)pick;
}

// Row tiles of a group (LmTile): hidden states of at most 32 MB, a quarter of L2, in equal groups.
int row_group(const augtree_lm *lm, int64_t rows) {
  const int64_t tiles = rows / kLmTile, most = std::max<int64_t>(((int64_t)32 << 20) / (kLmTile * pad_cols(lm) * 2), 1);
  const int64_t groups = (tiles + most - 1) / most;
  return (int)((tiles + groups - 1) / groups);
}

// Few rows: shares of the vocabulary that fill the CTAs in one go.
int few_splits(const augtree_lm *lm, int64_t cols) {
  const int64_t tiles = (lm->hidden + 255) / 256;
  return (int)std::min<int64_t>(std::max<int64_t>(lm->n_lanes / tiles, 1), (cols + 63) / 64);
}

// Cuts the scratch of a call on `tokens` tokens.  What a call needs does not always grow with its tokens (pieces, shares and the
// few-row kernels change with them), so the size that a caller is told (`told`) takes the most of each part up to there.
size_t loss_layout(const augtree_lm *lm, int64_t tokens, bool bwd, uint8_t *base, LossWs *w, bool told = false) {
  const int64_t few = few_rows(tokens), rp = tile_rows(tokens), gr = rp * halves(tokens), few_most = std::min<int64_t>(rp, kLmFew);
  Cursor c{base};
  w->rows.n_rows = c.take<int>(1);
  w->rows.idx = c.take<int>(rp);
  w->rows.pos = c.take<int>(std::max(rp, tokens));
  w->rows.target = c.take<int>(rp);
  w->h = c.take<__nv_bfloat16>((bwd ? gr : rp) * pad_cols(lm));
  if (!bwd) {
    const int64_t part_few = 4ll * lm->n_lanes * few_most, part_many = few ? 0 : (int64_t)n_part(lm) * rp;
    w->rows.lse2 = w->rows.gscale = nullptr;
    w->rows.x_target = c.take<float>(rp);
    w->tlogit = c.take<float>(rp);
    w->part = c.take<float2>(told ? std::max(part_few, part_many) : few ? part_few : part_many);
  } else {
    const int64_t cols = piece_cols(lm, gr);
    int64_t grad = gr * cols, dh = (few ? few_splits(lm, cols) : dh_splits(lm, rp, halves(tokens), cols)) * rp;
    if (told) {
      const int64_t whole = up(lm->vocab, kLmTile), bound = std::max(piece_bound(lm) / 2, gr * piece_least(lm));
      grad = std::min(gr * whole, bound + gr * kLmTile);   // (equal pieces are rounded up to whole tiles)
      dh = std::max(few_splits(lm, whole) * few_most, few ? 0 : std::min<int64_t>(32 * rp, std::max<int64_t>(16384, 2 * rp)));
    }
    w->rows.x_target = c.take<float>(rp);
    w->rows.lse2 = c.take<float>(rp);
    w->rows.gscale = c.take<float>(rp);
    w->grad = c.take<__nv_bfloat16>(grad);
    w->dh_part = c.take<float>(dh * lm->hidden);
  }
  return c.off;
}

struct EmbedWs {
  uint32_t *key[2];
  int *val[2];
  int *hist, *total, *joins;
  uint32_t *seen;
  float *part;   // [2 x chunks][hidden] sums of the rows that cross from chunk to chunk
  int chunk, n_chunks;
};

// Sorted tokens of a chunk.  A few tokens wait for memory, a chunk's one after the other, so they are spread over four blocks an
// SM as far as chunks of 8 allow (2000 tokens into 5000 x 256: 16 us with 8 a chunk, 22 with 16; 100 tokens into 5000 x 1024: 16 us
// with 8, 22 with 4, which leave more rows to join); many take chunks of 32 (24576
// tokens x 3584 bf16: 237 us against 243 with 16; 131071 x 1032 fp32: 151 against 155 with 64), and more when the sums of the rows
// that cross chunks would grow large.
int embed_chunk(const augtree_lm *lm, int64_t n) {
  int chunk = 8;
  while (chunk < 32 && n / chunk > 4ll * lm->n_lanes) chunk *= 2;
  while (chunk < kEmbedMaxChunk && n / chunk > 64ll * lm->n_lanes) chunk *= 2;
  return chunk;
}

size_t embed_layout(const augtree_lm *lm, int64_t tokens, uint8_t *base, EmbedWs *w, bool told = false) {
  const int64_t n = std::max<int64_t>(tokens, 1), blocks = (n + kRadixBlock - 1) / kRadixBlock;
  Cursor c{base};
  for (int i = 0; i < 2; ++i) { w->key[i] = c.take<uint32_t>(n); w->val[i] = c.take<int>(n); }
  w->hist = c.take<int>(blocks * kSortBins);
  w->total = c.take<int>(kSortBins);
  w->chunk = embed_chunk(lm, n);
  w->n_chunks = (int)((tokens + w->chunk - 1) / w->chunk);
  const int64_t most = std::max(std::min<int64_t>((n + 7) / 8, 4ll * lm->n_lanes + 1), std::min<int64_t>((n + 31) / 32, 64ll * lm->n_lanes + 1));
  const int64_t chunks = told ? std::max<int64_t>(most, w->n_chunks) : w->n_chunks;
  w->joins = c.take<int>(chunks + 2);
  w->seen = c.take<uint32_t>((lm->vocab + 31) / 32);
  w->part = c.take<float>(2 * chunks * lm->hidden);
  return c.off;
}

int check_lm(const augtree_lm *lm) {
  if (!lm || lm->device < 0) return AUGTREE_ERR_INVALID_ARG;
  int cur = -1;
  if (cudaGetDevice(&cur) != cudaSuccess) return cuda_failed();
  return cur == lm->device ? AUGTREE_OK : AUGTREE_ERR_INVALID_ARG;
}

// Scored rows packed into the scratch, and their targets' logits (forward: lse null) or gradients.
int compact(const augtree_lm *lm, const void *targets, int id_bytes, int64_t tokens, const void *hidden, const void *weight, const LossWs &w,
            const float *lse, const float *d_loss, float *loss_out, float *lse_out, cudaStream_t st) {
  const auto *ids64 = static_cast<const long long *>(targets);
  const auto *ids32 = static_cast<const int *>(targets);
  const auto *src = static_cast<const uint4 *>(hidden), *wt = static_cast<const uint4 *>(weight);
  auto *dst = reinterpret_cast<uint4 *>(w.h);
  const int n = (int)tokens, row_vecs = lm->hidden / 8, out_vecs = (int)pad_cols(lm) / 8;
  if (tokens <= kRowsOneLaunch) {
    const int twice = lse && halves(tokens) == 2;
    const unsigned rows = (unsigned)tile_rows(tokens);
    auto run = [&](auto kernel, int threads, auto *ids) {
      return launch(kernel, rows, threads, 0, st, ids, n, lm->vocab, w.rows, lse, d_loss, lm->logit_scale, loss_out, lse_out, lm->d_status, src,
                    dst, row_vecs, out_vecs, twice, wt);
    };
    if (few_rows(tokens))
      return id_bytes == 8 ? run(lm_rows_kernel<long long, kLmFew>, kLmFew, ids64) : run(lm_rows_kernel<int, kLmFew>, kLmFew, ids32);
    return id_bytes == 8 ? run(lm_rows_kernel<long long, kRowsOneLaunch>, kRowsOneLaunch, ids64)
                         : run(lm_rows_kernel<int, kRowsOneLaunch>, kRowsOneLaunch, ids32);
  }
  const int r = id_bytes == 8 ? launch(lm_compact_kernel<long long>, 1, 1024, 0, st, ids64, n, lm->vocab, w.rows, lse, d_loss, lm->logit_scale,
                                       loss_out, lse_out, lm->d_status)
                              : launch(lm_compact_kernel<int>, 1, 1024, 0, st, ids32, n, lm->vocab, w.rows, lse, d_loss, lm->logit_scale,
                                       loss_out, lse_out, lm->d_status);
  if (r) return r;
  const unsigned grid = (unsigned)std::min<int64_t>(up(tokens, 256), 8 * lm->n_lanes);
  return launch(lm_gather_kernel, grid, 256, 0, st, src, w.rows, dst, row_vecs, out_vecs, wt, lse, lm->logit_scale);
}

LmParams base_params(const augtree_lm *lm, const LossWs &w, int64_t rows_pad) {
  LmParams p = {};
  p.n_rows = w.rows.n_rows;
  p.vocab = lm->vocab; p.hidden = lm->hidden;
  p.rows_pad = rows_pad;
  p.halves = 1;
  p.scale_log2 = lm->logit_scale * 1.4426950408889634f;
  p.target = w.rows.target; p.lse2 = w.rows.lse2; p.gscale = w.rows.gscale; p.gtarget = w.rows.x_target;
  p.status = lm->d_status;
  p.wait_budget = (lm->flags & AUGTREE_FLAG_TEST_SHORT_WAIT) ? kWaitBudgetClocksTest : kWaitBudgetClocks;
  p.test_flags = (lm->flags & AUGTREE_FLAG_TEST_SKIP_FWD_LOAD) ? TEST_SKIP_FWD_LOAD : 0;
  return p;
}

struct Maps { CUtensorMap h, w, g, h_mn, w_mn, g_mn, out, dh; };

int launch_tiles(const augtree_lm *lm, const Maps &m, const LmParams &p, cudaStream_t st) {
  return launch(lm_tile_kernel, std::max(lm->n_lanes / 2, 1) * 2, kLmThreads, LmSmem::kBytes, st, m.h, m.w, m.g, m.h_mn, m.w_mn, m.g_mn, m.out,
                m.dh, p);
}

template <int KIND, int N>
int launch_few_n(const augtree_lm *lm, const CUtensorMap &mw, const CUtensorMap &mb, const FewParams &p, cudaStream_t st) {
  return launch(lm_few_kernel<KIND, N>, lm->n_lanes, kFewThreads, FewSmem<KIND, N>::kBytes, st, mw, mb, p);
}
// calls f with the row count as a compile-time constant
template <class F>
int with_few(int few, F f) {
  switch (few) {
    case 16: return f(std::integral_constant<int, 16>{});
    case 32: return f(std::integral_constant<int, 32>{});
    case 48: return f(std::integral_constant<int, 48>{});
    case 64: return f(std::integral_constant<int, 64>{});
    case 80: return f(std::integral_constant<int, 80>{});
    case 96: return f(std::integral_constant<int, 96>{});
    case 112: return f(std::integral_constant<int, 112>{});
    default: return f(std::integral_constant<int, 128>{});
  }
}
template <int KIND>
int launch_few(const augtree_lm *lm, int few, const CUtensorMap &mw, const CUtensorMap &mb, const FewParams &p, cudaStream_t st) {
  return with_few(few, [&](auto n) { return launch_few_n<KIND, decltype(n)::value>(lm, mw, mb, p, st); });
}
template <int KIND>
int few_attributes() {
  for (int few = 16; few <= kLmFew; few += 16) {
    const int r = with_few(few, [](auto n) {
      constexpr int N = decltype(n)::value;
      return cudaFuncSetAttribute(lm_few_kernel<KIND, N>, cudaFuncAttributeMaxDynamicSharedMemorySize, FewSmem<KIND, N>::kBytes) == cudaSuccess
                 ? AUGTREE_OK : AUGTREE_ERR_CUDA;
    });
    if (r) return r;
  }
  return AUGTREE_OK;
}

FewParams few_params(const augtree_lm *lm, const LossWs &w, const LmParams &b) {
  FewParams p = {};
  p.n_rows = b.n_rows; p.vocab = b.vocab; p.hidden = b.hidden; p.scale_log2 = b.scale_log2;
  p.target = b.target; p.lse2 = b.lse2; p.gscale = b.gscale; p.gtarget = b.gtarget;
  p.part = w.part; p.tlogit = w.tlogit; p.grad = w.grad; p.dh_part = w.dh_part;
  p.status = b.status; p.wait_budget = b.wait_budget; p.test_flags = b.test_flags;
  return p;
}

template <typename Id, typename In>
int embed_fwd_out(const augtree_lm *lm, const void *table, const void *ids, int tokens, void *out, int out_dtype, cudaStream_t st) {
  const unsigned grid = (unsigned)std::min<int64_t>(tokens, 32ll * lm->n_lanes);
  const In *tb = static_cast<const In *>(table);
  const Id *id = static_cast<const Id *>(ids);
  auto run = [&](auto *o) {
    return launch(embed_fwd_kernel<Id, In, std::remove_pointer_t<decltype(o)>>, grid, 128, 0, st, tb, id, tokens, lm->vocab, lm->hidden,
                  lm->embed_scale, o, lm->d_status);
  };
  if (out_dtype == AUGTREE_BF16) return run(static_cast<__nv_bfloat16 *>(out));
  if (out_dtype == AUGTREE_F16) return run(static_cast<__half *>(out));
  return run(static_cast<float *>(out));
}

template <typename Id>
int embed_fwd_in(const augtree_lm *lm, const void *table, int table_dtype, const void *ids, int tokens, void *out, int out_dtype, cudaStream_t st) {
  if (table_dtype == AUGTREE_BF16) return embed_fwd_out<Id, __nv_bfloat16>(lm, table, ids, tokens, out, out_dtype, st);
  if (table_dtype == AUGTREE_F16) return embed_fwd_out<Id, __half>(lm, table, ids, tokens, out, out_dtype, st);
  return embed_fwd_out<Id, float>(lm, table, ids, tokens, out, out_dtype, st);
}

// Tokens sorted by id into w.key[*src], w.val[*src].
template <typename Id>
int embed_sort(const augtree_lm *lm, const Id *ids, int n, int passes, int bits, const EmbedWs &w, int *src, cudaStream_t st) {
  int r;
  *src = 0;
  if (n <= kSortSmall && lm->vocab <= (1 << 20)) {  // (a larger vocabulary's bits are cleared by more than one block)
    return launch(embed_sort_small_kernel<Id>, 1, 512, kSortSmallBytes, st, ids, n, lm->vocab, passes, bits, w.key[0], w.val[0], w.joins,
                  w.seen, lm->d_status);
  }
  const int blocks = (n + kRadixBlock - 1) / kRadixBlock;
  const KeysFromIds<Id> from_ids{ids, lm->vocab, lm->d_status};
  for (int i = 0; i < passes; ++i) {
    const KeysSorted sorted{w.key[*src], w.val[*src]};
    const int to = i == 0 ? 0 : *src ^ 1;
    if (i == 0) r = launch(embed_hist_kernel<KeysFromIds<Id>>, blocks, kRadixThreads, 0, st, from_ids, n, 0, bits, w.hist, blocks, w.seen,
                           (lm->vocab + 31) / 32);
    else r = launch(embed_hist_kernel<KeysSorted>, blocks, kRadixThreads, 0, st, sorted, n, i * bits, bits, w.hist, blocks, nullptr, 0);
    if (r) return r;
    if ((r = launch(embed_scan_kernel, ((1 << bits) + 7) / 8, 256, 0, st, w.hist, blocks, 1 << bits, w.total))) return r;
    if (i == 0) r = launch(embed_scatter_kernel<KeysFromIds<Id>>, blocks, kRadixThreads, 0, st, from_ids, n, 0, bits, w.hist, blocks, w.total,
                           w.key[to], w.val[to]);
    else r = launch(embed_scatter_kernel<KeysSorted>, blocks, kRadixThreads, 0, st, sorted, n, i * bits, bits, w.hist, blocks, w.total,
                    w.key[to], w.val[to]);
    if (r) return r;
    *src = to;
  }
  return launch(embed_mark_kernel, (unsigned)((n + 255) / 256), 256, 0, st, w.key[*src], n, lm->vocab, w.seen, w.joins);
}

template <typename In, typename Out>
int embed_sum_out(const augtree_lm *lm, const void *d_out, const EmbedWs &w, int src, int n, void *d_table, int accumulate, cudaStream_t st) {
  const unsigned zero_blocks = accumulate ? 0u : (unsigned)((lm->vocab + kEmbedZeroRows - 1) / kEmbedZeroRows);
  Out *dt = static_cast<Out *>(d_table);
  if (w.n_chunks + zero_blocks == 0) return AUGTREE_OK;
  const int vecs = lm->hidden / 8, slabs = (vecs + kEmbedMaxThreads - 1) / kEmbedMaxThreads;
  const int threads = (int)up((vecs + slabs - 1) / slabs, 32);
  int r = launch(embed_sum_kernel<In, Out>, dim3(w.n_chunks + zero_blocks, slabs), threads, 0, st, static_cast<const In *>(d_out), w.key[src],
                 w.val[src], n, w.chunk, w.n_chunks, lm->vocab, lm->hidden, lm->embed_scale, accumulate, dt, w.part, w.joins, w.seen);
  if (r || w.n_chunks < 2) return r;
  const unsigned grid = (unsigned)std::min<int64_t>((int64_t)(w.n_chunks - 1) * ((lm->hidden + 255) / 256), 8 * lm->n_lanes);
  return launch(embed_join_kernel<Out>, grid, 256, 0, st, w.key[src], w.chunk, w.n_chunks, lm->hidden, lm->embed_scale, accumulate, dt, w.part,
                w.joins);
}

template <typename In>
int embed_sum(const augtree_lm *lm, const void *d_out, const EmbedWs &w, int src, int n, void *d_table, int dtype, int accumulate, cudaStream_t st) {
  if (dtype == AUGTREE_BF16) return embed_sum_out<In, __nv_bfloat16>(lm, d_out, w, src, n, d_table, accumulate, st);
  if (dtype == AUGTREE_F16) return embed_sum_out<In, __half>(lm, d_out, w, src, n, d_table, accumulate, st);
  return embed_sum_out<In, float>(lm, d_out, w, src, n, d_table, accumulate, st);
}

}  // namespace

extern "C" {

int augtree_lm_create(const augtree_lm_desc_t *desc, int device, augtree_lm_t **out) {
  if (!out) return AUGTREE_ERR_INVALID_ARG;
  *out = nullptr;
  if (!desc || desc->struct_size != sizeof(augtree_lm_desc_t) || desc->version != AUGTREE_VERSION) return AUGTREE_ERR_INVALID_ARG;
  if (desc->vocab < 1 || desc->hidden < 1 || desc->n_lanes < 0 || desc->piece_bytes < 0) return AUGTREE_ERR_INVALID_ARG;
  if (!(desc->embed_scale - desc->embed_scale == 0.f) || !(desc->logit_scale - desc->logit_scale == 0.f)) return AUGTREE_ERR_INVALID_ARG;
  if (desc->hidden % 8 != 0 || desc->hidden > (1 << 20) || desc->vocab > (1 << 27) || desc->n_lanes > kMaxLanes) return AUGTREE_ERR_UNSUPPORTED;
  if (device < 0 && desc->n_lanes < 1) return AUGTREE_ERR_INVALID_ARG;
  augtree_lm *lm = new (std::nothrow) augtree_lm();
  if (!lm) return AUGTREE_ERR_INTERNAL;
  lm->vocab = desc->vocab; lm->hidden = desc->hidden; lm->flags = desc->flags; lm->n_lanes = desc->n_lanes;
  lm->embed_scale = desc->embed_scale == 0.f ? 1.f : desc->embed_scale;
  lm->logit_scale = desc->logit_scale == 0.f ? 1.f : desc->logit_scale;
  lm->piece_bytes = desc->piece_bytes;
  lm->device = device;
  int r = AUGTREE_OK;
  if (device >= 0) {
    int prev = 0;
    cudaGetDevice(&prev);
    if (cudaSetDevice(device) != cudaSuccess) r = AUGTREE_ERR_CUDA;
    if (!r) {
      int sms = 0;
      if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || sms < 1) r = AUGTREE_ERR_CUDA;
      else if (lm->n_lanes == 0) lm->n_lanes = sms;
    }
    if (!r && cudaFuncSetAttribute(lm_tile_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, LmSmem::kBytes) != cudaSuccess) r = AUGTREE_ERR_CUDA;
    if (!r && !(r = few_attributes<LM_STATS>()) && !(r = few_attributes<LM_GRAD>())) r = few_attributes<LM_DH>();
    if (!r && (cudaFuncSetAttribute(embed_sort_small_kernel<int>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSortSmallBytes) != cudaSuccess ||
               cudaFuncSetAttribute(embed_sort_small_kernel<long long>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSortSmallBytes) != cudaSuccess))
      r = AUGTREE_ERR_CUDA;
    if (!r && (cudaMalloc(&lm->d_status, 2 * sizeof(int)) != cudaSuccess || cudaMemset(lm->d_status, 0, 2 * sizeof(int)) != cudaSuccess)) r = AUGTREE_ERR_CUDA;
    cudaSetDevice(prev);
  }
  if (r) {
    augtree_lm_destroy(lm);
    if (r == AUGTREE_ERR_CUDA) cuda_failed();
    return r;
  }
  *out = lm;
  return AUGTREE_OK;
}

int augtree_lm_destroy(augtree_lm_t *lm) {
  if (!lm) return AUGTREE_ERR_INVALID_ARG;
  if (lm->device >= 0) {
    const RelaxedCapture relaxed;
    int prev = 0;
    cudaGetDevice(&prev);
    cudaSetDevice(lm->device);
    cudaFree(lm->d_status);
    cudaSetDevice(prev);
  }
  delete lm;
  return AUGTREE_OK;
}

int augtree_lm_workspace_bytes(const augtree_lm_t *lm, int64_t n_tokens, size_t *loss_fwd, size_t *loss_bwd, size_t *embed_bwd) {
  if (!lm || n_tokens < 0) return AUGTREE_ERR_INVALID_ARG;
  if (n_tokens > kMaxTokens) return AUGTREE_ERR_UNSUPPORTED;
  LossWs l;
  EmbedWs e;
  if (loss_fwd) *loss_fwd = loss_layout(lm, n_tokens, false, nullptr, &l, true);
  if (loss_bwd) *loss_bwd = loss_layout(lm, n_tokens, true, nullptr, &l, true);
  if (embed_bwd) *embed_bwd = embed_layout(lm, n_tokens, nullptr, &e, true);
  return AUGTREE_OK;
}

int augtree_embed_fwd(const augtree_lm_t *lm, const void *table, int table_dtype, const void *ids, int id_bytes, int64_t n_tokens,
                      void *out, int out_dtype, void *stream) {
  int r = check_lm(lm);
  if (r) return r;
  if (n_tokens < 0 || (id_bytes != 4 && id_bytes != 8) || !dtype_ok(table_dtype) || !dtype_ok(out_dtype)) return AUGTREE_ERR_INVALID_ARG;
  if (n_tokens > kMaxTokens) return AUGTREE_ERR_UNSUPPORTED;
  if (n_tokens == 0) return AUGTREE_OK;
  if (!table || !ids || !out || !aligned16(table) || !aligned16(out) || !aligned(ids, id_bytes)) return AUGTREE_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return id_bytes == 8 ? embed_fwd_in<long long>(lm, table, table_dtype, ids, (int)n_tokens, out, out_dtype, st)
                       : embed_fwd_in<int>(lm, table, table_dtype, ids, (int)n_tokens, out, out_dtype, st);
}

int augtree_embed_bwd(const augtree_lm_t *lm, const void *d_out, int out_dtype, const void *ids, int id_bytes, int64_t n_tokens,
                      void *d_table, int table_dtype, int accumulate, void *ws, size_t ws_bytes, void *stream) {
  int r = check_lm(lm);
  if (r) return r;
  if (n_tokens < 0 || (id_bytes != 4 && id_bytes != 8) || !dtype_ok(table_dtype) || !dtype_ok(out_dtype)) return AUGTREE_ERR_INVALID_ARG;
  if (n_tokens > kMaxTokens || (accumulate && table_dtype != AUGTREE_F32)) return AUGTREE_ERR_UNSUPPORTED;
  if (!d_table || !aligned16(d_table) || (n_tokens > 0 && (!d_out || !ids || !aligned16(d_out) || !aligned(ids, id_bytes)))) return AUGTREE_ERR_INVALID_ARG;
  EmbedWs w;
  if (!ws || !aligned16(ws) || ws_bytes < embed_layout(lm, n_tokens, static_cast<uint8_t *>(ws), &w)) return AUGTREE_ERR_WORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int n = (int)n_tokens;
  int key_bits = 1;
  while ((lm->vocab >> key_bits) != 0) ++key_bits;
  const int passes = (key_bits + 8) / 9, bits = (key_bits + passes - 1) / passes;
  int src = 0;
  if (n > 0) {
    r = id_bytes == 8 ? embed_sort(lm, static_cast<const long long *>(ids), n, passes, bits, w, &src, st)
                      : embed_sort(lm, static_cast<const int *>(ids), n, passes, bits, w, &src, st);
    if (r) return r;
  }
  if (out_dtype == AUGTREE_BF16) return embed_sum<__nv_bfloat16>(lm, d_out, w, src, n, d_table, table_dtype, accumulate, st);
  if (out_dtype == AUGTREE_F16) return embed_sum<__half>(lm, d_out, w, src, n, d_table, table_dtype, accumulate, st);
  return embed_sum<float>(lm, d_out, w, src, n, d_table, table_dtype, accumulate, st);
}

int augtree_lm_loss_fwd(const augtree_lm_t *lm, const void *hidden, const void *weight, const void *targets, int id_bytes,
                        int64_t n_tokens, float *loss, float *lse, void *ws, size_t ws_bytes, void *stream) {
  int r = check_lm(lm);
  if (r) return r;
  if (n_tokens < 0 || (id_bytes != 4 && id_bytes != 8)) return AUGTREE_ERR_INVALID_ARG;
  if (n_tokens > kMaxTokens) return AUGTREE_ERR_UNSUPPORTED;
  if (n_tokens == 0) return AUGTREE_OK;
  if (!hidden || !weight || !targets || !loss || !lse || !aligned16(hidden) || !aligned16(weight)) return AUGTREE_ERR_INVALID_ARG;
  if (!aligned(targets, id_bytes) || !aligned(loss, 4) || !aligned(lse, 4)) return AUGTREE_ERR_INVALID_ARG;
  LossWs w;
  if (!ws || !aligned16(ws) || ws_bytes < loss_layout(lm, n_tokens, false, static_cast<uint8_t *>(ws), &w)) return AUGTREE_ERR_WORKSPACE;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int64_t rp = tile_rows(n_tokens);
  const int few = few_rows(n_tokens);
  Maps m = {};
  if (few) {
    FewParams p = few_params(lm, w, base_params(lm, w, few));
    p.n = lm->vocab;
    p.ids = targets; p.id_bytes = id_bytes; p.tokens = (int)n_tokens;
    if ((r = map_2d(&m.h, hidden, n_tokens, lm->hidden, few)) || (r = map_2d(&m.w, weight, lm->vocab, lm->hidden, 128))) return r;
    if ((r = launch_few<LM_STATS>(lm, few, m.w, m.h, p, st))) return r;
    auto finish = [&](auto kernel, auto *ids) {
      return launch(kernel, (unsigned)n_tokens, 256, 0, st, w.part, 4 * lm->n_lanes, ids, lm->vocab, static_cast<const uint4 *>(hidden),
                    static_cast<const uint4 *>(weight), lm->hidden / 8, w.tlogit, lm->logit_scale, loss, lse, lm->d_status);
    };
    return id_bytes == 8 ? finish(lm_few_finish_kernel<long long>, static_cast<const long long *>(targets))
                         : finish(lm_few_finish_kernel<int>, static_cast<const int *>(targets));
  }
  if ((r = compact(lm, targets, id_bytes, n_tokens, hidden, weight, w, nullptr, nullptr, loss, lse, st))) return r;
  if ((r = map_2d(&m.h, w.h, rp, pad_cols(lm), 128)) || (r = map_2d(&m.w, weight, lm->vocab, lm->hidden, 128))) return r;
  LmParams p = base_params(lm, w, rp);
  p.n_jobs = 1;
  p.job[0] = {LM_STATS, 0, lm->vocab, lm->hidden, 1, row_group(lm, rp)};
  p.part = w.part; p.tlogit = w.tlogit;
  if ((r = launch_tiles(lm, m, p, st))) return r;
  const unsigned grid = (unsigned)std::min<int64_t>((n_tokens + 31) / 32, 2 * lm->n_lanes);
  return launch(lm_finish_kernel, grid, 1024, 0, st, w.part, n_part(lm), rp, w.rows, w.tlogit, lm->logit_scale, loss, lse);
}

int augtree_lm_loss_bwd(const augtree_lm_t *lm, const void *hidden, const void *weight, const void *targets, int id_bytes,
                        const float *lse, const float *d_loss, int64_t n_tokens, void *d_hidden, void *d_weight,
                        int weight_dtype, int accumulate, void *ws, size_t ws_bytes, void *stream) {
  int r = check_lm(lm);
  if (r) return r;
  if (n_tokens < 0 || (id_bytes != 4 && id_bytes != 8)) return AUGTREE_ERR_INVALID_ARG;
  if (d_weight && weight_dtype != AUGTREE_BF16 && weight_dtype != AUGTREE_F32) return AUGTREE_ERR_INVALID_ARG;
  if (n_tokens > kMaxTokens || (d_weight && accumulate && weight_dtype != AUGTREE_F32)) return AUGTREE_ERR_UNSUPPORTED;
  if (!aligned16(d_hidden) || !aligned16(d_weight)) return AUGTREE_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (n_tokens == 0) {
    if (d_weight && !accumulate &&
        cudaMemsetAsync(d_weight, 0, (size_t)lm->vocab * lm->hidden * (weight_dtype == AUGTREE_F32 ? 4 : 2), st) != cudaSuccess)
      return cuda_failed();
    return AUGTREE_OK;
  }
  if (!hidden || !weight || !targets || !lse || !d_loss || !aligned16(hidden) || !aligned16(weight)) return AUGTREE_ERR_INVALID_ARG;
  if (!aligned(targets, id_bytes) || !aligned(lse, 4) || !aligned(d_loss, 4)) return AUGTREE_ERR_INVALID_ARG;
  LossWs w;
  if (!ws || !aligned16(ws) || ws_bytes < loss_layout(lm, n_tokens, true, static_cast<uint8_t *>(ws), &w)) return AUGTREE_ERR_WORKSPACE;
  if (!d_hidden && !d_weight) return AUGTREE_OK;
  const int few = few_rows(n_tokens), half = halves(n_tokens);
  const int64_t rp = tile_rows(n_tokens), gr = rp * half, cols = piece_cols(lm, gr);
  const int splits = few ? few_splits(lm, cols) : dh_splits(lm, rp, half, cols), chunks = lm->hidden % 64 == 0 ? 2 : 1;
  if ((r = compact(lm, targets, id_bytes, n_tokens, hidden, weight, w, lse, d_loss, nullptr, nullptr, st))) return r;
  Maps m = {};
  if ((r = map_2d(&m.h, w.h, gr, pad_cols(lm), few ? few : 128)) || (r = map_2d(&m.w, weight, lm->vocab, lm->hidden, 128)) ||
      (r = map_mn(&m.h_mn, w.h, gr, pad_cols(lm), 2)) || (r = map_mn(&m.w_mn, weight, lm->vocab, lm->hidden, chunks)) ||
      (r = map_2d(&m.g, w.grad, gr, cols, few ? 2 * few : 128)) || (r = map_mn(&m.g_mn, w.grad, gr, cols, 2)))
    return r;
  LmParams p = base_params(lm, w, rp);
  p.mn_chunks = chunks;
  p.halves = half;
  p.grad_lo = w.grad + rp * cols; p.ld_grad = cols;
  p.dw_f32 = weight_dtype == AUGTREE_F32; p.dw_add = accumulate;
  CUtensorMap out_g, out_dw;
  if (!few && ((r = map_out(&out_g, w.grad, gr, cols, false)) || (r = map_out(&m.dh, w.dh_part, splits * rp, lm->hidden, true)))) return r;
  if (d_weight && (r = map_out(&out_dw, d_weight, lm->vocab, lm->hidden, p.dw_f32))) return r;
  FewParams f = few_params(lm, w, p);
  f.ld_grad = cols; f.splits = splits; f.mn_chunks = chunks;
  for (int64_t v0 = 0; v0 < lm->vocab; v0 += cols) {
    const int n = (int)std::min<int64_t>(cols, lm->vocab - v0);
    p.v0 = f.v0 = (int)v0;
    p.dh_add = f.dh_add = v0 > 0;
    f.n = n;
    p.n_jobs = 0;
    p.half_k = (int)up(n, 64);
    if (few) {
      if ((r = launch_few<LM_GRAD>(lm, few, m.w, m.h, f, st))) return r;
      if (d_hidden && (r = launch_few<LM_DH>(lm, few, m.w_mn, m.g, f, st))) return r;
    } else {
      p.n_jobs = 1;
      p.job[0] = {LM_GRAD, 0, n, lm->hidden, 1, row_group(lm, rp)};
      m.out = out_g;
      if ((r = launch_tiles(lm, m, p, st))) return r;
      p.n_jobs = 0;
      if (d_hidden) p.job[p.n_jobs++] = {LM_DH, 0, lm->hidden, half * p.half_k, splits, 0};
    }
    // (with two halves of G the rows of the packed hidden states are there twice)
    if (d_weight) p.job[p.n_jobs++] = {LM_DW, n, lm->hidden, half == 2 ? (int)gr : 0, 1, 0};
    if (d_weight) m.out = out_dw;
    if (p.n_jobs && (r = launch_tiles(lm, m, p, st))) return r;
  }
  if (d_hidden) {
    const unsigned grid = (unsigned)std::min<int64_t>(n_tokens, 16 * lm->n_lanes);
    return launch(lm_dh_kernel, grid, 256, 0, st, w.dh_part, splits, rp, lm->hidden, w.rows.pos, (int)n_tokens,
                  static_cast<__nv_bfloat16 *>(d_hidden));
  }
  return AUGTREE_OK;
}

int augtree_lm_last_device_status(const augtree_lm_t *lm, int *status, int *detail) {
  if (!lm || lm->device < 0 || !status) return AUGTREE_ERR_INVALID_ARG;
  int prev = 0;
  cudaGetDevice(&prev);
  cudaSetDevice(lm->device);
  int h[2] = {0, 0};
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpy(h, lm->d_status, sizeof(h), cudaMemcpyDeviceToHost);
  if (e == cudaSuccess && (h[0] || h[1])) e = cudaMemset(lm->d_status, 0, sizeof(h));
  cudaSetDevice(prev);
  if (e != cudaSuccess) return cuda_failed();
  *status = h[0];
  if (detail) *detail = h[1];
  return AUGTREE_OK;
}

}  // extern "C"
