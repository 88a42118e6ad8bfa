// C-ABI entry points of a decoder block's ends, of the 8-bit activation checkpoints and of what reads them in the backward pass.
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <initializer_list>
#include <new>
#include <type_traits>

#include "act_kernels.cuh"
#include "block_kernels.cuh"
#include "handle.h"
#include "wgrad_kernel.cuh"
#include "../../include/augtree.h"

using namespace augtree;

static_assert((int)T_BF16 == (int)AUGTREE_BF16 && (int)T_F16 == (int)AUGTREE_F16 && (int)T_F32 == (int)AUGTREE_F32 && (int)T_CKPT == AUGTREE_CKPT, "type codes");
static_assert((int)GATE_NONE == (int)AUGTREE_GATE_NONE && (int)GATE_TOKEN == (int)AUGTREE_GATE_TOKEN &&
              (int)GATE_CHANNEL == (int)AUGTREE_GATE_CHANNEL && (int)GATE_FULL == (int)AUGTREE_GATE_FULL, "gate codes");

struct augtree_block {
  int32_t hidden = 0;
  float eps = 1e-6f, scale = 1.f;
  int32_t gate = 0, sigmoid = 0;
  uint32_t flags = 0;
  int32_t n_lanes = 0;
  int device = -1;
  int *d_status = nullptr;  // status, detail
};

namespace {

constexpr int64_t kMaxCols = 1 << 20;

int size_of(int type) { return type == AUGTREE_F32 ? 4 : 2; }

int check_block(const augtree_block *b) {
  if (!b || b->device < 0) return AUGTREE_ERR_INVALID_ARG;
  int cur = -1;
  if (cudaGetDevice(&cur) != cudaSuccess) return cuda_failed();
  return cur == b->device ? AUGTREE_OK : AUGTREE_ERR_INVALID_ARG;
}

// tokens and columns of a tensor of its own width
int check_size(int64_t n, int64_t cols) {
  if (n < 0 || cols < 1) return AUGTREE_ERR_INVALID_ARG;
  return n > kMaxTokens || cols % 8 != 0 || cols > kMaxCols ? AUGTREE_ERR_UNSUPPORTED : AUGTREE_OK;
}

// Leading size of a matrix in elements: 0 stands for its columns.
bool ld_ok(int64_t &ld, int64_t cols) {
  if (ld == 0) ld = cols;
  return ld >= cols && ld % 8 == 0;
}

// The walk over matrices of `cols` columns (act_kernels.cuh) and its grid: as many blocks as the SMs hold at a time.
struct Matrix { const void *p; int64_t ld; int bytes; };    // bytes of an element
Pieces pieces(const augtree_block *b, int64_t rows, int64_t cols, int blocks, std::initializer_list<Matrix> all, unsigned *grid) {
  Pieces p;
  p.per_row = (int)(up(cols, 32) / 16);
  p.valid = (int)(cols / 8);
  p.total = rows * p.per_row;
  p.inv = ~0ull / (unsigned long long)p.per_row + 1;   // (per_row is at least 2; where it divides 2^64 this is the quotient)
  p.wide = true;
  for (const Matrix &m : all) p.wide = p.wide && aligned(m.p, 32) && m.ld * m.bytes % 32 == 0;
  *grid = (unsigned)std::min<int64_t>((p.total + kActThreads - 1) / kActThreads, (int64_t)blocks * b->n_lanes);
  const int64_t step = (int64_t)*grid * kActThreads;
  p.step_rows = step / p.per_row;
  p.step_pieces = (int)(step % p.per_row);
  return p;
}
CkptRows ckpt_rows(const void *p, int64_t cols) { return {static_cast<uint8_t *>(const_cast<void *>(p)), ckpt_pitch(cols), ckpt_scale_offset(cols)}; }

// calls f with a null pointer of the type
template <class F>
int with_type(int type, F f) {
  if (type == AUGTREE_BF16) return f(static_cast<__nv_bfloat16 *>(nullptr));
  if (type == AUGTREE_F16) return f(static_cast<__half *>(nullptr));
  return f(static_cast<float *>(nullptr));
}

// ---------------------------------------------------------------- block ends
// Pieces of 8 columns of a thread (kParts): one for rows that a warp covers with them, two otherwise, four forward with a 16-bit stream: the more, the
// fewer warps share a row and the less its reductions and addresses cost (16384 x 3584 bf16 with checkpoints, forward: 130 us with two, 109 with four), but an
// fp32 stream, whose rows are as near to memory's rate with two, takes the stages that more groups need (a pass of 24576 x 3584 in both directions: 414 us with
// two, 443 with four).
// The backward pass keeps its sums over tokens in registers, which leave no room for more than two.
int fwd_parts(int hidden, int x) { return hidden <= 256 ? 1 : x == T_BF16 ? 4 : 2; }
int bwd_parts(int hidden) { return hidden <= 256 ? 1 : 2; }
bool wide_bwd(int hidden) { return hidden > kBlockBwdWarps * 512; }

// calls f with the kernel for a width, a stream type (kAny: types looked up), a form of the call and a gate
template <int P, int X, class F>
int with_fwd_form(int form, int gate, F f) {
  if (form == kBefore) return f(block_fwd_kernel<P, X, T_BF16, kBefore, GATE_NONE>);
  if (gate == GATE_NONE) return f(block_fwd_kernel<P, X, T_BF16, kBoth, GATE_NONE>);
  if (gate == GATE_TOKEN) return f(block_fwd_kernel<P, X, T_BF16, kBoth, GATE_TOKEN>);
  if (gate == GATE_CHANNEL) return f(block_fwd_kernel<P, X, T_BF16, kBoth, GATE_CHANNEL>);
  return f(block_fwd_kernel<P, X, T_BF16, kBoth, GATE_FULL>);
}
template <int P, class F>
int with_fwd_types(int x, int form, int gate, F f) {
  if constexpr (P != 4) {
    if (x == T_F32) return with_fwd_form<P, T_F32>(form, gate, f);
    if (x == kAny) return f(block_fwd_kernel<P, kAny, kAny, kAny, kAny>);
  }
  if constexpr (P != 2) return with_fwd_form<P, T_BF16>(form, gate, f);
  return AUGTREE_ERR_INTERNAL;
}
template <class F>
int with_fwd(int hidden, int x, int form, int gate, F f) {
  switch (fwd_parts(hidden, x)) {
    case 1: return with_fwd_types<1>(x, form, gate, f);
    case 2: return with_fwd_types<2>(x, form, gate, f);
    default: return with_fwd_types<4>(x, form, gate, f);
  }
}
template <int P, int X, bool kKept, class F>
int with_bwd_form(int form, int gate, F f) {
  constexpr int W = kBlockBwdWarps;
  if (form == kBefore) return f(block_bwd_kernel<P, W, X, T_BF16, kBefore, GATE_NONE, kKept>);
  if (gate == GATE_NONE) return f(block_bwd_kernel<P, W, X, T_BF16, kBoth, GATE_NONE, kKept>);
  if (gate == GATE_TOKEN) return f(block_bwd_kernel<P, W, X, T_BF16, kBoth, GATE_TOKEN, kKept>);
  if (gate == GATE_CHANNEL) return f(block_bwd_kernel<P, W, X, T_BF16, kBoth, GATE_CHANNEL, kKept>);
  return f(block_bwd_kernel<P, W, X, T_BF16, kBoth, GATE_FULL, kKept>);
}
template <int P, class F>
int with_bwd_types(int x, int form, int gate, bool kept, F f) {
  if (x == T_F32) return kept ? with_bwd_form<P, T_F32, true>(form, gate, f) : with_bwd_form<P, T_F32, false>(form, gate, f);
  if (x == T_BF16) return kept ? with_bwd_form<P, T_BF16, true>(form, gate, f) : with_bwd_form<P, T_BF16, false>(form, gate, f);
  return f(block_bwd_kernel<P, kBlockBwdWarps, kAny, kAny, kAny, kAny, false>);
}
// (rows of more than 7680 columns are always looked up)
template <class F>
int with_bwd(int hidden, int x, int form, int gate, bool kept, F f) {
  if (wide_bwd(hidden)) return f(block_bwd_kernel<2, kBlockBwdWarpsWide, kAny, kAny, kAny, kAny, false>);
  return bwd_parts(hidden) == 1 ? with_bwd_types<1>(x, form, gate, kept, f) : with_bwd_types<2>(x, form, gate, kept, f);
}
// what is there has the branch's usual type
bool bf16_or_none(bool there, int type) { return !there || type == AUGTREE_BF16; }

struct Input { const void *p; int64_t row_bytes; };

// Groups, stages and grid of a call; false if one row of all inputs does not fit shared memory.
bool block_shape(const augtree_block *b, int64_t rows, const Input *in, int n_in, int weights, int max_warps, int parts, BlockShape *s, int *grid, size_t *smem) {
  const int hidden = b->hidden;
  *s = {};
  s->rows = (int)rows; s->hidden = hidden; s->vecs = hidden / 8; s->weights = weights;
  const int warp_vecs = 32 * parts;
  s->warps_row = (s->vecs + warp_vecs - 1) / warp_vecs;
  int64_t row = 0;
  for (int i = 0; i < n_in; ++i) row += in[i].row_bytes;
  const int64_t fixed = kBlockFixed + (int64_t)weights * hidden * 4, room = kBlockSmem - fixed;
  if (row > room) return false;
  // As many groups as leave three stages, or two where two groups would not.
  const int64_t most = max_warps / s->warps_row;
  int64_t groups = std::min<int64_t>(most, std::max<int64_t>(room / (3 * row), std::min<int64_t>(2, room / (2 * row))));
  groups = std::max<int64_t>(groups, 1);
  s->groups = (int)groups;
  // Rows of a stage: one a group, more for narrow rows (a bulk copy of a few KB costs as much as one of 32 KB) as long as every
  // lane still gets eight blocks; fewer than one a group if the rows would not reach all lanes otherwise.
  int64_t per = 1, block = groups;
  if (rows < groups * b->n_lanes) block = std::max<int64_t>((rows + b->n_lanes - 1) / b->n_lanes, 1);
  else while (per < 8 && groups * (per + 1) * row <= 32 << 10 && rows >= groups * (per + 1) * b->n_lanes * 8) block = groups * ++per;
  // As many turns of the lanes as that takes, but no lane has more rows than it has to (2183 x 1032 fp32, blocks of 5 rows instead of 6: forward 9.1 to 8.4 us).
  const int64_t round = (rows + block * b->n_lanes - 1) / (block * b->n_lanes) * b->n_lanes;
  block = (rows + round - 1) / round;
  s->block_rows = (int)block;
  s->blocks = (int)((rows + block - 1) / block);
  int64_t off = 0;
  s->n_inputs = n_in;
  for (int i = 0; i < n_in; ++i) {
    s->input[i] = static_cast<const uint8_t *>(in[i].p);
    s->row_bytes[i] = (int)in[i].row_bytes;
    s->offset[i] = (int)off;
    off += block * in[i].row_bytes;
  }
  s->stage_bytes = (int)off;
  *grid = (int)std::min<int64_t>(b->n_lanes, s->blocks);
  const int64_t turns = (s->blocks + *grid - 1) / *grid;
  s->stages = (int)std::min<int64_t>(std::min<int64_t>(kBlockMaxStages, room / off), turns);
  *smem = (size_t)(fixed + std::max<int64_t>(s->stages * off, groups * 2 * hidden * 4));   // (the backward pass adds up there)
  return true;
}

BlockParams base_params(const augtree_block *b) {
  BlockParams p = {};
  p.inv_hidden = (float)(1.0 / b->hidden); p.eps = b->eps; p.scale = b->scale;
  p.sigmoid = b->sigmoid;
  p.status = b->d_status;
  p.wait_budget = (b->flags & AUGTREE_FLAG_TEST_SHORT_WAIT) ? kWaitBudgetClocksTest : kWaitBudgetClocks;
  p.test_flags = (b->flags & AUGTREE_FLAG_TEST_SKIP_FWD_LOAD) ? TEST_SKIP_FWD_LOAD : 0;
  return p;
}

// A gate belongs to a branch: given exactly if the handle has one.
int check_gate(const augtree_block *b, const void *o, const void *gate, int gate_type) {
  if (b->gate == AUGTREE_GATE_NONE || !o) return gate ? AUGTREE_ERR_INVALID_ARG : AUGTREE_OK;
  if (!gate || !dtype_ok(gate_type)) return AUGTREE_ERR_INVALID_ARG;
  return aligned(gate, b->gate == AUGTREE_GATE_TOKEN ? size_of(gate_type) : 16) ? AUGTREE_OK : AUGTREE_ERR_INVALID_ARG;
}

size_t bwd_bytes(const augtree_block *b) { return (size_t)b->n_lanes * 2 * b->hidden * 4; }

// ---------------------------------------------------------------- weight gradient
// How a call is done: shares of the contraction, and whether X is turned into bf16 in the kernel (kBits, wgrad_kernel.cuh).  By the time of the longest
// CTA pair (a stage of 64 tokens 0.28 us from bf16 and 0.4 from bits, a tile's start and end 2 us), of the partial sums' way through memory (4 us and
// their bytes, written and read, at 6 TB/s) and of a bf16 X's (2 us and its 3 bytes a value).
struct WgradWay { int splits; bool bits; int parts; };    // parts: results of the tensors' size in fp32 that the scratch has room for
WgradWay wgrad_way(int lanes, int64_t n, int64_t out, int64_t cols) {
  const int64_t pairs = std::max(lanes / 2, 1), tiles = ((out + kLmTile - 1) / kLmTile) * ((cols + kLmTile - 1) / kLmTile);
  const int64_t steps = std::max<int64_t>((n + 63) / 64, 1);
  auto cost = [&](int64_t s, bool bits) {
    const double longest = (double)((tiles * s + pairs - 1) / pairs) * ((bits ? 0.4 : 0.28) * (double)((steps + s - 1) / s) + 2.0);
    return longest + (s > 1 ? 4.0 + (double)(s * out * cols) * 8e-6 / 6.0 : 0.0) + (bits ? 0.0 : 2.0 + (double)(n * cols) * 3e-6 / 6.0);
  };
  WgradWay pick = {1, true, 0};
  for (bool bits : {true, false})
    for (int64_t s = 1; s <= std::min<int64_t>(steps, 32); ++s)
      if (cost(s, bits) < cost(pick.splits, pick.bits)) pick = {(int)s, bits, 0};
  const int64_t share = (steps + pick.splits - 1) / pick.splits;
  pick.splits = (int)((steps + share - 1) / share);   // (no empty share)
  pick.parts = pick.splits > 1 || steps > kWgLong ? pick.splits : 0;    // (a call does not say here what its result's type will be)
  return pick;
}

struct WgradWs { __nv_bfloat16 *x; float *part; };
size_t wgrad_layout(const WgradWay &way, int64_t n, int64_t out, int64_t cols, uint8_t *base, WgradWs *w) {
  Cursor c{base};
  w->x = c.take<__nv_bfloat16>(way.bits ? 0 : n * up(cols, 64));
  w->part = c.take<float>(way.parts * up(out, kLmTile) * cols);
  return c.off;
}

}  // namespace

extern "C" {

int augtree_block_create(const augtree_block_desc_t *desc, int device, augtree_block_t **out) {
  if (!out) return AUGTREE_ERR_INVALID_ARG;
  *out = nullptr;
  if (!desc || desc->struct_size != sizeof(augtree_block_desc_t) || desc->version != AUGTREE_VERSION) return AUGTREE_ERR_INVALID_ARG;
  if (desc->hidden < 1 || desc->n_lanes < 0 || desc->gate < AUGTREE_GATE_NONE || desc->gate > AUGTREE_GATE_FULL) return AUGTREE_ERR_INVALID_ARG;
  if (!(desc->eps - desc->eps == 0.f) || desc->eps < 0.f || !(desc->residual_scale - desc->residual_scale == 0.f)) return AUGTREE_ERR_INVALID_ARG;
  if (desc->hidden % 8 != 0 || desc->hidden > kBlockMaxHidden || desc->n_lanes > kMaxLanes) return AUGTREE_ERR_UNSUPPORTED;
  if (device < 0 && desc->n_lanes < 1) return AUGTREE_ERR_INVALID_ARG;
  augtree_block *b = new (std::nothrow) augtree_block();
  if (!b) return AUGTREE_ERR_INTERNAL;
  b->hidden = desc->hidden; b->gate = desc->gate; b->sigmoid = desc->gate_sigmoid != 0; b->flags = desc->flags; b->n_lanes = desc->n_lanes;
  b->eps = desc->eps == 0.f ? 1e-6f : desc->eps;
  b->scale = desc->residual_scale == 0.f ? 1.f : desc->residual_scale;
  b->device = device;
  int r = AUGTREE_OK;
  if (device >= 0) {
    int prev = 0;
    cudaGetDevice(&prev);
    if (cudaSetDevice(device) != cudaSuccess) r = AUGTREE_ERR_CUDA;
    if (!r) {
      int sms = 0;
      if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess || sms < 1) r = AUGTREE_ERR_CUDA;
      else if (b->n_lanes == 0) b->n_lanes = sms;
    }
    auto room = [&](auto kernel, int bytes) {
      if (!r && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) r = AUGTREE_ERR_CUDA;
    };
    // (the kernels that calls with this handle can reach)
    auto kernel_room = [&](auto kernel) { room(kernel, kBlockSmem); return 0; };
    for (int x : {(int)T_F32, (int)T_BF16, kAny})
      for (int form : {(int)kBoth, (int)kBefore}) {
        with_fwd(b->hidden, x, form, b->gate, kernel_room);
        for (bool kept : {false, true}) with_bwd(b->hidden, x, form, b->gate, kept, kernel_room);
      }
    room(wgrad_kernel<true>, WgSmem<true>::kBytes); room(wgrad_kernel<false>, WgSmem<false>::kBytes);
    if (!r && (cudaMalloc(&b->d_status, 2 * sizeof(int)) != cudaSuccess || cudaMemset(b->d_status, 0, 2 * sizeof(int)) != cudaSuccess)) r = AUGTREE_ERR_CUDA;
    cudaSetDevice(prev);
  }
  if (r) {
    augtree_block_destroy(b);
    if (r == AUGTREE_ERR_CUDA) cuda_failed();
    return r;
  }
  *out = b;
  return AUGTREE_OK;
}

int augtree_block_destroy(augtree_block_t *b) {
  if (!b) return AUGTREE_ERR_INVALID_ARG;
  if (b->device >= 0) {
    const RelaxedCapture relaxed;
    int prev = 0;
    cudaGetDevice(&prev);
    cudaSetDevice(b->device);
    cudaFree(b->d_status);
    cudaSetDevice(prev);
  }
  delete b;
  return AUGTREE_OK;
}

int augtree_ckpt_pitch(int64_t cols, int64_t *pitch) {
  if (!pitch || cols < 1) return AUGTREE_ERR_INVALID_ARG;
  if (cols % 8 != 0 || cols > kMaxCols) return AUGTREE_ERR_UNSUPPORTED;
  *pitch = ckpt_pitch(cols);
  return AUGTREE_OK;
}

int augtree_block_workspace_bytes(const augtree_block_t *b, int64_t n_tokens, size_t *bytes) {
  if (!b || !bytes || n_tokens < 0) return AUGTREE_ERR_INVALID_ARG;
  if (n_tokens > kMaxTokens) return AUGTREE_ERR_UNSUPPORTED;
  *bytes = bwd_bytes(b);
  return AUGTREE_OK;
}

int augtree_block_fwd(const augtree_block_t *b, const void *x, int x_dtype, const void *o, int o_dtype, const void *gate, int gate_dtype,
                      const void *w_out, const void *w_in, int w_dtype, int64_t n_tokens, void *y, void *h, int h_dtype, float *r_out,
                      float *r_in, void *ckpt_y, void *ckpt_o, void *stream) {
  int r = check_block(b);
  if (r) return r;
  if (n_tokens < 0 || !dtype_ok(x_dtype) || (o && !dtype_ok(o_dtype)) || ((w_out || w_in) && !dtype_ok(w_dtype)) || (h && !dtype_ok(h_dtype)))
    return AUGTREE_ERR_INVALID_ARG;
  if (n_tokens > kMaxTokens) return AUGTREE_ERR_UNSUPPORTED;
  if (n_tokens == 0) return AUGTREE_OK;     // (tensors of no tokens have no address)
  if (!h != !w_in || (!o && (y || w_out || ckpt_o)) || (o && !y)) return AUGTREE_ERR_INVALID_ARG;
  if (!x || (!o && !h && !ckpt_y)) return AUGTREE_ERR_INVALID_ARG;
  if ((r = check_gate(b, o, gate, gate_dtype))) return r;
  for (const void *q : {x, o, w_out, w_in, (const void *)y, (const void *)h, (const void *)ckpt_y, (const void *)ckpt_o})
    if (!aligned16(q)) return AUGTREE_ERR_INVALID_ARG;
  if (!aligned(r_out, 4) || !aligned(r_in, 4)) return AUGTREE_ERR_INVALID_ARG;
  BlockParams p = base_params(b);
  const int64_t c = b->hidden;
  p.gate = o ? b->gate : GATE_NONE;
  const Input in[3] = {{x, c * size_of(x_dtype)}, {o, o ? c * size_of(o_dtype) : 0}, {gate, p.gate == GATE_FULL ? c * size_of(gate_dtype) : 0}};
  // what is compiled in (block_kernels.cuh): everything of the branch in bf16, a norm before the next block
  const bool usual = h && bf16_or_none(h, h_dtype) && bf16_or_none(o, o_dtype) && bf16_or_none(p.gate == GATE_FULL, gate_dtype) && x_dtype != AUGTREE_F16;
  const int types = usual ? x_dtype : kAny;
  int grid;
  size_t smem;
  if (!block_shape(b, n_tokens, in, o ? p.gate == GATE_FULL ? 3 : 2 : 1, !!w_in + !!w_out + (p.gate == GATE_CHANNEL), kBlockFwdWarps,
                   fwd_parts(b->hidden, types), &p.s, &grid, &smem))
    return AUGTREE_ERR_UNSUPPORTED;
  p.gate_type = gate_dtype; p.gate_ptr = gate;
  p.w_out = w_out; p.w_in = w_in; p.w_type = w_dtype;
  p.r_out = r_out; p.r_in = r_in;
  p.x_type = x_dtype; p.o_type = o_dtype; p.h_type = h_dtype;
  p.has_branch = !!o;
  p.y = y; p.h = h;
  p.ckpt_y = ckpt_rows(ckpt_y, c); p.ckpt_o = ckpt_rows(ckpt_o, c);
  const int threads = (p.s.groups * p.s.warps_row + 1) * 32;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return with_fwd(b->hidden, types, o ? kBoth : kBefore, p.gate, [&](auto kernel) { return launch(kernel, grid, threads, smem, st, p); });
}

int augtree_block_bwd(const augtree_block_t *b, const void *dy, int x_dtype, const void *dh, int h_dtype, const void *y, int y_dtype,
                      const void *o, int o_dtype, const void *gate, int gate_dtype, const void *w_out, const void *w_in, int w_dtype,
                      const float *r_out, const float *r_in, int64_t n_tokens, void *dx, void *d_o, int do_dtype, void *d_gate, void *dw_out,
                      void *dw_in, int accumulate, void *ws, size_t ws_bytes, void *stream) {
  int r = check_block(b);
  if (r) return r;
  auto saved_ok = [](int t) { return dtype_ok(t) || t == AUGTREE_CKPT; };
  if (n_tokens < 0 || !dtype_ok(x_dtype) || (dh && !dtype_ok(h_dtype)) || (y && !saved_ok(y_dtype)) || (o && !saved_ok(o_dtype)) ||
      ((w_out || w_in) && !dtype_ok(w_dtype)) || (d_o && !dtype_ok(do_dtype)))
    return AUGTREE_ERR_INVALID_ARG;
  const int gate_kind = o || n_tokens == 0 ? b->gate : GATE_NONE;
  if ((dw_in && !w_in) || (dw_out && !w_out) || (d_gate && gate_kind == GATE_NONE)) return AUGTREE_ERR_INVALID_ARG;
  const bool channel = gate_kind == GATE_CHANNEL;
  if (n_tokens > kMaxTokens) return AUGTREE_ERR_UNSUPPORTED;
  if (accumulate && (((dw_in || dw_out) && w_dtype != AUGTREE_F32) || (channel && d_gate && gate_dtype != AUGTREE_F32))) return AUGTREE_ERR_UNSUPPORTED;
  for (const void *q : {dy, dh, y, o, w_out, w_in, (const void *)dx, (const void *)d_o, (const void *)dw_out, (const void *)dw_in})
    if (!aligned16(q)) return AUGTREE_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (n_tokens == 0) {
    // sums over no tokens
    if (channel && d_gate && !dtype_ok(gate_dtype)) return AUGTREE_ERR_INVALID_ARG;
    auto zero = [&](void *q, int type) {
      if (q && !accumulate && !r && cudaMemsetAsync(q, 0, (size_t)b->hidden * size_of(type), st) != cudaSuccess) r = cuda_failed();
    };
    zero(dw_in, w_dtype); zero(dw_out, w_dtype);
    if (channel) zero(d_gate, gate_dtype);
    return r;
  }
  if (!dy && !dh) return AUGTREE_ERR_INVALID_ARG;
  if (!dh != !w_in || (dh && (!y || !r_in)) || (!o && (w_out || d_o)) || (w_out && !r_out)) return AUGTREE_ERR_INVALID_ARG;
  if ((r = check_gate(b, o, gate, gate_dtype))) return r;
  if (d_gate && !aligned(d_gate, b->gate == AUGTREE_GATE_TOKEN ? size_of(gate_dtype) : 16)) return AUGTREE_ERR_INVALID_ARG;
  if (!aligned(r_out, 4) || !aligned(r_in, 4)) return AUGTREE_ERR_INVALID_ARG;
  if (!ws || !aligned16(ws) || ws_bytes < bwd_bytes(b)) return AUGTREE_ERR_WORKSPACE;
  BlockParams p = base_params(b);
  const int64_t c = b->hidden;
  p.gate = gate_kind;
  auto row_of = [&](int type) { return type == AUGTREE_CKPT ? ckpt_pitch(c) : c * size_of(type); };
  Input in[kBlockMaxInputs];
  int n_in = 0;
  if (dy) in[n_in++] = {dy, row_of(x_dtype)};
  if (dh) { in[n_in++] = {dh, row_of(h_dtype)}; in[n_in++] = {y, row_of(y_dtype)}; }
  if (o) in[n_in++] = {o, row_of(o_dtype)};
  if (p.gate == GATE_FULL) in[n_in++] = {gate, row_of(gate_dtype)};
  int grid;
  size_t smem;
  if (!block_shape(b, n_tokens, in, n_in, !!w_in + !!w_out + channel, wide_bwd(b->hidden) ? kBlockBwdWarpsWide : kBlockBwdWarps, bwd_parts(b->hidden), &p.s, &grid, &smem)) return AUGTREE_ERR_UNSUPPORTED;
  p.gate_type = gate_dtype; p.gate_ptr = gate;
  p.w_out = w_out; p.w_in = w_in; p.w_type = w_dtype;
  p.r_out = const_cast<float *>(r_out); p.r_in = const_cast<float *>(r_in);
  p.x_type = x_dtype; p.o_type = o_dtype; p.h_type = h_dtype; p.y_type = y_dtype; p.do_type = do_dtype;
  p.has_branch = !!o; p.has_dy = !!dy; p.has_dh = !!dh;
  p.dx = dx; p.d_o = d_o; p.dg = d_gate;
  p.part = static_cast<float *>(ws);
  const int threads = (p.s.groups * p.s.warps_row + 1) * 32;
  const bool kept = y_dtype == AUGTREE_CKPT;
  const bool usual = dy && dh && dx && !o == !d_o && bf16_or_none(dh, h_dtype) && bf16_or_none(d_o, do_dtype) && bf16_or_none(p.gate == GATE_FULL, gate_dtype) && x_dtype != AUGTREE_F16 &&
                     (kept || y_dtype == x_dtype) && (!o || o_dtype == (kept ? AUGTREE_CKPT : (int)AUGTREE_BF16));
  r = with_bwd(b->hidden, usual ? x_dtype : kAny, o ? kBoth : kBefore, p.gate, kept, [&](auto kernel) { return launch(kernel, grid, threads, smem, st, p); });
  const bool second = dw_out || (channel && d_gate);
  if (r || (!dw_in && !second)) return r;
  const BlockSums q = {p.part, grid, b->hidden, w_out, channel ? gate : nullptr, w_dtype, gate_dtype, b->sigmoid, accumulate, dw_in, dw_out, channel ? d_gate : nullptr};
  return launch(block_sums_kernel, dim3((b->hidden + 31) / 32, second ? 2 : 1), 1024, 0, st, q);
}

int augtree_ckpt_pack(const augtree_block_t *b, const void *x, int dtype, int64_t ld, int64_t n_tokens, int64_t cols, void *ckpt, void *stream) {
  int r = check_block(b);
  if (r || (r = check_size(n_tokens, cols))) return r;
  if (!dtype_ok(dtype) || !ld_ok(ld, cols)) return AUGTREE_ERR_INVALID_ARG;
  if (n_tokens == 0) return AUGTREE_OK;
  if (!x || !ckpt || !aligned16(x) || !aligned16(ckpt)) return AUGTREE_ERR_INVALID_ARG;
  unsigned grid;
  const Pieces p = pieces(b, n_tokens, cols, dtype == AUGTREE_F32 ? kPackBlocks<float> : kPackBlocks<__half>, {{x, ld, size_of(dtype)}}, &grid);
  return with_type(dtype, [&](auto *t) {
    using T = std::remove_pointer_t<decltype(t)>;
    return launch(ckpt_pack_kernel<T>, grid, kActThreads, 0, static_cast<cudaStream_t>(stream), static_cast<const T *>(x), ld, p, ckpt_rows(ckpt, cols));
  });
}

int augtree_ckpt_unpack(const augtree_block_t *b, const void *ckpt, int64_t n_tokens, int64_t cols, const float *row, const void *col,
                        int col_dtype, void *out, int dtype, int64_t ld, void *stream) {
  int r = check_block(b);
  if (r || (r = check_size(n_tokens, cols))) return r;
  if (!dtype_ok(dtype) || (col && !dtype_ok(col_dtype)) || !ld_ok(ld, cols)) return AUGTREE_ERR_INVALID_ARG;
  if (n_tokens == 0) return AUGTREE_OK;
  if (!ckpt || !out || !aligned16(ckpt) || !aligned16(out) || !aligned(row, 4) || !aligned16(col)) return AUGTREE_ERR_INVALID_ARG;
  unsigned grid;
  const Pieces p = pieces(b, n_tokens, cols, kUnpackBlocks, {{out, ld, size_of(dtype)}}, &grid);
  return with_type(dtype, [&](auto *t) {
    using T = std::remove_pointer_t<decltype(t)>;
    return launch(ckpt_unpack_kernel<T>, grid, kActThreads, 0, static_cast<cudaStream_t>(stream), ckpt_rows(ckpt, cols), p, (int)(cols / 8), row, col,
                  col_dtype, static_cast<T *>(out), ld);
  });
}

int augtree_glu_fwd(const augtree_block_t *b, const void *g, const void *u, int64_t ld, int dtype, int64_t n_tokens, int64_t cols, void *a,
                    void *ckpt_g, void *ckpt_u, void *stream) {
  int r = check_block(b);
  if (r || (r = check_size(n_tokens, cols))) return r;
  if (!dtype_ok(dtype) || !ld_ok(ld, cols) || !ckpt_g != !ckpt_u) return AUGTREE_ERR_INVALID_ARG;
  if (n_tokens == 0) return AUGTREE_OK;
  if (!g || !u || !a || !aligned16(g) || !aligned16(u) || !aligned16(a) || !aligned16(ckpt_g) || !aligned16(ckpt_u)) return AUGTREE_ERR_INVALID_ARG;
  const int size = size_of(dtype);
  unsigned grid;
  const Pieces p = pieces(b, n_tokens, cols, kGluBlocks, {{g, ld, size}, {u, ld, size}, {a, cols, size}}, &grid);
  return with_type(dtype, [&](auto *t) {
    using T = std::remove_pointer_t<decltype(t)>;
    auto run = [&](auto kernel) {
      return launch(kernel, grid, kActThreads, 0, static_cast<cudaStream_t>(stream), static_cast<const T *>(g), static_cast<const T *>(u), ld, p,
                    static_cast<T *>(a), cols, ckpt_rows(ckpt_g, cols), ckpt_rows(ckpt_u, cols));
    };
    return ckpt_g ? run(glu_fwd_kernel<T, true>) : run(glu_fwd_kernel<T, false>);
  });
}

int augtree_glu_bwd(const augtree_block_t *b, const void *da, int dtype, const void *g, const void *u, int64_t ld, int saved_dtype, int64_t n_tokens,
                    int64_t cols, void *dg, void *du, int64_t ld_grad, void *a, void *stream) {
  int r = check_block(b);
  if (r || (r = check_size(n_tokens, cols))) return r;
  const bool kept = saved_dtype == AUGTREE_CKPT;
  if (!dtype_ok(dtype) || (!kept && saved_dtype != dtype) || !ld_ok(ld, cols) || !ld_ok(ld_grad, cols)) return AUGTREE_ERR_INVALID_ARG;
  if (n_tokens == 0) return AUGTREE_OK;
  if (!da || !g || !u || !dg || !du) return AUGTREE_ERR_INVALID_ARG;
  for (const void *q : {da, g, u, (const void *)dg, (const void *)du, (const void *)a})
    if (!aligned16(q)) return AUGTREE_ERR_INVALID_ARG;
  const int size = size_of(dtype);
  unsigned grid;
  const Pieces p = kept ? pieces(b, n_tokens, cols, kGluBlocks, {{da, cols, size}, {dg, ld_grad, size}, {du, ld_grad, size}, {a, cols, size}}, &grid)
                        : pieces(b, n_tokens, cols, kGluBlocks, {{da, cols, size}, {g, ld, size}, {u, ld, size}, {dg, ld_grad, size}, {du, ld_grad, size},
                                                                     {a, cols, size}}, &grid);
  return with_type(dtype, [&](auto *t) {
    using T = std::remove_pointer_t<decltype(t)>;
    auto run = [&](auto kernel) {
      return launch(kernel, grid, kActThreads, 0, static_cast<cudaStream_t>(stream), static_cast<const T *>(da), static_cast<const T *>(g),
                    static_cast<const T *>(u), ld, ckpt_rows(g, cols), ckpt_rows(u, cols), p, cols, static_cast<T *>(dg), static_cast<T *>(du),
                    ld_grad, static_cast<T *>(a));
    };
    return kept ? run(glu_bwd_kernel<T, true>) : run(glu_bwd_kernel<T, false>);
  });
}

int augtree_ckpt_wgrad_bytes(const augtree_block_t *b, int64_t n_tokens, int64_t out_features, int64_t cols, size_t *bytes) {
  if (!b || !bytes) return AUGTREE_ERR_INVALID_ARG;
  int r = check_size(n_tokens, cols);
  if (r || (r = check_size(n_tokens, out_features))) return r;
  WgradWs w;
  *bytes = wgrad_layout(wgrad_way(b->n_lanes, n_tokens, out_features, cols), n_tokens, out_features, cols, nullptr, &w);
  return AUGTREE_OK;
}

int augtree_ckpt_wgrad(const augtree_block_t *b, const void *dy, int64_t n_tokens, int64_t out_features, const void *ckpt, int64_t cols,
                       const float *row, const void *col, int col_dtype, void *d_weight, int weight_dtype, int accumulate, void *ws,
                       size_t ws_bytes, void *stream) {
  int r = check_block(b);
  if (r || (r = check_size(n_tokens, cols)) || (r = check_size(n_tokens, out_features))) return r;
  if ((weight_dtype != AUGTREE_BF16 && weight_dtype != AUGTREE_F32) || (col && !dtype_ok(col_dtype))) return AUGTREE_ERR_INVALID_ARG;
  if (accumulate && weight_dtype != AUGTREE_F32) return AUGTREE_ERR_UNSUPPORTED;
  if (!d_weight || !aligned16(d_weight) || !aligned16(col) || !aligned(row, 4)) return AUGTREE_ERR_INVALID_ARG;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const bool f32 = weight_dtype == AUGTREE_F32;
  if (n_tokens == 0) {
    if (!accumulate && cudaMemsetAsync(d_weight, 0, (size_t)out_features * cols * (f32 ? 4 : 2), st) != cudaSuccess) return cuda_failed();
    return AUGTREE_OK;
  }
  if (!dy || !ckpt || !aligned16(dy) || !aligned16(ckpt)) return AUGTREE_ERR_INVALID_ARG;
  const WgradWay way = wgrad_way(b->n_lanes, n_tokens, out_features, cols);
  WgradWs w;
  if (!ws || !aligned16(ws) || ws_bytes < wgrad_layout(way, n_tokens, out_features, cols, static_cast<uint8_t *>(ws), &w)) return AUGTREE_ERR_WORKSPACE;
  const int64_t padded = up(cols, 64);
  if (!way.bits) {
    unsigned blocks;
    const Pieces pc = pieces(b, n_tokens, padded, kUnpackBlocks, {{w.x, padded, 2}}, &blocks);
    if ((r = launch(ckpt_unpack_kernel<__nv_bfloat16>, blocks, kActThreads, 0, st, ckpt_rows(ckpt, cols), pc, (int)(cols / 8), row, nullptr, 0, w.x, padded)))
      return r;
  }
  WgradParams p = {};
  p.out = (int)out_features; p.cols = (int)cols; p.steps = (int)((n_tokens + 63) / 64);
  p.mt = (int)((out_features + kLmTile - 1) / kLmTile); p.nt = (int)((cols + kLmTile - 1) / kLmTile);
  p.splits = way.splits;
  p.share = (p.steps + p.splits - 1) / p.splits;
  p.a_chunks = out_features % 64 == 0 ? 2 : 1;
  p.part_rows = (int64_t)p.mt * kLmTile;
  p.scales = (int)ckpt_scale_offset(cols); p.rows = (int)n_tokens; p.row = row;
  const bool joined = p.splits > 1 || (!f32 && p.steps > kWgLong);
  p.f32 = joined || f32; p.add = !joined && accumulate;
  p.col = joined ? nullptr : col; p.col_type = col_dtype;
  p.status = b->d_status;
  p.wait_budget = (b->flags & AUGTREE_FLAG_TEST_SHORT_WAIT) ? kWaitBudgetClocksTest : kWaitBudgetClocks;
  p.test_flags = (b->flags & AUGTREE_FLAG_TEST_SKIP_FWD_LOAD) ? TEST_SKIP_FWD_LOAD : 0;
  CUtensorMap m_dy, m_x = {}, m_raw = {}, m_scale = {}, m_out;
  if ((r = map_mn(&m_dy, dy, n_tokens, out_features, p.a_chunks)) ||
      (r = joined ? map_out(&m_out, w.part, p.splits * p.part_rows, cols, true) : map_out(&m_out, d_weight, out_features, cols, f32)))
    return r;
  if (way.bits) {
    if ((r = map_bytes(&m_raw, ckpt, n_tokens, ckpt_pitch(cols), 128)) || (r = map_bytes(&m_scale, ckpt, n_tokens, ckpt_pitch(cols), 16))) return r;
  } else if ((r = map_mn(&m_x, w.x, n_tokens, padded, 2))) {
    return r;
  }
  const int pairs = std::max(b->n_lanes / 2, 1);
  r = way.bits ? launch(wgrad_kernel<true>, 2 * pairs, kWgThreads<true>, WgSmem<true>::kBytes, st, m_dy, m_x, m_raw, m_scale, m_out, p)
               : launch(wgrad_kernel<false>, 2 * pairs, kWgThreads<false>, WgSmem<false>::kBytes, st, m_dy, m_x, m_raw, m_scale, m_out, p);
  if (r || !joined) return r;
  const unsigned grid = (unsigned)std::min<int64_t>((out_features * (cols / 8) + 255) / 256, 8ll * b->n_lanes);
  return launch(wgrad_join_kernel, grid, 256, 0, st, w.part, p.splits, p.part_rows, (int)out_features, (int)cols, col, col_dtype, d_weight, weight_dtype, accumulate);
}

int augtree_block_last_device_status(const augtree_block_t *b, int *status, int *detail) {
  if (!b || b->device < 0 || !status) return AUGTREE_ERR_INVALID_ARG;
  int prev = 0;
  cudaGetDevice(&prev);
  cudaSetDevice(b->device);
  int h[2] = {0, 0};
  cudaError_t e = cudaDeviceSynchronize();
  if (e == cudaSuccess) e = cudaMemcpy(h, b->d_status, sizeof(h), cudaMemcpyDeviceToHost);
  if (e == cudaSuccess && (h[0] || h[1])) e = cudaMemset(b->d_status, 0, sizeof(h));
  cudaSetDevice(prev);
  if (e != cudaSuccess) return cuda_failed();
  *status = h[0];
  if (detail) *detail = h[1];
  return AUGTREE_OK;
}

}  // extern "C"
