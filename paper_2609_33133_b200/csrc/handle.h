// What the entry points with a handle share (lm.cu, block.cu): argument checks, scratch, tensor maps, launches.
#pragma once
#include <algorithm>
#include <cstdint>

#include "launch.h"
#include "../../include/augtree.h"

namespace augtree {

inline bool aligned(const void *p, int bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0; }
inline bool aligned16(const void *p) { return aligned(p, 16); }
inline constexpr int64_t kMaxTokens = (1ll << 31) - 4096;
inline constexpr int kMaxLanes = 1 << 20;   // as a plan's: grids are at most 32 times that

inline int64_t up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// A failed runtime call is reported by the return value and not left in the runtime's last error as well, where the attention's
// entry points, which look at it behind their launches, would find it and report a failure of their own.
inline int cuda_failed() {
  cudaGetLastError();
  return AUGTREE_ERR_CUDA;
}

// Scratch of one call, cut from the caller's block: every part starts on 256 bytes.
struct Cursor {
  uint8_t *base;
  size_t off = 0;
  template <typename T>
  T *take(int64_t n) {
    T *p = base ? reinterpret_cast<T *>(base + off) : nullptr;
    off += (size_t)up((int64_t)sizeof(T) * std::max<int64_t>(n, 1), 256);
    return p;
  }
};

// 2-D map over a row-major bf16 matrix: a box is 64 columns (128 bytes, swizzled) x `box_rows` rows; what lies outside
// reads as zero.  Box origins are multiples of 64 columns, so every copy starts on a 16-byte boundary.
inline int map_2d(CUtensorMap *m, const void *ptr, int64_t rows, int64_t cols, int box_rows) {
  EncodeTiledFn enc = get_encode();
  if (!enc) return AUGTREE_ERR_CUDA;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)cols * 2};
  const cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
  const cuuint32_t estr[2] = {1, 1};
  const CUresult r = enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(ptr), dims, strides, box, estr,
                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? AUGTREE_OK : AUGTREE_ERR_CUDA;
}

// The same for an operand whose contraction runs along the rows: a box is 64 rows of `chunks` neighbouring 64-column chunks,
// each chunk a block of 64 x 128 bytes of its own.  With two chunks the matrix is seen as [cols / 64][rows][64], which needs cols to
// be a multiple of 64 (a chunk that runs past the row's end would read the next row, and past the tensor in the last one).
inline int map_mn(CUtensorMap *m, const void *ptr, int64_t rows, int64_t cols, int chunks) {
  EncodeTiledFn enc = get_encode();
  if (!enc) return AUGTREE_ERR_CUDA;
  const cuuint64_t dims[3] = {(cuuint64_t)(chunks == 2 ? 64 : cols), (cuuint64_t)rows, (cuuint64_t)(chunks == 2 ? cols / 64 : 1)};
  const cuuint64_t strides[2] = {(cuuint64_t)cols * 2, 128};
  const cuuint32_t box[3] = {64, 64, (cuuint32_t)chunks};
  const cuuint32_t estr[3] = {1, 1, 1};
  const CUresult r = enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(ptr), dims, strides, box, estr,
                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? AUGTREE_OK : AUGTREE_ERR_CUDA;
}

// Map over bytes: a box is `box_bytes` of a row x 64 rows.
inline int map_bytes(CUtensorMap *m, const void *ptr, int64_t rows, int64_t pitch, int box_bytes) {
  EncodeTiledFn enc = get_encode();
  if (!enc) return AUGTREE_ERR_CUDA;
  const cuuint64_t dims[2] = {(cuuint64_t)pitch, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)pitch};
  const cuuint32_t box[2] = {(cuuint32_t)box_bytes, 64};
  const cuuint32_t estr[2] = {1, 1};
  const CUresult r = enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(ptr), dims, strides, box, estr,
                         CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? AUGTREE_OK : AUGTREE_ERR_CUDA;
}

// Map for results that leave through shared memory: a box is 128 bytes (swizzled) x 32 rows.
inline int map_out(CUtensorMap *m, const void *ptr, int64_t rows, int64_t cols, bool f32) {
  EncodeTiledFn enc = get_encode();
  if (!enc) return AUGTREE_ERR_CUDA;
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
  const cuuint64_t strides[1] = {(cuuint64_t)cols * (f32 ? 4 : 2)};
  const cuuint32_t box[2] = {f32 ? 32u : 64u, 32};
  const cuuint32_t estr[2] = {1, 1};
  const CUresult r = enc(m, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(ptr), dims, strides, box,
                         estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  return r == CUDA_SUCCESS ? AUGTREE_OK : AUGTREE_ERR_CUDA;
}

// The kernels of lm.cu and block.cu are launched as programmatic dependents of the one before them in the stream: they may be set up
// while that one still runs, and begin with wait_previous() (ptx.cuh).
template <typename... P, typename... A>
inline int launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t st, A &&...args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid; cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr; cfg.numAttrs = 1;
  ++g_launches;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...) == cudaSuccess ? AUGTREE_OK : cuda_failed();
}

inline bool dtype_ok(int t) { return t == AUGTREE_BF16 || t == AUGTREE_F16 || t == AUGTREE_F32; }

}  // namespace augtree
