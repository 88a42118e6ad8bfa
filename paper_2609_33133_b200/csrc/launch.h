// What the entry-point files share: the launch counter, the driver's tensor-map encoder, the way memory is given back.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>

namespace augtree {

extern std::atomic<long long> g_launches;  // kernel launches enqueued since the library was loaded

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn get_encode();  // null when the driver has none

// While one of these lives, calls of this thread that a capture forbids (cudaFree among them) go through and leave the capture as
// it is.  A handle or plan may be destroyed at any time: a garbage collector does so in the middle of a capture.
struct RelaxedCapture {
  cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
  RelaxedCapture() { cudaThreadExchangeStreamCaptureMode(&mode); }
  ~RelaxedCapture() { cudaThreadExchangeStreamCaptureMode(&mode); }
};

}  // namespace augtree
