// What the entry-point files share: the launch counter and the driver's tensor-map encoder.
#pragma once
#include <cuda.h>

#include <atomic>

namespace augtree {

extern std::atomic<long long> g_launches;  // kernel launches enqueued since the library was loaded

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn get_encode();  // null when the driver has none

}  // namespace augtree
