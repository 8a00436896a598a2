// Host-side state shared by the translation units of the library (defined in api.cu).
#pragma once
#include <atomic>
#include <cuda.h>

namespace mmv {

extern std::atomic<long long> g_launches;                 // kernels launched since the library was loaded
extern std::atomic<unsigned long long> g_budget_ns;       // time after which a device-side wait gives up

using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                   const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                   CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn get_encode();                               // cuTensorMapEncodeTiled, or null

}  // namespace mmv
