// Host side of TMA: the driver's encoder of tensor maps.
#pragma once

#include <cuda.h>

#include <mutex>

#include "common.cuh"

namespace moska {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                  const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's tensor-map encoder, looked up through the runtime (no link against libcuda).
inline int tensor_map_encoder(EncodeTiledFn* out)
{
    static EncodeTiledFn fn = nullptr;
    static std::mutex mtx;
    std::lock_guard<std::mutex> lock(mtx);
    if (fn == nullptr) {
        void* sym = nullptr;
        cudaDriverEntryPointQueryResult res;
        MOSKA_CUDA_TRY(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &res));
        if (sym == nullptr || res != cudaDriverEntryPointSuccess)
            return fail(MOSKA_ERR_CUDA, "the driver does not provide cuTensorMapEncodeTiled");
        fn = reinterpret_cast<EncodeTiledFn>(sym);
    }
    *out = fn;
    return MOSKA_OK;
}

}  // namespace moska
