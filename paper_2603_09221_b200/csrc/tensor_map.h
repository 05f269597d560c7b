// The driver's function that describes tensors to the copy engines, found once.
#pragma once

#include <cuda.h>

#include "block_host.h"

namespace ttc {
namespace blk {

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline int encoder(EncodeTiled& f)
{
    static std::atomic<void*> known;
    void* p = known.load(std::memory_order_relaxed);
    if (!p) {
        cudaDriverEntryPointQueryResult found;
        TTC_CUDA(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &found));
        if (found != cudaDriverEntryPointSuccess || !p)
            return fail(TTC_STATUS_CUDA_ERROR, "the driver has no cuTensorMapEncodeTiled");
        known.store(p, std::memory_order_relaxed);
    }
    f = reinterpret_cast<EncodeTiled>(p);
    return TTC_OK;
}

} // namespace blk
} // namespace ttc
