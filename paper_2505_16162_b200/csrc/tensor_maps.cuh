// The driver's tensor-map encoder.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

namespace knnssd {

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                  const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's tensor-map encoder, looked up through the runtime (the library does not link against the driver).
inline EncodeTiledFn encode_tiled_fn() {
    static const EncodeTiledFn fn = [] {                 // once, and for all threads that come meanwhile
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        const bool found = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess && q == cudaDriverEntryPointSuccess;
        return found ? reinterpret_cast<EncodeTiledFn>(p) : nullptr;
    }();
    return fn;
}

// Map of bf16 values of `dims` dimensions (innermost first; strides in bytes of all but the innermost) read in boxes, 128-byte swizzle;
// places outside read as zero.
inline bool bf16_map(CUtensorMap *m, const void *base, int dims, const cuuint64_t *sizes, const cuuint64_t *strides, const cuuint32_t *box) {
    const EncodeTiledFn fn = encode_tiled_fn();
    const cuuint32_t one[4] = {1u, 1u, 1u, 1u};
    return fn && fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, (cuuint32_t)dims, const_cast<void *>(base), sizes, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace knnssd
