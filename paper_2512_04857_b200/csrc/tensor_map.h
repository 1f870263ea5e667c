// Tensor maps for the paged kernels.
#pragma once
#include <cuda.h>

#include "../../include/lar.h"
#include "host_util.h"

namespace lar {

enum MapType { kMapBytes, kMapBf16, kMapFp32 };

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// dim and box in elements, the strides of the dimensions from 1 on in elements; swizzle: 0, 64 or 128 bytes; l2: bytes that a miss
// brings into L2 (64, 128 or 256).  Encoding is a call of the driver: the
// runtime must have been called in this thread before, which makes the device's context current.
template <int RANK>
lar_status_t encode_map(CUtensorMap* m, MapType type, int swizzle, void* p, const cuuint64_t (&dim)[RANK], const int64_t (&stride)[RANK - 1],
                        const cuuint32_t (&box)[RANK], int l2 = 256) {
    static const EncodeTiledFn encode = [] {
        void* fp = nullptr;
        cudaDriverEntryPointQueryResult res;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fp, cudaEnableDefault, &res) != cudaSuccess || res != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            fp = nullptr;
        }
        return reinterpret_cast<EncodeTiledFn>(fp);
    }();
    if (!encode) {
        last_cuda_error() = (int)cudaErrorNotSupported;
        return LAR_ERR_CUDA;
    }
    const cuuint64_t elt = type == kMapBytes ? 1 : type == kMapBf16 ? 2 : 4;
    cuuint32_t one[RANK];
    cuuint64_t st[RANK - 1];
    for (int i = 0; i < RANK; ++i) {
        one[i] = 1;
        if (i > 0) st[i - 1] = (cuuint64_t)stride[i - 1] * elt;
    }
    if (encode(m, type == kMapBytes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : type == kMapBf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32,
               RANK, p, dim, st, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
               swizzle == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : swizzle == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_NONE,
               l2 == 256 ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : l2 == 128 ? CU_TENSOR_MAP_L2_PROMOTION_L2_128B : CU_TENSOR_MAP_L2_PROMOTION_L2_64B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) {
        last_cuda_error() = (int)cudaErrorInvalidValue;
        return LAR_ERR_CUDA;
    }
    return LAR_OK;
}

}  // namespace lar
