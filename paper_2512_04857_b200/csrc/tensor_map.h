// 4-D tensor maps for the paged kernels.
#pragma once
#include <cuda.h>

#include "../../include/lar.h"
#include "host_util.h"

namespace lar {

enum MapType { kMapBytes, kMapBf16, kMapFp32 };

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// dim and box in elements, the strides of dimensions 1 to 3 in elements; swizzle: 0, 64 or 128 bytes.  Encoding is a call of the driver: the
// runtime must have been called in this thread before, which makes the device's context current.
inline lar_status_t encode_map_4d(CUtensorMap* m, MapType type, int swizzle, void* p, const cuuint64_t (&dim)[4], const int64_t (&stride)[3],
                                  const cuuint32_t (&box)[4]) {
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
    const cuuint32_t one[4] = {1, 1, 1, 1};
    const cuuint64_t st[3] = {(cuuint64_t)stride[0] * elt, (cuuint64_t)stride[1] * elt, (cuuint64_t)stride[2] * elt};
    if (encode(m, type == kMapBytes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : type == kMapBf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32,
               4, p, dim, st, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
               swizzle == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : swizzle == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_NONE,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS) {
        last_cuda_error() = (int)cudaErrorInvalidValue;
        return LAR_ERR_CUDA;
    }
    return LAR_OK;
}

}  // namespace lar
