// Host-side helpers shared by the translation units of the library: the thread's last CUDA error and the macro that
// turns a failed runtime call into LAR_ERR_CUDA.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdio.h>
#include <stdlib.h>

namespace lar {
constexpr int kMaxSmem = 227 * 1024;  // dynamic shared memory a CTA can have
int& last_cuda_error();  // cudaError_t of the last failed runtime call in this thread (defined in lar_api.cu)
}

#define LAR_CUDA(call)                                   \
    do {                                                 \
        cudaError_t e__ = (call);                        \
        if (e__ != cudaSuccess) {                        \
            lar::last_cuda_error() = (int)e__;           \
            (void)cudaGetLastError();                    \
            if (getenv("LAR_DEBUG"))                     \
                fprintf(stderr, "lar: line %d: %s -> %s\n", __LINE__, #call, cudaGetErrorString(e__)); \
            return LAR_ERR_CUDA;                         \
        }                                                \
    } while (0)
