// Pieces shared by the two host files of the C ABI: error capture, alignment, bf16 tensor maps.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/mars.h"

namespace mars {

extern thread_local int32_t g_last_cuda_error;

inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

// bf16 (or fp32) tensor map with the 128-byte swizzle (mars_api.cu); box[0] is at most 128 bytes.
mars_status_t make_tiled_map(CUtensorMap* tm, const void* base, int rank, const cuuint64_t* dims,
                             const cuuint64_t* strides_bytes, const cuuint32_t* box, bool f32 = false);

}  // namespace mars

#define CUDA_TRY(expr)                                   \
    do {                                                 \
        cudaError_t _e = (expr);                         \
        if (_e != cudaSuccess) {                         \
            mars::g_last_cuda_error = (int32_t)_e;       \
            return MARS_ERR_CUDA;                        \
        }                                                \
    } while (0)
