// Pieces shared by the host files of the C ABI: error capture, checks of pointers and overlaps, device guard, bf16 tensor maps.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/mars.h"

#define CUDA_TRY(expr)                                   \
    do {                                                 \
        cudaError_t _e = (expr);                         \
        if (_e != cudaSuccess) {                         \
            mars::g_last_cuda_error = (int32_t)_e;       \
            return MARS_ERR_CUDA;                        \
        }                                                \
    } while (0)
#define RUN(expr)                                              \
    do {                                                       \
        const mars_status_t _s = (expr);                       \
        if (_s != MARS_OK) return _s;                          \
    } while (0)

namespace mars {

extern thread_local int32_t g_last_cuda_error;

inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }

// bf16 (or fp32) tensor map with the 128-byte swizzle (mars_api.cu); box[0] is at most 128 bytes.
mars_status_t make_tiled_map(CUtensorMap* tm, const void* base, int rank, const cuuint64_t* dims,
                             const cuuint64_t* strides_bytes, const cuuint32_t* box, bool f32 = false);

struct DeviceGuard {           // calls run on the handle's device, whatever is current
    int prev = -1;
    bool ok = true;
    explicit DeviceGuard(int dev) {
        int cur = -1;
        ok = cudaGetDevice(&cur) == cudaSuccess;
        if (ok && cur != dev) {
            ok = cudaSetDevice(dev) == cudaSuccess;
            if (ok) prev = cur;
        }
    }
    ~DeviceGuard() { if (prev >= 0) cudaSetDevice(prev); }
};

inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    return na && nb && x < y + nb && y < x + na;
}
inline size_t span(int64_t rows, int64_t ld, int64_t cols, size_t elem) {
    return rows > 0 ? (size_t)((rows - 1) * ld + cols) * elem : 0;
}
// Two [rows][..] matrices with row strides (elements).  Column ranges of one buffer lie inside each other's span without
// sharing a byte: with equal strides, b's columns must then fall between the end of a's and the end of the row.
inline bool rows_overlap(const void* a, int64_t ld_a, int64_t cols_a, size_t elem_a, const void* b, int64_t ld_b, int64_t cols_b, size_t elem_b,
                  int64_t rows) {
    if (!overlap(a, span(rows, ld_a, cols_a, elem_a), b, span(rows, ld_b, cols_b, elem_b))) return false;
    const size_t pitch = (size_t)ld_a * elem_a;
    if (rows < 2 || pitch != (size_t)ld_b * elem_b) return true;
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    const size_t at = y >= x ? (y - x) % pitch : (pitch - (x - y) % pitch) % pitch;       // of b's columns in a's rows
    return at < (size_t)cols_a * elem_a || at + (size_t)cols_b * elem_b > pitch;
}
inline bool aligned16(const void* p) { return (uintptr_t)p % 16 == 0; }
inline bool aligned4(const void* p) { return (uintptr_t)p % 4 == 0; }

inline mars_status_t launched(cudaError_t e) {
    if (e == cudaSuccess) return MARS_OK;
    g_last_cuda_error = (int32_t)e;
    return MARS_ERR_CUDA;
}
inline mars_status_t device_info(int* dev, int* sms) {
    int major = 0;
    CUDA_TRY(cudaGetDevice(dev));
    CUDA_TRY(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, *dev));
    CUDA_TRY(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, *dev));
    return major == 10 ? MARS_OK : MARS_ERR_UNSUPPORTED;
}

}  // namespace mars
