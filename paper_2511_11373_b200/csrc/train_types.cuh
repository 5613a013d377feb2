// Element access of the training-pass kernels: fp32, bf16 and fp16 values in groups of eight, computed in fp32.
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"

namespace mars {

template <typename T> struct Raw8;                 // eight values as they lie in memory
template <> struct Raw8<float> { uint4 v[2]; };
template <> struct Raw8<__nv_bfloat16> { uint4 v[1]; };
template <> struct Raw8<__half> { uint4 v[1]; };

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

__device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b, __nv_bfloat16) { a = bf16_lo(w); b = bf16_hi(w); }
__device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b, __half) {
    const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&w));
    a = t.x; b = t.y;
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __nv_bfloat16) { return pack_bf16(a, b); }
__device__ __forceinline__ uint32_t pack2(float a, float b, __half) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

template <typename T>
__device__ __forceinline__ void unpack8(const Raw8<T>& r, float (&f)[8]) {
    const uint32_t w[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2(w[i], f[2 * i], f[2 * i + 1], T());
}
template <>
__device__ __forceinline__ void unpack8<float>(const Raw8<float>& r, float (&f)[8]) {
    f[0] = __uint_as_float(r.v[0].x); f[1] = __uint_as_float(r.v[0].y); f[2] = __uint_as_float(r.v[0].z); f[3] = __uint_as_float(r.v[0].w);
    f[4] = __uint_as_float(r.v[1].x); f[5] = __uint_as_float(r.v[1].y); f[6] = __uint_as_float(r.v[1].z); f[7] = __uint_as_float(r.v[1].w);
}
template <typename T>
__device__ __forceinline__ Raw8<T> pack8(const float (&f)[8]) {
    Raw8<T> r;
    r.v[0] = make_uint4(pack2(f[0], f[1], T()), pack2(f[2], f[3], T()), pack2(f[4], f[5], T()), pack2(f[6], f[7], T()));
    return r;
}
template <>
__device__ __forceinline__ Raw8<float> pack8<float>(const float (&f)[8]) {
    Raw8<float> r;
    r.v[0] = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    r.v[1] = make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7]));
    return r;
}
// Plain loads (not the read-only path): outputs may lie in place of inputs.
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T* p) {
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r.v[i] = *(reinterpret_cast<const uint4*>(p) + i);
    return r;
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const Raw8<T>& r) {
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 2); ++i) *(reinterpret_cast<uint4*>(p) + i) = r.v[i];
}
// A value, or 0 without a load.
__device__ __forceinline__ float load_if(const float* p, bool in) { return in ? *p : 0.f; }
__device__ __forceinline__ float load_if(const __nv_bfloat16* p, bool in) {
    const uint32_t b = in ? *reinterpret_cast<const uint16_t*>(p) : 0u;
    return __uint_as_float(b << 16);
}
__device__ __forceinline__ float load_if(const __half* p, bool in) {
    const uint16_t b = in ? *reinterpret_cast<const uint16_t*>(p) : (uint16_t)0;
    return __half2float(__ushort_as_half(b));
}

// Value i of a small tensor whose type is known at run time (MARS_F32, MARS_BF16, MARS_F16).
__device__ __forceinline__ float load_any(const void* p, int type, int64_t i) {
    if (type == 0) return static_cast<const float*>(p)[i];
    if (type == 1) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
    return __half2float(static_cast<const __half*>(p)[i]);
}

// Two fp32 operations in one instruction, each rounded as the scalar one.
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 r;
    asm("{.reg .b64 a, b, r;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tadd.rn.f32x2 r, a, b;\n\tmov.b64 {%0, %1}, r;}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 r;
    asm("{.reg .b64 a, b, r;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 r, a, b;\n\tmov.b64 {%0, %1}, r;}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 r;
    asm("{.reg .b64 a, b, c, r;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\tfma.rn.f32x2 r, a, b, c;\n\tmov.b64 {%0, %1}, r;}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}

// 2^x, results below the normal numbers are 0.
__device__ __forceinline__ float ex2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ double warp_sum_double(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

}  // namespace mars
