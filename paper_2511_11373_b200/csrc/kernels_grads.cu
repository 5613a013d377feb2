// The norm over all gradients of a list of tensors, and the list scaled down to a largest norm.
//   norm = sqrt(sum_t sum_i t_i^2),   out_t = t min(1, max_norm / (norm + 1e-6))
// Bound by HBM: the list is read once for the norm and, because no output may be written before the norm is
// known, once more for the outputs.  The list is cut into chunks of kChunkBytes of a tensor's own memory; every
// block takes a contiguous run of chunks (the tensor is searched once per run, then followed), so one launch covers
// tensors of any number and size.  A thread has its eight 16-byte loads of a chunk in flight together.  The scaling
// pass walks each run backwards: what the norm read last is still in L2.  Squares are added in fp32 over
// at most a chunk's share of one thread and in fp64 beyond; a chunk whose fp32 sum overflowed, or is so small
// that squares were lost below the smallest fp32 number, is summed again in fp64.  All sums run in a fixed
// order: the same list gives the same bits on every call.  The factor is kept in fp64 and rounded to fp32 for the products
// (2^-24 beside the rounding of the result); one too small for fp32's full precision multiplies in fp64.
#include <cuda_fp16.h>

#include "common.cuh"
#include "kernels.h"
#include "update.h"

namespace mars {

namespace {
constexpr int kChunkBytes = 32768, kThreads = 256;
constexpr int kBlocksPerSm = 8;

__host__ __device__ constexpr int elem_bytes(int type) { return type == 0 ? 4 : 2; }     // MARS_F32, MARS_BF16, MARS_F16

template <int T>
__device__ __forceinline__ void unpack(uint4 v, float (&f)[8]) {         // fp32 fills the first four
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (T == 0) {
            f[i] = __uint_as_float(w[i]);
            f[i + 4] = 0.f;
        } else if (T == 1) {
            f[2 * i] = bf16_lo(w[i]); f[2 * i + 1] = bf16_hi(w[i]);
        } else {
            const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            f[2 * i] = t.x; f[2 * i + 1] = t.y;
        }
    }
}
template <int T>
__device__ __forceinline__ uint4 scaled(uint4 v, float s) {
    float f[8];
    unpack<T>(v, f);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] *= s;
    if (T == 0) return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (T == 1) {
            w[q] = pack_bf16(f[2 * q], f[2 * q + 1]);
        } else {
            const __half2 h = __floats2half2_rn(f[2 * q], f[2 * q + 1]);
            w[q] = *reinterpret_cast<const uint32_t*>(&h);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ float load_one(const unsigned char* p, int type) {
    if (type == 0) return *reinterpret_cast<const float*>(p);
    if (type == 1) return __bfloat162float(*reinterpret_cast<const __nv_bfloat16*>(p));
    return __half2float(*reinterpret_cast<const __half*>(p));
}
__device__ __forceinline__ void store_one(unsigned char* p, int type, float v) {
    if (type == 0) *reinterpret_cast<float*>(p) = v;
    else if (type == 1) *reinterpret_cast<__nv_bfloat16*>(p) = __float2bfloat16_rn(v);
    else *reinterpret_cast<__half*>(p) = __float2half_rn(v);
}

// A chunk is what lies between two multiples of kChunkBytes of the tensor's memory, counted from its address
// rounded down to 16 bytes: inside a chunk 16-byte loads are aligned, and only its ends can be ragged.
struct Chunk {
    const unsigned char *src, *lo, *hi;    // lo..hi: whole 16-byte pieces
    unsigned char* dst;
    int64_t begin, end;                    // bytes of the tensor covered, [begin, end)
    int type;
};

__device__ __forceinline__ int find_tensor(const GradEntry* table, int n, int64_t chunk) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (table[mid].first_chunk <= chunk) lo = mid; else hi = mid - 1;
    }
    return lo;
}
__device__ __forceinline__ Chunk chunk_at(const GradEntry& g, int64_t chunk) {
    Chunk c;
    c.type = g.type;
    c.src = reinterpret_cast<const unsigned char*>(g.src);
    c.dst = reinterpret_cast<unsigned char*>(g.dst);
    const int64_t shift = (int64_t)((uintptr_t)g.src & 15), bytes = g.numel * elem_bytes(g.type);
    const int64_t k = chunk - g.first_chunk;
    c.begin = max((int64_t)0, k * kChunkBytes - shift);
    c.end = min(bytes, (k + 1) * kChunkBytes - shift);
    uintptr_t a = ((uintptr_t)c.src + c.begin + 15) & ~(uintptr_t)15, b = ((uintptr_t)c.src + c.end) & ~(uintptr_t)15;
    if (b < a) b = a;
    c.lo = reinterpret_cast<const unsigned char*>(a);
    c.hi = reinterpret_cast<const unsigned char*>(b);
    return c;
}
// Elements before the first and behind the last whole piece, by index 0 .. ragged() - 1 (at most 14).
__device__ __forceinline__ int ragged_head(const Chunk& c) {
    const int64_t h = min((int64_t)(c.lo - c.src), c.end) - c.begin;
    return (int)(h / elem_bytes(c.type));
}
__device__ __forceinline__ int ragged_tail(const Chunk& c) {
    const int64_t from = max((int64_t)(c.hi - c.src), c.begin + (int64_t)ragged_head(c) * elem_bytes(c.type));
    return from < c.end ? (int)((c.end - from) / elem_bytes(c.type)) : 0;
}
__device__ __forceinline__ int64_t ragged_offset(const Chunk& c, int i, int head, int tail) {
    const int eb = elem_bytes(c.type);
    return i < head ? c.begin + (int64_t)i * eb : c.end - (int64_t)(tail - (i - head)) * eb;
}

__device__ __forceinline__ double block_sum_double(double v, double* scratch) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if (lane == 0) scratch[warp] = v;
    __syncthreads();
    double t = 0.;
    for (int i = 0; i < (int)(blockDim.x >> 5); ++i) t += scratch[i];
    return t;
}

constexpr int kPieces = kChunkBytes / 16 / kThreads;       // 16-byte pieces of a thread in a whole chunk

// Sum of this thread's squares of a chunk.
template <int T>
__device__ __forceinline__ double chunk_squares(const Chunk& c) {
    const int pieces = (int)((c.hi - c.lo) >> 4);
    uint4 v[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int at = i * kThreads + threadIdx.x;
        v[i] = at < pieces ? ldg_stream(c.lo + (size_t)at * 16) : make_uint4(0, 0, 0, 0);
    }
    float part[4] = {0.f, 0.f, 0.f, 0.f};
    uint32_t seen = 0;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        float f[8];
        unpack<T>(v[i], f);
#pragma unroll
        for (int j = 0; j < (T == 0 ? 4 : 8); ++j) part[j & 3] = fmaf(f[j], f[j], part[j & 3]);
        seen |= v[i].x | v[i].y | v[i].z | v[i].w;
    }
    float sum = (part[0] + part[1]) + (part[2] + part[3]);
    const int head = ragged_head(c), tail = ragged_tail(c);
    float edge = 0.f;
    if (threadIdx.x < head + tail) {
        edge = load_one(c.src + ragged_offset(c, threadIdx.x, head, tail), T);
        sum = fmaf(edge, edge, sum);
        seen |= edge != 0.f;
    }
    // squares of one thread that left the range of fp32: again in fp64 (an infinity or a NaN comes out the same)
    if (!(sum < 1e37f) || (sum < 1e-20f && (seen & (T == 0 ? 0x7fffffffu : 0x7fff7fffu)))) {
        double d = (double)edge * (double)edge;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            float f[8];
            unpack<T>(v[i], f);
#pragma unroll
            for (int j = 0; j < 8; ++j) d = fma((double)f[j], (double)f[j], d);
        }
        return d;
    }
    return sum;
}

// The run of chunks of a block.
__device__ __forceinline__ int64_t run_begin(int64_t n_chunks, int64_t b) { return n_chunks * b / gridDim.x; }

__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const GradEntry* table, int n, int64_t n_chunks, double* partials,
                                                             int32_t* ticket, float max_norm, float* norm_out, double* scale) {
    __shared__ double scratch[kThreads / 32];
    __shared__ int last;
    pdl_wait();
    double total = 0.;
    const int64_t begin = run_begin(n_chunks, blockIdx.x), end = run_begin(n_chunks, blockIdx.x + 1);
    if (begin < end) {
        int t = find_tensor(table, n, begin);
        for (int64_t chunk = begin; chunk < end; ++chunk) {
            while (t + 1 < n && table[t + 1].first_chunk <= chunk) ++t;
            const Chunk c = chunk_at(table[t], chunk);
            total += c.type == 0 ? chunk_squares<0>(c) : c.type == 1 ? chunk_squares<1>(c) : chunk_squares<2>(c);
        }
    }
    total = block_sum_double(total, scratch);
    if (threadIdx.x == 0) {
        partials[blockIdx.x] = total;
        __threadfence();
        last = atomicAdd(ticket, 1) == (int)gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    double t = 0.;
    for (int i = threadIdx.x; i < (int)gridDim.x; i += kThreads) t += __ldcg(partials + i);
    t = block_sum_double(t, scratch);
    if (threadIdx.x == 0) {
        *ticket = 0;
        const double norm = sqrt(t);
        *norm_out = (float)norm;
        if (scale) {
            const double s = (double)max_norm / (norm + 1e-6);
            *scale = s >= 1. ? 1. : s;      // a NaN norm gives NaN
        }
    }
}

template <int T>
__device__ __forceinline__ void scale_chunk(const Chunk& c, float s) {
    const int pieces = (int)((c.hi - c.lo) >> 4);
    const int64_t first = c.lo - c.src;
    constexpr int eb = elem_bytes(T);
    uint4 v[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int at = i * kThreads + threadIdx.x;
        if (at < pieces) v[i] = __ldcs(reinterpret_cast<const uint4*>(c.lo + (size_t)at * 16));
    }
    if ((((uintptr_t)c.dst ^ (uintptr_t)c.src) & 15) == 0) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int at = i * kThreads + threadIdx.x;
            if (at < pieces) __stcs(reinterpret_cast<uint4*>(c.dst + first + (int64_t)at * 16), scaled<T>(v[i], s));
        }
    } else {                                  // grad and out lie differently in their 16 bytes
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int at = i * kThreads + threadIdx.x;
            if (at >= pieces) continue;
            float f[8];
            unpack<T>(v[i], f);
#pragma unroll
            for (int j = 0; j < 16 / eb; ++j) store_one(c.dst + first + (int64_t)at * 16 + j * eb, T, f[j] * s);
        }
    }
    const int head = ragged_head(c), tail = ragged_tail(c);
    if (threadIdx.x < head + tail) {
        const int64_t at = ragged_offset(c, threadIdx.x, head, tail);
        store_one(c.dst + at, T, load_one(c.src + at, T) * s);
    }
}

// The same with a factor below the normal numbers of fp32 (finite gradients with a norm of 1e38 and more, or a tiny largest
// norm): products in fp64, element by element.
__device__ void scale_chunk_tiny(const Chunk& c, double s) {
    const int eb = elem_bytes(c.type);
    for (int64_t at = c.begin + (int64_t)threadIdx.x * eb; at < c.end; at += kThreads * eb)
        store_one(c.dst + at, c.type, (float)((double)load_one(c.src + at, c.type) * s));
}

__global__ void __launch_bounds__(kThreads) grad_scale_kernel(const GradEntry* table, int n, int64_t n_chunks, const double* scale) {
    pdl_wait();
    const double exact = *scale;
    const float s = (float)exact;
    const bool tiny = exact > 0. && exact < 1.17549435e-38;
    const int64_t begin = run_begin(n_chunks, blockIdx.x), end = run_begin(n_chunks, blockIdx.x + 1);
    if (begin >= end) return;
    int t = find_tensor(table, n, end - 1);
    for (int64_t chunk = end - 1; chunk >= begin; --chunk) {
        while (table[t].first_chunk > chunk || table[t].numel == 0) --t;
        const Chunk c = chunk_at(table[t], chunk);
        if (s == 1.f && c.src == c.dst) continue;
        if (tiny) scale_chunk_tiny(c, exact);
        else if (c.type == 0) scale_chunk<0>(c, s);
        else if (c.type == 1) scale_chunk<1>(c, s);
        else scale_chunk<2>(c, s);
    }
}
}  // namespace

int64_t grad_chunks(const void* src, int64_t numel, int type) {
    const int64_t bytes = (int64_t)((uintptr_t)src & 15) + numel * elem_bytes(type);
    return numel ? (bytes + kChunkBytes - 1) / kChunkBytes : 0;
}
int grad_blocks(int sms) { return sms * kBlocksPerSm; }

cudaError_t launch_grad_norm(const GradEntry* table, int n_tensors, int64_t n_chunks, double* partials, int32_t* ticket,
                             float max_norm, float* norm_out, double* scale, int blocks, cudaStream_t st) {
    const int grid = (int)(n_chunks < 1 ? 1 : n_chunks < blocks ? n_chunks : blocks);
    return launch_chained(grad_norm_kernel, dim3(grid), dim3(kThreads), 0, st, table, n_tensors, n_chunks, partials, ticket,
                          max_norm, norm_out, scale);
}
cudaError_t launch_grad_scale(const GradEntry* table, int n_tensors, int64_t n_chunks, const double* scale, int blocks,
                              cudaStream_t st) {
    const int grid = (int)(n_chunks < 1 ? 1 : n_chunks < blocks ? n_chunks : blocks);
    return launch_chained(grad_scale_kernel, dim3(grid), dim3(kThreads), 0, st, table, n_tensors, n_chunks, scale);
}

}  // namespace mars
