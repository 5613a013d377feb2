// Norms of rows and their gradients.
//   s = x (+ add, rounded to x's type);  RMS: u = s, layer: u = s - mean(s);  r = 1 / sqrt(mean(u^2) + eps)
//   y = u r w (+ b);   n = u r, g = dy w:
//   dx = r (g - n mean(g n) - [layer] mean(g)) (+ d_sum),   dw = sum over rows of dy n,   db = sum of dy
// Bound by HBM: every matrix is read or written once.  A row stays in the registers of a group of threads (a part of a warp, a warp,
// or several that meet at a named barrier of their own, so that groups of a block do not wait for one another), in 16-byte
// pieces, or value by value where a row allows no such pieces.  The variance is taken from the centred
// values, in a second sum over the registers: sum of squares minus square of the sum would lose a mean that is large
// beside the spread.
// The gradient runs on a grid that fits the SMs at once: a thread keeps the sums of dw and db of its columns in fp32
// registers over all rows of its group and asks for the next row before it reduces the present one; groups of a block meet in
// shared memory, blocks in a second kernel that adds their sums in fp64 in a fixed order: the same call gives the same bits.
// Measured (B200, copy rate 6463 GB/s): RMS 32768 x 2048 bf16 with residual 88 us, 6.1 TB/s; its gradient 99 us, 5.4 TB/s with the
// second kernel (the first alone 93 us); gradient of 524288 heads of 128 bf16 80 us, 23 instructions a value.
#include <type_traits>

#include "train.h"
#include "train_types.cuh"

namespace mars {

namespace {

constexpr int kChunk = 8;
constexpr int kEach = 16;                // values of a thread where rows go value by value

// Threads of a row and chunks of eight neighbouring values of a thread; blocks of at most 256 threads.  Rows of up to 256 in one warp; two
// chunks for a thread beyond it, four where 256 threads need them.  2^26 values bf16, one / two / four chunks: forward 131072 x 512 65 / 50 /
// 109 us, 32768 x 2048 68 / 52 / 66; gradient 74 / 78 / 126 and 80 / 83 / 87 us, but 1000 x 2048 14.4 / 11.6 and layer norms 49 / 46.
struct NormPlan { int group, nv, block; };
NormPlan norm_plan(int width) {
    const int chunks = (width + kChunk - 1) / kChunk;
    NormPlan p;
    if (chunks <= 32) {
        p.nv = 1;
        p.group = 1;
        while (p.group < chunks) p.group *= 2;
    } else {
        p.nv = chunks <= 512 ? 2 : 4;
        p.group = (chunks + 32 * p.nv - 1) / (32 * p.nv) * 32;
    }
    p.block = 256 / p.group * p.group;
    return p;
}
// Blocks on an SM for which registers are planned, forward and backward; rows of a group that are worked on together.  Gradient of
// 32768 x 2048 bf16: two blocks 106 us, three, which spill, 112.  Narrow rows have registers for two rows at a time: the heads above, one
// row and two blocks 141 us -> two rows, three blocks and rounds without conditions 80.
__host__ __device__ constexpr int forward_blocks(int nv, bool x_is_fp32) { return nv == 4 ? 1 : nv == 2 ? (x_is_fp32 ? 2 : 3) : x_is_fp32 ? 3 : 4; }
__host__ __device__ constexpr int grad_blocks_sm(int nv, bool x_is_fp32, bool layer) { return nv == 4 ? 1 : nv == 1 && !x_is_fp32 && !layer ? 3 : 2; }
__host__ __device__ constexpr int rows_together(int nv) { return nv == 1 ? 2 : 1; }

// Rows value by value: threads of a row, a power of two from 32 to 512.
int scalar_group(int width) {
    int group = 32;
    while (group * kEach < width) group *= 2;
    return group;
}
constexpr int scalar_block(int group) { return group < 256 ? 256 : group; }

// Chunk j of a thread, zeros behind the row.
template <typename T>
__device__ __forceinline__ Raw8<T> load_chunk(const T* row, int j, int lane, int group, int width) {
    const int c = (j * group + lane) * kChunk;
    Raw8<T> r;
    if (c < width) {
        r = load8(row + c);
    } else {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(T) / 2); ++i) r.v[i] = make_uint4(0, 0, 0, 0);
    }
    return r;
}
template <typename T>
__device__ __forceinline__ void store_chunk(T* row, int j, int lane, int group, int width, const Raw8<T>& r) {
    const int c = (j * group + lane) * kChunk;
    if (c < width) store8(row + c, r);
}
__device__ __forceinline__ void load_weight(const void* w, int type, int j, int lane, int group, int width, float (&o)[8]) {
    const int c = (j * group + lane) * kChunk;
    if (c >= width) {
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = 0.f;
    } else if (type == 0) unpack8<float>(load8(static_cast<const float*>(w) + c), o);
    else if (type == 1) unpack8<__nv_bfloat16>(load8(static_cast<const __nv_bfloat16*>(w) + c), o);
    else unpack8<__half>(load8(static_cast<const __half*>(w) + c), o);
}

// Sums over the threads of a group.  Groups of more than a warp use one half of `scratch` after the other: who writes a half
// again has passed the barrier that all readers of it reached after reading.
template <int N>
__device__ __forceinline__ void group_sum(float (&v)[N], int group, int index, float* scratch, int& half) {
    if (group <= 32) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            if (o < group)
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
    const int warps = group >> 5, warp = threadIdx.x >> 5, first = index * warps;
    float* s = scratch + half * 16 * N;
    half ^= 1;
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) s[warp * N + i] = v[i];
    }
    asm volatile("bar.sync %0, %1;" ::"r"(index + 1), "r"(group) : "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = 0.f;
    for (int w = 0; w < warps; ++w)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += s[(first + w) * N + i];
}

// Offset of row (t, h); ld and heads * width fit 32 bits.
__device__ __forceinline__ int64_t row_offset(int row, int heads, int width, int64_t ld) {
    if (heads == 1) return (int64_t)((uint64_t)(uint32_t)row * (uint32_t)ld);
    const int t = (heads & (heads - 1)) == 0 ? row >> (31 - __clz(heads)) : row / heads;
    return (int64_t)((uint64_t)(uint32_t)t * (uint32_t)ld) + (row - t * heads) * width;
}

// Rows in registers.  A block stays for many rows: the weight's values stay too, and the next rows are on their way while the present
// ones are reduced (32768 x 2048 bf16 with residual: 87 us; a block for every four rows, that loads, reduces and stores, 120 us).
template <typename XT, typename YT, int NV>
__global__ void __launch_bounds__(256, forward_blocks(NV, sizeof(XT) == 4)) norm_rows_kernel(const NormArgs a, const int group) {
    __shared__ float scratch[2 * 16];
    const int index = threadIdx.x / group, lane = threadIdx.x - index * group, groups = blockDim.x / group;
    int half = 0;
    const float inv = 1.f / (float)a.width;
    float weight[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j) load_weight(a.weight, a.w_type, j, lane, group, a.width, weight[j]);
    Raw8<XT> x[NV];
    Raw8<YT> add[NV];
    auto fetch = [&](int64_t r) {
        const bool on = r < a.rows;
        const int row = on ? (int)r : 0, W = on ? a.width : 0;
#pragma unroll
        for (int j = 0; j < NV; ++j) x[j] = load_chunk(static_cast<const XT*>(a.x) + row_offset(row, a.heads, a.width, a.ld_x), j, lane, group, W);
        if (a.has_add) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
                add[j] = load_chunk(static_cast<const YT*>(a.add) + row_offset(row, a.heads, a.width, a.ld_add), j, lane, group, W);
        }
    };
    const int64_t stride = (int64_t)gridDim.x * groups;
    int64_t base = (int64_t)blockIdx.x * groups;
    if (base < a.rows) fetch(base + index);
    for (; base < a.rows; base += stride) {                   // the trip count is the same for all threads of a block
        const bool on = base + index < a.rows;
        const int row = on ? (int)(base + index) : 0;
        const int W = on ? a.width : 0;
        float v[NV][8];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            unpack8<XT>(x[j], v[j]);
            if (a.has_add) {
                float b[8];
                unpack8<YT>(add[j], b);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[j][i] += b[i];
                const Raw8<XT> s = pack8<XT>(v[j]);           // the norm is that of the stored sum
                unpack8<XT>(s, v[j]);
                if (a.sum) store_chunk(static_cast<XT*>(a.sum) + row_offset(row, a.heads, a.width, a.ld_sum), j, lane, group, W, s);
            }
        }
        fetch(base + stride + index);
        float mean = 0.f;
        if (a.layer) {
            float s[1] = {0.f};
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) s[0] += v[j][i];
            group_sum(s, group, index, scratch, half);
            mean = s[0] * inv;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const bool in = (j * group + lane) * kChunk < a.width;
#pragma unroll
                for (int i = 0; i < 8; ++i) v[j][i] = in ? v[j][i] - mean : 0.f;
            }
        }
        float q[1] = {0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) q[0] = fmaf(v[j][i], v[j][i], q[0]);
        group_sum(q, group, index, scratch, half);
        const float rstd = 1.f / sqrtf(q[0] * inv + a.eps);
        YT* y = static_cast<YT*>(a.y) + row_offset(row, a.heads, a.width, a.ld_y);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[j][i] = v[j][i] * rstd * weight[j][i];
            if (a.has_bias) {
                float b[8];
                load_weight(a.bias, a.w_type, j, lane, group, W, b);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[j][i] += b[i];
            }
            store_chunk(y, j, lane, group, W, pack8<YT>(v[j]));
        }
        if (on && lane == 0) {
            if (a.rstd) a.rstd[row] = rstd;
            if (a.mean && a.layer) a.mean[row] = mean;
        }
    }
}

// Any alignment: the same value by value, a thread having those that are a group apart.  16 loads of 2 or 4 bytes a thread in flight, bound
// by their number: 20000 x 1111 bf16 60 us (1.5 TB/s), fp32 53 us (3.4 TB/s); in loops that read a row again for each sum 178 us.
template <typename XT, typename YT, int G>
__global__ void __launch_bounds__(G < 256 ? 256 : G, G < 512 ? 3 : 1) norm_scalar_kernel(const NormArgs a) {
    constexpr int kGroups = (G < 256 ? 256 : G) / G;
    __shared__ float scratch[2 * 16];
    const int index = threadIdx.x / G, lane = threadIdx.x % G;
    int half = 0;
    const float inv = 1.f / (float)a.width;
    float weight[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) weight[i] = i * G + lane < a.width ? load_any(a.weight, a.w_type, i * G + lane) : 0.f;
    for (int64_t base = (int64_t)blockIdx.x * kGroups; base < a.rows; base += (int64_t)gridDim.x * kGroups) {
        const bool on = base + index < a.rows;
        const int row = on ? (int)(base + index) : 0;
        const int W = on ? a.width - lane : 0;                // value i lies inside where i * G < W
        const XT* x = static_cast<const XT*>(a.x) + row_offset(row, a.heads, a.width, a.ld_x) + lane;
        float v[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) v[i] = load_if(x + i * G, i * G < W);
        if (a.has_add) {
            const YT* add = static_cast<const YT*>(a.add) + row_offset(row, a.heads, a.width, a.ld_add) + lane;
            XT* sum = static_cast<XT*>(a.sum) + row_offset(row, a.heads, a.width, a.ld_sum) + lane;
            float b[kEach];
#pragma unroll
            for (int i = 0; i < kEach; ++i) b[i] = load_if(add + i * G, i * G < W);
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const XT s = from_float<XT>(v[i] + b[i]);
                v[i] = to_float(s);
                if (a.sum && i * G < W) sum[i * G] = s;
            }
        }
        float mean = 0.f;
        if (a.layer) {
            float s[1] = {0.f};
#pragma unroll
            for (int i = 0; i < kEach; ++i) s[0] += v[i];
            group_sum(s, G, index, scratch, half);
            mean = s[0] * inv;
#pragma unroll
            for (int i = 0; i < kEach; ++i) v[i] = i * G < W ? v[i] - mean : 0.f;
        }
        float q[1] = {0.f};
#pragma unroll
        for (int i = 0; i < kEach; ++i) q[0] = fmaf(v[i], v[i], q[0]);
        group_sum(q, G, index, scratch, half);
        const float rstd = 1.f / sqrtf(q[0] * inv + a.eps);
        YT* y = static_cast<YT*>(a.y) + row_offset(row, a.heads, a.width, a.ld_y) + lane;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            float o = v[i] * rstd * weight[i];
            if (a.has_bias && i * G < W) o += load_any(a.bias, a.w_type, i * G + lane);
            if (i * G < W) y[i * G] = from_float<YT>(o);
        }
        if (on && lane == 0) {
            if (a.rstd) a.rstd[row] = rstd;
            if (a.mean && a.layer) a.mean[row] = mean;
        }
    }
}

// Rows in registers, with the sums of the weight's gradient.  The weight lies in shared memory: its registers go to the next row.  The
// residual's gradient is asked for after the first pass over a row: before it, it costs registers (99 -> 118 us).
// FULL: the chunks of a group's threads are the row's, none lies behind it.
template <typename XT, typename YT, int NV, bool LAYER, bool FULL>
__global__ void __launch_bounds__(256, grad_blocks_sm(NV, sizeof(XT) == 4, LAYER)) norm_grad_rows_kernel(const NormGradArgs a, const int group) {
    constexpr int R = rows_together(NV), N = LAYER ? 2 * R : R;
    __shared__ float scratch[2 * 16 * N];
    extern __shared__ float sums[];                           // the weight, in the end the sums [groups][width]
    const int index = threadIdx.x / group, lane = threadIdx.x - index * group, groups = blockDim.x / group;
    int half = 0;
    const float inv = 1.f / (float)a.width;
    for (int c = threadIdx.x; c < a.width; c += blockDim.x) sums[c] = load_any(a.weight, a.w_type, c);
    __syncthreads();
    float acc_w[NV][8], acc_b[LAYER ? NV : 1][8];
    bool in[NV];                                              // chunks of this thread inside the row; the others are zeros throughout
    Raw8<XT> x[R][NV], ds[R][NV];
    Raw8<YT> dy[R][NV];
    const float zeros[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        in[j] = FULL || (j * group + lane) * kChunk < a.width;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            acc_w[j][i] = 0.f;
            if (LAYER) acc_b[j][i] = 0.f;
        }
        if (!FULL) {
#pragma unroll
            for (int k = 0; k < R; ++k) {
                x[k][j] = ds[k][j] = pack8<XT>(zeros);
                dy[k][j] = pack8<YT>(zeros);
            }
        }
    }
    const XT* px = static_cast<const XT*>(a.x) + lane * kChunk;
    const YT* pdy = static_cast<const YT*>(a.dy) + lane * kChunk;
    const XT* pds = static_cast<const XT*>(a.d_sum) + lane * kChunk;
    XT* pdx = static_cast<XT*>(a.dx) + lane * kChunk;
    const int step = group * kChunk;                          // from a chunk of a thread to its next
    float rstd[R], mean[R];
    auto fetch = [&](int64_t first) {                         // rows behind the last one: the last one again, left out where it is used
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int row = (int)min(first + (int64_t)k * groups, (int64_t)a.rows - 1);
            const XT* p = px + row_offset(row, a.heads, a.width, a.ld_x);
            const YT* q = pdy + row_offset(row, a.heads, a.width, a.ld_dy);
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (in[j]) x[k][j] = load8(p + j * step);
#pragma unroll
            for (int j = 0; j < NV; ++j)
                if (in[j]) dy[k][j] = load8(q + j * step);
            rstd[k] = a.rstd[row];
            mean[k] = LAYER ? a.mean[row] : 0.f;
        }
    };
    const int64_t stride = (int64_t)gridDim.x * groups * R;
    int64_t base = (int64_t)blockIdx.x * groups * R;
    // one round of the block; whole: all of its rows exist
    auto round = [&](auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        float n[R][NV][8], g[R][NV][8], c[N], r[R];
        bool on[R];
#pragma unroll
        for (int k = 0; k < R; ++k) on[k] = WHOLE || base + index + (int64_t)k * groups < a.rows;
#pragma unroll
        for (int k = 0; k < R; ++k) r[k] = rstd[k];
#pragma unroll
        for (int i = 0; i < N; ++i) c[i] = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            float w[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (in[j]) {
                const float4 lo = *reinterpret_cast<const float4*>(sums + lane * kChunk + j * step);
                const float4 hi = *reinterpret_cast<const float4*>(sums + lane * kChunk + j * step + 4);
                w[0] = lo.x; w[1] = lo.y; w[2] = lo.z; w[3] = lo.w; w[4] = hi.x; w[5] = hi.y; w[6] = hi.z; w[7] = hi.w;
            }
#pragma unroll
            for (int k = 0; k < R; ++k) {
                unpack8<XT>(x[k][j], n[k][j]);
                unpack8<YT>(dy[k][j], g[k][j]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    n[k][j][i] = (LAYER ? n[k][j][i] - mean[k] : n[k][j][i]) * rstd[k];
                    if (!WHOLE && !on[k]) n[k][j][i] = g[k][j][i] = 0.f;
                    acc_w[j][i] = fmaf(g[k][j][i], n[k][j][i], acc_w[j][i]);
                    if (LAYER) acc_b[j][i] += g[k][j][i];
                    g[k][j][i] *= w[i];
                    c[k] = fmaf(g[k][j][i], n[k][j][i], c[k]);
                    if (LAYER) c[R + k] += g[k][j][i];
                }
            }
        }
        int64_t at[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int row = (int)min(base + index + (int64_t)k * groups, (int64_t)a.rows - 1);
            at[k] = row_offset(row, a.heads, a.width, a.ld_dx);
            if (a.has_d_sum) {
                const XT* p = pds + row_offset(row, a.heads, a.width, a.ld_d_sum);
#pragma unroll
                for (int j = 0; j < NV; ++j)
                    if (in[j]) ds[k][j] = load8(p + j * step);
            }
        }
        fetch(base + stride + index);                         // the next rows are on their way while these are reduced
        group_sum(c, group, index, scratch, half);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const float c0 = -c[k] * inv * r[k], c1 = LAYER ? c[LAYER ? R + k : 0] * inv : 0.f;
#pragma unroll
            for (int j = 0; j < NV; ++j) {
#pragma unroll
                for (int i = 0; i < 8; ++i) g[k][j][i] = fmaf(LAYER ? g[k][j][i] - c1 : g[k][j][i], r[k], n[k][j][i] * c0);
                if (a.has_d_sum) {
                    float s[8];
                    unpack8<XT>(ds[k][j], s);
#pragma unroll
                    for (int i = 0; i < 8; ++i) g[k][j][i] += s[i];
                }
                if (in[j] && on[k]) store8(pdx + at[k] + j * step, pack8<XT>(g[k][j]));
            }
        }
    };
    if (base < a.rows) fetch(base + index);
    for (; base + groups * R <= a.rows; base += stride) round(std::true_type());
    if (base < a.rows) round(std::false_type());
    __syncthreads();                                          // the weight is not needed any more
#pragma unroll
    for (int which = 0; which < (LAYER ? 2 : 1); ++which) {
        float* out = which ? a.part_b : a.part_w;
        if (!out) continue;
        out += (int64_t)blockIdx.x * a.width;
        float* own = groups == 1 ? out : sums + index * a.width;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = (j * group + lane) * kChunk + i;
                if (c < a.width) own[c] = which ? acc_b[LAYER ? j : 0][i] : acc_w[j][i];
            }
        if (groups == 1) continue;
        __syncthreads();
        for (int c = threadIdx.x; c < a.width; c += blockDim.x) {
            float t = 0.f;
            for (int k = 0; k < groups; ++k) t += sums[k * a.width + c];
            out[c] = t;
        }
    }
}

// Any alignment: the same value by value (20000 x 1111 bf16 127 us; in loops that read a row again 276 us).
template <typename XT, typename YT, int G, bool LAYER>
__global__ void __launch_bounds__(G < 256 ? 256 : G, G < 512 ? 2 : 1) norm_grad_scalar_kernel(const NormGradArgs a) {
    constexpr int kGroups = (G < 256 ? 256 : G) / G;
    __shared__ float scratch[2 * 16 * 2];
    extern __shared__ float sums[];                           // [groups][width]
    const int index = threadIdx.x / G, lane = threadIdx.x % G;
    int half = 0;
    const float inv = 1.f / (float)a.width;
    float weight[kEach], acc_w[kEach], acc_b[LAYER ? kEach : 1];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        weight[i] = i * G + lane < a.width ? load_any(a.weight, a.w_type, i * G + lane) : 0.f;
        acc_w[i] = 0.f;
        if (LAYER) acc_b[i] = 0.f;
    }
    for (int64_t base = (int64_t)blockIdx.x * kGroups; base < a.rows; base += (int64_t)gridDim.x * kGroups) {
        const bool on = base + index < a.rows;
        const int row = on ? (int)(base + index) : 0;
        const int W = on ? a.width - lane : 0;
        const XT* x = static_cast<const XT*>(a.x) + row_offset(row, a.heads, a.width, a.ld_x) + lane;
        const YT* dy = static_cast<const YT*>(a.dy) + row_offset(row, a.heads, a.width, a.ld_dy) + lane;
        float n[kEach], g[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) n[i] = load_if(x + i * G, i * G < W);
#pragma unroll
        for (int i = 0; i < kEach; ++i) g[i] = load_if(dy + i * G, i * G < W);
        const float r = on ? a.rstd[row] : 0.f, mean = LAYER && on ? a.mean[row] : 0.f;
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            n[i] = i * G < W ? (n[i] - mean) * r : 0.f;
            acc_w[i] = fmaf(g[i], n[i], acc_w[i]);
            if (LAYER) acc_b[i] += g[i];
            g[i] *= weight[i];
            s[0] = fmaf(g[i], n[i], s[0]);
            if (LAYER) s[1] += g[i];
        }
        group_sum(s, G, index, scratch, half);
        const float c0 = -s[0] * inv * r, c1 = LAYER ? s[1] * inv : 0.f;
        const XT* ds = static_cast<const XT*>(a.d_sum) + row_offset(row, a.heads, a.width, a.ld_d_sum) + lane;
        XT* dx = static_cast<XT*>(a.dx) + row_offset(row, a.heads, a.width, a.ld_dx) + lane;
        if (a.has_d_sum) {
            float d[kEach];
#pragma unroll
            for (int i = 0; i < kEach; ++i) d[i] = load_if(ds + i * G, i * G < W);
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                if (i * G < W) dx[i * G] = from_float<XT>(fmaf(g[i] - c1, r, n[i] * c0) + d[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                if (i * G < W) dx[i * G] = from_float<XT>(fmaf(g[i] - c1, r, n[i] * c0));
        }
    }
#pragma unroll
    for (int which = 0; which < (LAYER ? 2 : 1); ++which) {
        float* out = which ? a.part_b : a.part_w;
        if (!out) continue;
        out += (int64_t)blockIdx.x * a.width;
        float* own = kGroups == 1 ? out : sums + index * a.width;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (i * G + lane < a.width) own[i * G + lane] = which ? acc_b[LAYER ? i : 0] : acc_w[i];
        if (kGroups == 1) continue;
        __syncthreads();
        for (int c = threadIdx.x; c < a.width; c += blockDim.x) {
            float t = 0.f;
            for (int k = 0; k < kGroups; ++k) t += sums[k * a.width + c];
            out[c] = t;
        }
    }
}

// Rounded once: over fp32, a sum next to the middle between two numbers of 16 bits would lose what decides.
__device__ __forceinline__ void store_any(void* p, int type, int64_t i, double v) {
    if (type == 0) static_cast<float*>(p)[i] = (float)v;
    else if (type == 1) static_cast<__nv_bfloat16*>(p)[i] = __double2bfloat16(v);
    else static_cast<__half*>(p)[i] = __double2half(v);
}
// dw (block row 0) and db (row 1): the blocks' sums of 32 columns, 32 runs of blocks side by side.  7 us for 296 x 2048, most of it launch
// and two chains of loads; the last block of the kernel before would have 2.4 MB to read alone.
__global__ void __launch_bounds__(1024) norm_columns_kernel(const float* part_w, const float* part_b, int blocks, int width, void* dw,
                                                            void* db, int type, int accumulate) {
    __shared__ double s[32][33];
    const float* part = blockIdx.y ? part_b : part_w;
    void* out = blockIdx.y ? db : dw;
    const int c = blockIdx.x * 32 + threadIdx.x;
    double t = 0.;
    pdl_wait();
    if (out && c < width) {
#pragma unroll 8
        for (int b = threadIdx.y; b < blocks; b += 32) t += part[(int64_t)b * width + c];
    }
    s[threadIdx.y][threadIdx.x] = t;
    __syncthreads();
    if (threadIdx.y == 0 && out && c < width) {
        t = 0.;
        for (int i = 0; i < 32; ++i) t += s[i][threadIdx.x];
        if (accumulate) t += (double)load_any(out, type, c);
        store_any(out, type, c, t);
    }
}

int64_t row_blocks(int64_t rows, int groups) { return (rows + groups - 1) / groups; }

template <typename XT, typename YT>
cudaError_t norm_typed(const NormArgs& a, bool vector, int sms, cudaStream_t st) {
    const NormPlan p = norm_plan(a.width);
    const int scalar = scalar_group(a.width);
    const int64_t blocks = row_blocks(a.rows, vector ? p.block / p.group : scalar_block(scalar) / scalar);
    const int64_t most = (int64_t)sms * (vector ? forward_blocks(p.nv, sizeof(XT) == 4) : scalar < 512 ? 3 : 1);
    const dim3 grid((unsigned)(blocks < most ? blocks : most)), block(vector ? p.block : scalar_block(scalar));
    if (vector) {
        if (p.nv == 1) return launch_plain(norm_rows_kernel<XT, YT, 1>, grid, block, 0, st, a, p.group);
        if (p.nv == 2) return launch_plain(norm_rows_kernel<XT, YT, 2>, grid, block, 0, st, a, p.group);
        return launch_plain(norm_rows_kernel<XT, YT, 4>, grid, block, 0, st, a, p.group);
    }
    switch (scalar) {
        case 32: return launch_plain(norm_scalar_kernel<XT, YT, 32>, grid, block, 0, st, a);
        case 64: return launch_plain(norm_scalar_kernel<XT, YT, 64>, grid, block, 0, st, a);
        case 128: return launch_plain(norm_scalar_kernel<XT, YT, 128>, grid, block, 0, st, a);
        case 256: return launch_plain(norm_scalar_kernel<XT, YT, 256>, grid, block, 0, st, a);
        default: return launch_plain(norm_scalar_kernel<XT, YT, 512>, grid, block, 0, st, a);
    }
}

struct GradPlan {
    NormPlan p;
    bool vector;
    int blocks, smem;
};
GradPlan grad_plan(int64_t rows, int width, bool layer, bool x_is_fp32, bool vector, int sms) {
    GradPlan g;
    g.vector = vector;
    g.p = norm_plan(width);
    if (!vector) {
        g.p.group = scalar_group(width);
        g.p.block = scalar_block(g.p.group);
        g.p.nv = 0;
    }
    const int groups = g.p.block / g.p.group;
    g.smem = vector || groups > 1 ? groups * width * 4 : 0;
    // as many blocks as run at once
    const int most = sms * (vector ? grad_blocks_sm(g.p.nv, x_is_fp32, layer) : g.p.group < 512 ? 2 : 1);
    const int together = vector ? rows_together(g.p.nv) : 1;
    const int64_t need = (row_blocks(rows, groups) + together - 1) / together;
    g.blocks = (int)(need < 1 ? 1 : need < most ? need : most);
    return g;
}
template <typename XT, typename YT, bool LAYER>
cudaError_t norm_grad_typed(const NormGradArgs& a, const GradPlan& g, cudaStream_t st) {
    const dim3 grid(g.blocks), block(g.p.block);
    if (!g.vector) {
        switch (g.p.group) {
            case 32: return launch_plain(norm_grad_scalar_kernel<XT, YT, 32, LAYER>, grid, block, g.smem, st, a);
            case 64: return launch_plain(norm_grad_scalar_kernel<XT, YT, 64, LAYER>, grid, block, g.smem, st, a);
            case 128: return launch_plain(norm_grad_scalar_kernel<XT, YT, 128, LAYER>, grid, block, g.smem, st, a);
            case 256: return launch_plain(norm_grad_scalar_kernel<XT, YT, 256, LAYER>, grid, block, g.smem, st, a);
            default: return launch_plain(norm_grad_scalar_kernel<XT, YT, 512, LAYER>, grid, block, g.smem, st, a);
        }
    }
    if (g.p.group * g.p.nv * kChunk == a.width) {
        if (g.p.nv == 1) return launch_plain(norm_grad_rows_kernel<XT, YT, 1, LAYER, true>, grid, block, g.smem, st, a, g.p.group);
        if (g.p.nv == 2) return launch_plain(norm_grad_rows_kernel<XT, YT, 2, LAYER, true>, grid, block, g.smem, st, a, g.p.group);
        return launch_plain(norm_grad_rows_kernel<XT, YT, 4, LAYER, true>, grid, block, g.smem, st, a, g.p.group);
    }
    if (g.p.nv == 1) return launch_plain(norm_grad_rows_kernel<XT, YT, 1, LAYER, false>, grid, block, g.smem, st, a, g.p.group);
    if (g.p.nv == 2) return launch_plain(norm_grad_rows_kernel<XT, YT, 2, LAYER, false>, grid, block, g.smem, st, a, g.p.group);
    return launch_plain(norm_grad_rows_kernel<XT, YT, 4, LAYER, false>, grid, block, g.smem, st, a, g.p.group);
}

template <typename XT, typename YT, bool LAYER>
cudaError_t init_grad_rows() {
    return init_all(0, norm_grad_rows_kernel<XT, YT, 1, LAYER, false>, norm_grad_rows_kernel<XT, YT, 2, LAYER, false>,
                    norm_grad_rows_kernel<XT, YT, 4, LAYER, false>, norm_grad_rows_kernel<XT, YT, 1, LAYER, true>,
                    norm_grad_rows_kernel<XT, YT, 2, LAYER, true>, norm_grad_rows_kernel<XT, YT, 4, LAYER, true>,
                    norm_grad_scalar_kernel<XT, YT, 32, LAYER>, norm_grad_scalar_kernel<XT, YT, 64, LAYER>,
                    norm_grad_scalar_kernel<XT, YT, 128, LAYER>, norm_grad_scalar_kernel<XT, YT, 256, LAYER>,
                    norm_grad_scalar_kernel<XT, YT, 512, LAYER>);
}

// x and y of one type, or x fp32 (a residual stream) and y of 16 bits.
template <typename F>
cudaError_t for_types(int x_type, int y_type, F f) {
    if (x_type == 1) return f((__nv_bfloat16*)nullptr, (__nv_bfloat16*)nullptr);
    if (x_type == 2) return f((__half*)nullptr, (__half*)nullptr);
    if (y_type == 1) return f((float*)nullptr, (__nv_bfloat16*)nullptr);
    if (y_type == 2) return f((float*)nullptr, (__half*)nullptr);
    return f((float*)nullptr, (float*)nullptr);
}

}  // namespace

// Sums of dw or db: blocks x width (grad_plan: at most three blocks on an SM up to a width of 256, two up to 4096, one beyond).
size_t norm_grad_part_bytes(int max_width) {
    size_t most = 0;
    const int limit[3] = {256, 4096, kNormMaxWidth};
    for (int i = 0; i < 3; ++i) {
        const size_t n = (size_t)(3 - i) * (size_t)(max_width < limit[i] ? max_width : limit[i]);
        if (n > most) most = n;
    }
    return (size_t)kTrainSms * most * 4;
}

cudaError_t init_norm_kernels() {
    for (int t = 0; t < 5; ++t) {
        const cudaError_t e = for_types(t < 3 ? 0 : t - 2, t < 3 ? t : t - 2, [&](auto* x, auto* y) {
            using XT = std::remove_pointer_t<decltype(x)>;
            using YT = std::remove_pointer_t<decltype(y)>;
            cudaError_t r = init_all(0, norm_rows_kernel<XT, YT, 1>, norm_rows_kernel<XT, YT, 2>, norm_rows_kernel<XT, YT, 4>, norm_scalar_kernel<XT, YT, 32>,
                                     norm_scalar_kernel<XT, YT, 64>, norm_scalar_kernel<XT, YT, 128>, norm_scalar_kernel<XT, YT, 256>,
                                     norm_scalar_kernel<XT, YT, 512>);
            if (r == cudaSuccess) r = init_grad_rows<XT, YT, false>();
            if (r == cudaSuccess) r = init_grad_rows<XT, YT, true>();
            return r;
        });
        if (e != cudaSuccess) return e;
    }
    return init_all(0, norm_columns_kernel);
}

cudaError_t launch_norm(const NormArgs& a, int x_type, int y_type, bool vector, int sms, cudaStream_t st) {
    return for_types(x_type, y_type, [&](auto* x, auto* y) {
        using XT = std::remove_pointer_t<decltype(x)>;
        using YT = std::remove_pointer_t<decltype(y)>;
        return norm_typed<XT, YT>(a, vector, sms, st);
    });
}
cudaError_t launch_norm_grad(const NormGradArgs& a, int x_type, int y_type, bool vector, int sms, void* dw, void* db, int dw_type,
                             int accumulate, cudaStream_t st) {
    const GradPlan g = grad_plan(a.rows, a.width, a.layer, x_type == 0, vector, sms);
    if (a.rows > 0) {
        const cudaError_t e = for_types(x_type, y_type, [&](auto* x, auto* y) {
            using XT = std::remove_pointer_t<decltype(x)>;
            using YT = std::remove_pointer_t<decltype(y)>;
            return a.layer ? norm_grad_typed<XT, YT, true>(a, g, st) : norm_grad_typed<XT, YT, false>(a, g, st);
        });
        if (e != cudaSuccess) return e;
    }
    if (!dw && !db) return cudaSuccess;
    const dim3 grid((unsigned)((a.width + 31) / 32), db ? 2u : 1u), block(32, 32);
    const float *w = a.part_w, *b = a.part_b;
    if (a.rows == 0) return launch_plain(norm_columns_kernel, grid, block, 0, st, w, b, 0, a.width, dw, db, dw_type, accumulate);
    return launch_second(norm_columns_kernel, grid, block, 0, st, w, b, g.blocks, a.width, dw, db, dw_type, accumulate);
}

}  // namespace mars
