// The mixture's router in training: softmax over the experts, the k largest (the lower index on ties), their weights, and what
// the balance and z losses need; and the gradient of the logits.
//   p = softmax(z), lse = log sum exp z;   weights p_i, or p_i / sum of the selected p
//   balance = E sum_e f_e P_e,  f_e = counts_e / (N k),  P_e = sum_t p_te / N;   z loss = sum_t lse_t^2 / N;   N live rows
//   d z_j = p_j (g_j - sum_e p_e g_e) + 2 c_z lse / N p_j + (weights), g_e = c_b E f_e / N
//   weights' part: renormalised, over the selected: w_i (dw_i - sum w dw);  else  p_j ([j selected] dw_j - sum p dw)
// A warp has a row: its lanes hold the logits in registers, in neighbouring fours where alignment allows.  Logits are compared
// as integers that order like them; a lane keeps the best of its own, a round takes the largest of the lanes and, among
// equals, the lowest expert.  Sums over rows stay in fp32 registers for the rows of a warp, go through shared memory
// in the order of the warps, and the last block to finish adds the blocks' sums in fp64: the same call gives the same bits.
#include "train.h"
#include "train_types.cuh"

namespace mars {

namespace {

template <int NG> constexpr int kWarpsOf = NG == 8 ? 8 : 16;     // more registers for 32 logits of a lane

// Place of element i of group j of a lane among the experts.
template <bool V>
__device__ __forceinline__ int expert_of(int j, int i, int lane) { return V ? (j * 32 + lane) * 4 + i : (j * 4 + i) * 32 + lane; }

template <typename T, bool V>
__device__ __forceinline__ void load4(const T* row, int j, int lane, int experts, float (&o)[4], float fill) {
    if (V) {
        const int c = (j * 32 + lane) * 4;
        if (c >= experts) {
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = fill;
        } else if (sizeof(T) == 4) {
            const float4 v = *reinterpret_cast<const float4*>(row + c);
            o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w;
        } else {
            const uint2 v = *reinterpret_cast<const uint2*>(row + c);
            if constexpr (sizeof(T) == 2) {
                unpack2(v.x, o[0], o[1], T());
                unpack2(v.y, o[2], o[3], T());
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = expert_of<false>(j, i, lane);
            o[i] = load_if(row + c, c < experts);
            if (c >= experts) o[i] = fill;
        }
    }
}
// The same for groups of L lanes.
template <typename T, int L, bool V>
__device__ __forceinline__ void group_load4(const T* row, int j, int l, int experts, float (&o)[4]) {
    if constexpr (V) {
        const int c = (j * L + l) * 4;
        if (c >= experts) {
            o[0] = o[1] = o[2] = o[3] = 0.f;
        } else if constexpr (sizeof(T) == 4) {
            const float4 v = *reinterpret_cast<const float4*>(row + c);
            o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w;
        } else {
            const uint2 v = *reinterpret_cast<const uint2*>(row + c);
            unpack2(v.x, o[0], o[1], T());
            unpack2(v.y, o[2], o[3], T());
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = (j * 4 + i) * L + l;
            o[i] = load_if(row + c, c < experts);
        }
    }
}
// Four values as they lie in memory.
template <typename T> struct Four { uint2 v; };
template <> struct Four<float> { float4 v; };
__device__ __forceinline__ void unpack_four(const Four<float>& f, float2 (&o)[2]) {
    o[0] = make_float2(f.v.x, f.v.y);
    o[1] = make_float2(f.v.z, f.v.w);
}
template <typename T>
__device__ __forceinline__ void unpack_four(const Four<T>& f, float2 (&o)[2]) {
    unpack2(f.v.x, o[0].x, o[0].y, T());
    unpack2(f.v.y, o[1].x, o[1].y, T());
}
// -inf in all four
__device__ __forceinline__ uint32_t two_neg_inf(__nv_bfloat16) { return 0xff80ff80u; }
__device__ __forceinline__ uint32_t two_neg_inf(__half) { return 0xfc00fc00u; }
__device__ __forceinline__ void clear_four(Four<float>& f) { f.v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY); }
template <typename T>
__device__ __forceinline__ void clear_four(Four<T>& f) { f.v = make_uint2(two_neg_inf(T()), two_neg_inf(T())); }
// -inf behind the last expert
template <typename T, int L, bool V>
__device__ __forceinline__ Four<T> load_four(const T* row, int j, int l, int experts) {
    Four<T> f;
    if constexpr (V) {
        const int c = (j * L + l) * 4;
        clear_four(f);
        if (c < experts) f.v = *reinterpret_cast<const decltype(f.v)*>(row + c);
    } else {
        float o[4];
        group_load4<T, L, false>(row, j, l, experts, o);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if ((j * 4 + i) * L + l >= experts) o[i] = -INFINITY;
        if constexpr (sizeof(T) == 4) f.v = make_float4(o[0], o[1], o[2], o[3]);
        else f.v = make_uint2(pack2(o[0], o[1], T()), pack2(o[2], o[3], T()));
    }
    return f;
}
template <typename T, int L, bool V>
__device__ __forceinline__ void group_store4(T* row, int j, int l, int experts, const float (&v)[4]) {
    if constexpr (V) {
        const int c = (j * L + l) * 4;
        if (c >= experts) return;
        if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(row + c) = make_float4(v[0], v[1], v[2], v[3]);
        else *reinterpret_cast<uint2*>(row + c) = make_uint2(pack2(v[0], v[1], T()), pack2(v[2], v[3], T()));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int c = (j * 4 + i) * L + l;
            if (c < experts) row[c] = from_float<T>(v[i]);
        }
    }
}

// Unsigned integers that order like the floats; -0 counts as 0, a NaN as the largest.  0 is below the key of -inf.
__device__ __forceinline__ uint32_t order_key(float v) {
    if (v != v) return 0xffffffffu;
    const uint32_t b = __float_as_uint(v + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu)); }
constexpr uint32_t kKeyNegInf = 0x007fffffu;
constexpr float kLog2e = 1.44269504f;

// The end of a block: its sums and counts for all, and by the last block the call's totals.  sums, counts: [experts] in shared memory,
// complete; z: the sum of lse^2 of lane 0 of each warp.  The last block has all its loads in flight together; a block that is alone has
// none.
template <int WARPS>
__device__ __forceinline__ void router_finish(const RouterArgs& a, float* sums, int* counts, double z) {
    __shared__ double reduce[WARPS], part[WARPS * 32];
    __shared__ int last, scan[WARPS];
    constexpr int THREADS = WARPS * 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, E = a.experts, blocks = gridDim.x;
    if (lane == 0) reduce[warp] = z;
    __syncthreads();
    z = 0.;
    for (int w = 0; w < WARPS; ++w) z += reduce[w];
    if (blocks > 1) {
        for (int e = threadIdx.x; e < E; e += THREADS) {
            a.parts[(int64_t)blockIdx.x * E + e] = sums[e];
            if (counts[e]) atomicAdd(&a.work_counts[e], counts[e]);
        }
        if (threadIdx.x == 0) a.z_parts[blockIdx.x] = z;
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) last = atomicAdd(a.ticket, 1) == blocks - 1;
        __syncthreads();
        if (!last) return;
        __threadfence();
    }
    // a thread's share of the columns' sums: as many threads for a column as there are for all columns at once, each with a run of blocks
    const int slices = max(1, min(16, THREADS / E)), here = min(E, THREADS), slice = threadIdx.x / here, column = threadIdx.x - slice * here;
    auto column_sum = [&](int c) {
        if (blocks == 1) return slice == 0 ? (double)sums[c] : 0.;
        double v = 0.;
#pragma unroll 16
        for (int b = blocks * slice / slices; b < blocks * (slice + 1) / slices; ++b) v += __ldcg(a.parts + (int64_t)b * E + c);
        return v;
    };
    // counts: every thread has a run of neighbouring experts
    const int each = (E + THREADS - 1) / THREADS;
    int run = 0;
    for (int i = 0; i < each; ++i) {
        const int e = threadIdx.x * each + i;
        if (e < E) run += blocks > 1 ? __ldcg(a.work_counts + e) : counts[e];
    }
    double v = slice < slices ? column_sum(column) : 0., zs = 0.;
    if (blocks > 1)
        for (int b = threadIdx.x; b < blocks; b += THREADS) zs += __ldcg(a.z_parts + b);
    else if (threadIdx.x == 0)
        zs = z;
    int before = run;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, before, o);
        if (lane >= o) before += up;
    }
    zs = warp_sum_double(zs);
    __syncthreads();                                          // counts of this block and its z are read
    if (lane == 31) scan[warp] = before;
    if (lane == 0) reduce[warp] = zs;
    part[threadIdx.x] = v;
    __syncthreads();
    int base = 0, total = 0;
    z = 0.;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
        if (w < warp) base += scan[w];
        total += scan[w];
        z += reduce[w];
    }
    int at = base + before - run;
    for (int i = 0; i < each; ++i) {
        const int e = threadIdx.x * each + i;
        if (e >= E) break;
        const int n = blocks == 1 ? counts[e] : each == 1 ? run : __ldcg(a.work_counts + e);
        if (a.offsets) a.offsets[e] = at;
        at += n;
        if (a.counts) a.counts[e] = n;
        counts[e] = n;
        if (blocks > 1) a.work_counts[e] = 0;
    }
    if (threadIdx.x == 0) {
        if (a.offsets) a.offsets[E] = total;
        *a.ticket = 0;
    }
    __syncthreads();
    double balance = 0.;
    for (int c0 = 0; c0 < E; c0 += THREADS) {
        const int c = c0 + column;
        if (c0 > 0) v = c < E ? column_sum(c) : 0.;           // more columns than threads
        if (slice == 0 && c < E) {
            for (int i = 1; i < slices; ++i) v += part[i * here + threadIdx.x];
            if (a.prob_sums) a.prob_sums[c] = (float)v;
            balance += v * counts[c];
        }
    }
    balance = warp_sum_double(balance);
    __syncthreads();
    if (lane == 0) reduce[warp] = balance;
    __syncthreads();
    if (threadIdx.x == 0 && a.losses) {
        balance = 0.;
        for (int w = 0; w < WARPS; ++w) balance += reduce[w];
        const double n = (double)total / a.top_k;
        a.losses[0] = n > 0. ? (float)(E * balance / (n * n * a.top_k)) : 0.f;
        a.losses[1] = n > 0. ? (float)(z / n) : 0.f;
    }
}

template <typename T, int NG, bool V>
__global__ void __launch_bounds__(kWarpsOf<NG> * 32, NG <= 2 ? 2 : 1) router_kernel(const RouterArgs a) {
    constexpr int kWarps = kWarpsOf<NG>, kThreads = kWarps * 32;
    __shared__ float sums[kRouterMaxExperts];
    __shared__ int counts[kRouterMaxExperts];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, E = a.experts, k = a.top_k;
    for (int e = threadIdx.x; e < E; e += kThreads) { sums[e] = 0.f; counts[e] = 0; }
    __syncthreads();
    float acc[NG][4];
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
    double z = 0.;
    for (int64_t row = (int64_t)blockIdx.x * kWarps + warp; row < a.rows; row += (int64_t)gridDim.x * kWarps) {
        bool on = !a.has_live || a.live[row];
        float v[NG][4];
        uint32_t key[NG][4], best = 0;
        int at = 0;
        if (on) {
#pragma unroll
            for (int j = 0; j < NG; ++j) load4<T, V>(static_cast<const T*>(a.logits) + row * a.ld, j, lane, E, v[j], 0.f);
#pragma unroll
            for (int j = 0; j < NG; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    key[j][i] = expert_of<V>(j, i, lane) < E ? order_key(v[j][i]) : 0u;
                    if (key[j][i] > best) { best = key[j][i]; at = expert_of<V>(j, i, lane); }
                }
        }
        const uint32_t top = __reduce_max_sync(0xffffffffu, best);
        on = on && top > kKeyNegInf;                          // a row without a logit above -inf takes no part
        if (!on) {
            if (lane < k) { a.idx[row * k + lane] = -1; a.weights[row * k + lane] = 0.f; }
            if (a.lse && lane == 0) a.lse[row] = 0.f;
            continue;
        }
        const float m = key_value(top);
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < NG; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[j][i] = expert_of<V>(j, i, lane) < E ? expf(v[j][i] - m) : 0.f;
                sum += v[j][i];
            }
        sum = warp_sum(sum);
        const float inv = 1.f / sum;
#pragma unroll
        for (int j = 0; j < NG; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[j][i] = fmaf(v[j][i], inv, acc[j][i]);
        uint32_t mine = 0;                                    // lane i: key and expert of place i
        int chosen = 0;
        for (int i = 0; i < k; ++i) {
            const uint32_t most = i == 0 ? top : __reduce_max_sync(0xffffffffu, best);
            const int e = (int)__reduce_min_sync(0xffffffffu, best == most ? (uint32_t)at : 0xffffffffu);
            if (lane == i) { mine = most; chosen = e; }
            if (best == most && at == e) {
                best = 0;
#pragma unroll
                for (int j = 0; j < NG; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        if (expert_of<V>(j, q, lane) == e) key[j][q] = 0;
                        if (key[j][q] > best) { best = key[j][q]; at = expert_of<V>(j, q, lane); }
                    }
            }
        }
        const float w = lane < k ? expf(key_value(mine) - m) : 0.f;
        const float total = a.renormalise ? warp_sum(w) : sum;
        if (lane < k) {
            a.idx[row * k + lane] = chosen;
            a.weights[row * k + lane] = w / total;
            atomicAdd(&counts[chosen], 1);
        }
        const float lse = m + logf(sum);
        if (lane == 0) {
            if (a.lse) a.lse[row] = lse;
            z += (double)lse * (double)lse;
        }
    }
    for (int w = 0; w < kWarps; ++w) {
        if (w == warp)
#pragma unroll
            for (int j = 0; j < NG; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (expert_of<V>(j, i, lane) < E) sums[expert_of<V>(j, i, lane)] += acc[j][i];
        __syncthreads();
    }
    router_finish<kWarps>(a, sums, counts, z);
}

// Many rows: two threads have a row, each half of its columns.  A warp brings 16 rows into shared memory (fp32, rows apart by an odd number
// of 16 bytes, so that eight threads read their 16 bytes from different banks) and goes over them thread by thread.  The k <= 8 largest of a
// row lie in the eight fours with the largest maxima; both choices, of fours and of logits, are made on 32-bit keys (leading bits that order
// like the value, last bits that prefer the lower index), eight at a time: sorted (Batcher's odd-even merge, 19 exchanges) and merged into
// the eight largest so far (the larger ones of the two ends, then a bitonic merge of 12 exchanges), and so are the two halves.  The keys hold
// bf16 and fp16 in full; for fp32 a row whose last choice and largest loser agree in the leading bits, or whose choices are out of order, is
// checked against the values, and chosen again by the warp where that shows a difference.  The same pass over the row takes the
// exponentials, which go back to shared memory; the lanes then add the columns up.
// Bound by instructions and their latency: 136 of a warp for a row of 128 experts, where rounds over a warp take 590.  131072 x 128 fp32,
// 8 choices: 44 us (1.5 TB/s; the rounds 117), of which 17 are there for any number of rows: one tile's chain 8, launch 3, the meeting of the
// blocks 5.  50000 x 384: 60 us, the rounds 138.  One thread for a row took the 44 us too, with half the warps.
// From kManyRows on, one number for all widths and so a compromise: the two meet at some 6000 rows of 128 experts, 3000 of 384 and 10000 of 16.
// fp32, rounds / this kernel: 4096 x 128 14.2 / 16.9 us, 8192 x 128 20.4 / 17.8, 32768 x 128 39 / 22; 2048 x 384 20 / 26, 4096 x 384 34 / 29,
// 8192 x 384 46 / 30; 8192 x 16 13.8 / 15.2, 16384 x 16 18.3 / 15.5.
// Exponentials are ex2.approx of a product that is rounded once: off by some (max - z) 2^-23 of themselves, where expf, which the rounds
// take, has half of it for far logits (the argument z - max is rounded in both).  expf here: 44.4 -> 47.8 us, and the weights' error against 64
// bits goes from 6.9e-8 to 6.7e-8 of their norm (spread 1; 7.9e-8 for both at 16).
constexpr int kManyExperts = 512, kManyK = 8, kManyRows = 8192;
// Warps of the one block that an SM's shared memory holds: few blocks leave few sums for the last one to add.
// COLUMNS: 128 experts each.
template <int COLUMNS> constexpr int kManyWarps = 24 / COLUMNS;
constexpr int kTileRows = 16;
__host__ __device__ constexpr int many_pitch(int experts) { return (experts + 63) / 64 * 64 + 4; }

__device__ __forceinline__ void exchange(uint32_t& a, uint32_t& b) {       // the larger one first
    const uint32_t m = max(a, b);
    b = min(a, b);
    a = m;
}
__device__ __forceinline__ void sort8(uint32_t (&k)[8]) {
    exchange(k[0], k[1]); exchange(k[2], k[3]); exchange(k[4], k[5]); exchange(k[6], k[7]);
    exchange(k[0], k[2]); exchange(k[1], k[3]); exchange(k[4], k[6]); exchange(k[5], k[7]);
    exchange(k[1], k[2]); exchange(k[5], k[6]);
    exchange(k[0], k[4]); exchange(k[1], k[5]); exchange(k[2], k[6]); exchange(k[3], k[7]);
    exchange(k[2], k[4]); exchange(k[3], k[5]);
    exchange(k[1], k[2]); exchange(k[3], k[4]); exchange(k[5], k[6]);
}

// Merges eight sorted keys into the eight largest so far; lost: the largest that is not among them.
__device__ __forceinline__ void merge8(uint32_t (&best)[8], const uint32_t (&key)[8], uint32_t& lost) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        lost = max(lost, min(best[i], key[7 - i]));
        best[i] = max(best[i], key[7 - i]);
    }
#pragma unroll
    for (int d = 4; d > 0; d >>= 1)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((i & d) == 0) exchange(best[i], best[i + d]);
}
__device__ __forceinline__ void take8(uint32_t (&best)[8], uint32_t (&key)[8], uint32_t& lost) {
    sort8(key);
    merge8(best, key, lost);
}
// The leading bits of a float as an integer that orders like it (-0 as 0).
template <uint32_t LOW>
__device__ __forceinline__ uint32_t leading(float v) {
    const uint32_t b = __float_as_uint(v + 0.f);
    return (b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u)) & ~LOW;
}

template <typename T, bool V, int kColumns>
__global__ void __launch_bounds__(kManyWarps<kColumns> * 32, 1) router_many_kernel(const RouterArgs a) {
    constexpr int kWarps = kManyWarps<kColumns>, kThreads = kWarps * 32;
    // the last bits of a key: the largest number of a logit, or of a four, minus its number
    constexpr int kBits = kColumns > 2 ? 9 : 8;
    constexpr uint32_t kLow = (1u << kBits) - 1, kLowFour = kLow >> 2;
    extern __shared__ float tiles[];                          // [warps][16][pitch]
    __shared__ float sums[kColumns * 128], scale[kWarps][kTileRows];
    __shared__ int counts[kColumns * 128];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, E = a.experts, k = a.top_k, pitch = many_pitch(E), padded = pitch - 4, fours = (E + 3) / 4;
    const int r = lane & 15, h = lane >> 4, half = padded / 2;           // row of the tile and half of it
    float* tile = tiles + warp * kTileRows * pitch;
    float* mine = tile + r * pitch;
    for (int e = threadIdx.x; e < E; e += kThreads) { sums[e] = 0.f; counts[e] = 0; }
    __syncthreads();
    float acc[kColumns][4];
#pragma unroll
    for (int j = 0; j < kColumns; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;
    double z2 = 0.;
    const bool packed = k % 4 == 0 && (((uintptr_t)a.idx | (uintptr_t)a.weights) & 15) == 0;
    const int64_t stride = (int64_t)gridDim.x * kWarps * kTileRows;
    for (int64_t base = ((int64_t)warp * gridDim.x + blockIdx.x) * kTileRows; base < a.rows; base += stride) {     // few tiles: one for each SM first
        const int rows = (int)min((int64_t)kTileRows, a.rows - base);
        // the tile
        const T* in = static_cast<const T*>(a.logits) + base * a.ld;
        if (V && sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < kColumns; ++j) {
                const int c = j * 128 + lane * 4;
                if (c < E) {
                    const T* from = in + c;
                    float* to = tile + c;
                    const int64_t ld = a.ld;
#pragma unroll 8
                    for (int q = 0; q < rows; ++q, from += ld, to += pitch) cp_async16(to, from);
                }
            }
            cp_async_commit();
        } else if (V) {
            for (int r0 = 0; r0 < rows; r0 += 8)              // four values of 16 bits a load, eight rows' loads in flight
                for (int f = lane; f < fours; f += 32) {
                    float v[8][4];
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (r0 + q < rows) group_load4<T, 1, true>(in + (r0 + q) * a.ld + f * 4, 0, 0, 4, v[q]);
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (r0 + q < rows) *reinterpret_cast<float4*>(tile + (r0 + q) * pitch + f * 4) = make_float4(v[q][0], v[q][1], v[q][2], v[q][3]);
                }
        } else {
            for (int r0 = 0; r0 < rows; r0 += 8)
                for (int c = lane; c < E; c += 32) {
                    float v[8];
#pragma unroll
                    for (int q = 0; q < 8; ++q) v[q] = load_if(in + (r0 + q) * a.ld + c, r0 + q < rows);
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (r0 + q < rows) tile[(r0 + q) * pitch + c] = v[q];
                }
        }
        if (h) for (int c = E; c < padded; ++c) mine[c] = -INFINITY;
        const int64_t row = base + r;
        bool on = r < rows && (!a.has_live || a.live[row]);
        if (V && sizeof(T) == 4) cp_async_wait<0>();
        __syncwarp();
        // of this half the eight fours with the largest maxima, and the eight largest of them
        uint32_t groups[8] = {0, 0, 0, 0, 0, 0, 0, 0}, best[8] = {0, 0, 0, 0, 0, 0, 0, 0}, lost_group = 0, lost = 0;
        const int first = h * half / 4;                       // its first four
        if (half > 32) {
            for (int c = 0; c < half / 32; ++c) {
                uint32_t key[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int g = first + c * 8 + i;
                    const float4 v = *reinterpret_cast<const float4*>(mine + g * 4);
                    key[i] = leading<kLowFour>(fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w))) | (kLowFour - g);
                }
                take8(groups, key, lost_group);
            }
        } else {                                              // eight fours in all
#pragma unroll
            for (int i = 0; i < 8; ++i) groups[i] = ~kLowFour | (kLowFour - first - i);
        }
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            uint32_t key[8];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int g = min((int)(kLowFour - (groups[i + q] & kLowFour)), padded / 4 - 1);
                const float4 v = *reinterpret_cast<const float4*>(mine + g * 4);
                const uint32_t code = kLow - g * 4;
                key[q * 4] = leading<kLow>(v.x) | code;
                key[q * 4 + 1] = leading<kLow>(v.y) | (code - 1);
                key[q * 4 + 2] = leading<kLow>(v.z) | (code - 2);
                key[q * 4 + 3] = leading<kLow>(v.w) | (code - 3);
            }
            take8(best, key, lost);
        }
        {                                                     // with the other half
            uint32_t key[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) key[i] = __shfl_xor_sync(0xffffffffu, best[i], 16);
            merge8(best, key, lost);
            lost = max(lost, __shfl_xor_sync(0xffffffffu, lost, 16));
        }
        int idx[8];
        float val[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            idx[i] = min((int)(kLow - (best[i] & kLow)), E - 1);
            val[i] = mine[idx[i]];
        }
        float m = val[0], sum = 0.f;
        if (sizeof(T) == 4) {
            float least = val[0];
            uint32_t last = best[0], next = best[1];          // of the chosen, and the one behind it
            bool sorted = true;
#pragma unroll
            for (int i = 1; i < 8; ++i)
                if (i < k) {
                    sorted = sorted && (val[i - 1] > val[i] || (val[i - 1] == val[i] && idx[i - 1] < idx[i]));
                    least = val[i];
                    last = best[i];
                    next = i < 7 ? best[i < 7 ? i + 1 : 7] : 0u;
                }
            bool close = !sorted || (last >> kBits) == (max(next, lost) >> kBits) || (groups[7] >> (kBits - 2)) == (lost_group >> (kBits - 2));
            int larger = 0, above = 0;                        // logits, and chosen ones, that are larger than the least chosen
            if (__any_sync(0xffffffffu, on && close)) {
                for (int c = first; c < min(fours, first + half / 4); ++c) {
                    const float4 v = *reinterpret_cast<const float4*>(mine + c * 4);
                    larger += (v.x > least) + (v.y > least) + (v.z > least) + (v.w > least);
                }
                larger += __shfl_xor_sync(0xffffffffu, larger, 16);
#pragma unroll
                for (int i = 0; i < 8; ++i) above += i < k && val[i] > least;
            }
            // rows whose choice is not that of the values: the warp chooses again, one row after the other
            unsigned again = __ballot_sync(0xffffffffu, on && (!sorted || larger != above) && !(m != m)) & 0xffffu;
            while (again) {
                const int bad = __ffs(again) - 1;
                again &= again - 1;
                const float* other = tile + bad * pitch;
                uint32_t key[kColumns * 4];
#pragma unroll
                for (int j = 0; j < kColumns * 4; ++j) key[j] = j * 32 + lane < E ? order_key(other[j * 32 + lane]) : 0u;
                for (int i = 0; i < k; ++i) {
                    uint32_t top = 0;
                    int at = 0;
#pragma unroll
                    for (int j = 0; j < kColumns * 4; ++j)
                        if (key[j] > top) { top = key[j]; at = j * 32 + lane; }
                    const uint32_t most = __reduce_max_sync(0xffffffffu, top);
                    const int e = (int)__reduce_min_sync(0xffffffffu, top == most ? (uint32_t)at : 0xffffffffu);
#pragma unroll
                    for (int j = 0; j < kColumns * 4; ++j)
                        if (j * 32 + lane == e) key[j] = 0;
                    if (r == bad) {
#pragma unroll
                        for (int q = 0; q < 8; ++q)
                            if (q == i) { idx[q] = e; val[q] = mine[e]; }
                    }
                }
            }
            m = val[0];
        }
        // Nothing above -inf, or a NaN: the maxima of the fours pass over it, and with more than 64 experts its four need not be among the eight.
        if (__any_sync(0xffffffffu, on && m == -INFINITY)) {
            bool nan = false;
            for (int c = first; c < min(fours, first + half / 4); ++c) {
                const float4 v = *reinterpret_cast<const float4*>(mine + c * 4);
                nan = nan || v.x != v.x || v.y != v.y || v.z != v.z || v.w != v.w;
            }
            nan = __shfl_xor_sync(0xffffffffu, nan, 16) || nan;
            if (nan && m == -INFINITY) m = NAN;               // and so all that follows
        }
        on = on && !(m == -INFINITY);                         // a row without a logit above -inf takes no part
        __syncwarp();                                         // a half's exponentials take the place of what the other may still look at
        const int end = min(fours, first + half / 4);
        if (on) {
#pragma unroll 4
            for (int c = first; c < end; ++c) {
                float4 v = *reinterpret_cast<const float4*>(mine + c * 4);
                v.x = ex2((v.x - m) * kLog2e);
                v.y = ex2((v.y - m) * kLog2e);
                v.z = ex2((v.z - m) * kLog2e);
                v.w = ex2((v.w - m) * kLog2e);
                sum += (v.x + v.y) + (v.z + v.w);
                *reinterpret_cast<float4*>(mine + c * 4) = v;
            }
        } else {
            for (int c = first; c < end; ++c) *reinterpret_cast<float4*>(mine + c * 4) = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        sum += __shfl_xor_sync(0xffffffffu, sum, 16);
        float w[8], total = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            w[i] = i < k && on ? ex2((val[i] - m) * kLog2e) : 0.f;
            total += w[i];
        }
        // (a NaN in the row makes its sum NaN, and the weights)
        const float inv = !on ? 0.f : sum != sum ? sum : 1.f / (a.renormalise ? total : sum), lse = on ? m + logf(sum) : 0.f;
        if (h == 0) scale[warp][r] = on ? 1.f / sum : 0.f;
        if (r < rows) {
            if (h == 0) {                                     // the choices by one thread of a row, the weights by the other
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    idx[i] = on ? idx[i] : -1;
                    if (i < k && on) atomicAdd(&counts[idx[i]], 1);
                }
                if (packed) {
#pragma unroll
                    for (int i = 0; i < 8; i += 4)
                        if (i < k) *reinterpret_cast<int4*>(a.idx + row * k + i) = make_int4(idx[i], idx[i + 1], idx[i + 2], idx[i + 3]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i < k) a.idx[row * k + i] = idx[i];
                }
                if (a.lse) a.lse[row] = lse;
                z2 += (double)lse * (double)lse;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) w[i] *= inv;
                if (packed) {
#pragma unroll
                    for (int i = 0; i < 8; i += 4)
                        if (i < k) *reinterpret_cast<float4*>(a.weights + row * k + i) = make_float4(w[i], w[i + 1], w[i + 2], w[i + 3]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i < k) a.weights[row * k + i] = w[i];
                }
            }
        }
        __syncwarp();
        // columns (rows that take no part are zeros)
#pragma unroll
        for (int j = 0; j < kColumns; ++j) {
            const int c = j * 128 + lane * 4;
            if (c < fours * 4) {
#pragma unroll 8
                for (int q = 0; q < kTileRows; ++q) {
                    const float4 v = *reinterpret_cast<const float4*>(tile + q * pitch + c);
                    const float s = scale[warp][q];
                    acc[j][0] = fmaf(v.x, s, acc[j][0]);
                    acc[j][1] = fmaf(v.y, s, acc[j][1]);
                    acc[j][2] = fmaf(v.z, s, acc[j][2]);
                    acc[j][3] = fmaf(v.w, s, acc[j][3]);
                }
            }
        }
        __syncwarp();
    }
    for (int w = 0; w < kWarps; ++w) {
        if (w == warp)
#pragma unroll
            for (int j = 0; j < kColumns; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (j * 128 + lane * 4 + i < E) sums[j * 128 + lane * 4 + i] += acc[j][i];
        __syncthreads();
    }
    router_finish<kWarps>(a, sums, counts, warp_sum_double(z2));
}

template <int BYTES>
__device__ __forceinline__ void copy_async(void* smem_dst, const void* gsrc) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_u32(smem_dst)), "l"(gsrc), "n"(BYTES));
}
// Adds v to a place that holds 0 but for an expert that was chosen twice: an exchange is one instruction in shared memory, an addition a loop.
__device__ __forceinline__ void put(float* place, float v) {
    const float before = atomicExch(place, v);
    if (before != 0.f) atomicAdd(place, before);
}
constexpr int kAhead = 4;
constexpr float kNearLse = 8.f;
// Blocks on an SM: three of 16-bit logits, two of fp32 (shared memory of the ring), one of more than 512 experts.
template <typename T, int NG> constexpr int kGradBlocks = NG > 4 ? 1 : sizeof(T) == 2 ? 3 : 2;
template <typename T, int L, int NG, bool V>
constexpr int grad_smem(int experts) {
    return 8 * (32 / L) * ((experts + 3) / 4 * 4 + 4) * 4 + (V ? 8 * kAhead * 32 * (NG * 4 * (int)sizeof(T) + 12) : 0);
}
// Gradient: L lanes have a row (so that a warp reduces several rows in one go), NG fours of experts each.  Bound by the bytes
// that are on their way and by instructions: 131072 x 128 bf16 22 us (3.4 TB/s), fp32 26 (5.5 TB/s); without d_weights 17 and 24.  A warp
// for a row took 600 instructions of it and 70 us; eight lanes with the next two rows in registers, two blocks on an SM, 24 and 30; the
// weights' part added up in shared memory instead of exchanged + 1.  Exponentials as above, and the quotients by the approximate reciprocal (two
// steps): with expf and true quotients 22.6 -> 25.9 us for an error of 1.15e-7 instead of 1.37e-7 of the gradient's norm.
template <typename T, int L, int NG, bool V>
__global__ void __launch_bounds__(256, (kGradBlocks<T, NG>)) router_grad_kernel(const RouterGradArgs a) {
    constexpr int kWarps = 8, kThreads = 256, R = 32 / L;     // rows of a warp
    extern __shared__ float smem[];                           // [rows of the block][pitch]: the weights' part of a row
    __shared__ double reduce[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, E = a.experts, k = a.top_k;
    const int sub = lane / L, l = lane % L, pitch = (E + 3) / 4 * 4 + 4;
    float* mine = smem + (warp * R + sub) * pitch;
    double total = 0.;
    for (int e = threadIdx.x; e < E; e += kThreads) total += a.counts[e];
    total = warp_sum_double(total);
    if (lane == 0) reduce[warp] = total;
    for (int i = threadIdx.x; i < kWarps * R * pitch; i += kThreads) smem[i] = 0.f;
    __syncthreads();
    total = 0.;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) total += reduce[w];
    const double n = total > 0. ? total / k : 1.;             // live rows
    const float unit = total > 0. ? (float)((double)a.balance * E / n / total) : 0.f, zc = (float)(2. * (double)a.z / n);
    auto expert = [&](int j, int i) { return V ? (j * L + l) * 4 + i : (j * 4 + i) * L + l; };
    float2 g[NG][2];
#pragma unroll
    for (int j = 0; j < NG; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i)
            g[j][i] = make_float2(expert(j, 2 * i) < E ? unit * a.counts[expert(j, 2 * i)] : 0.f,
                                  expert(j, 2 * i + 1) < E ? unit * a.counts[expert(j, 2 * i + 1)] : 0.f);
    // Logits, lse and the first L choices of a row, with the weights' gradients.  Rows that allow it come by asynchronous copies into a ring of
    // kAhead stages, three of them on their way while a row is worked on; a thread copies what it will read.  Others come by loads, one row ahead.
    Four<T> z[NG];
    float row_lse = 0.f, row_dw = 0.f;
    int row_idx = -1;
    auto fetch = [&](int64_t row) {
        const bool in_range = row < a.rows;
        const int64_t r = in_range ? row : 0;
#pragma unroll
        for (int j = 0; j < NG; ++j) z[j] = load_four<T, L, V>(static_cast<const T*>(a.logits) + r * a.ld, j, l, in_range ? E : 0);
        row_lse = in_range ? a.lse[r] : 0.f;
        row_idx = in_range && l < k ? a.idx[r * k + l] : -1;
        row_dw = in_range && l < k && a.has_d_weights ? a.d_weights[r * k + l] : 0.f;
    };
    Four<T>* ring = reinterpret_cast<Four<T>*>(smem + kWarps * R * pitch) + warp * kAhead * NG * 32;                 // [stage][NG][lane]
    float* tail = smem + kWarps * R * pitch + kWarps * kAhead * NG * 32 * (int)sizeof(Four<T>) / 4 + warp * kAhead * 96;      // [stage][lse, dw, idx][lane]
    auto request = [&](int64_t row, int stage) {
        if (row < a.rows) {
            const T* in = static_cast<const T*>(a.logits) + row * a.ld + l * 4;
#pragma unroll
            for (int j = 0; j < NG; ++j)
                if (expert(j, 0) < E) copy_async<sizeof(Four<T>)>(ring + (stage * NG + j) * 32 + lane, in + j * L * 4);
            float* s = tail + stage * 96 + lane;
            copy_async<4>(s, a.lse + row);
            if (l < k) {
                copy_async<4>(s + 64, a.idx + row * k + l);
                if (a.has_d_weights) copy_async<4>(s + 32, a.d_weights + row * k + l);
            }
        }
        cp_async_commit();
    };
    const int64_t stride = (int64_t)gridDim.x * kWarps * R;
    int64_t base = ((int64_t)blockIdx.x * kWarps + warp) * R;
    int stage = 0;
    if constexpr (V) {
#pragma unroll
        for (int s = 0; s < kAhead - 1; ++s) request(base + s * stride + sub, s);
    } else {
        fetch(base + sub);
    }
    for (; base < a.rows; base += stride) {
        const bool in_range = base + sub < a.rows;
        const int64_t row = in_range ? base + sub : 0;
        const T* in = static_cast<const T*>(a.logits) + row * a.ld;
        T* out = static_cast<T*>(a.d_logits) + row * a.ld_d;
        const int here = stage;
        if constexpr (V) {
            cp_async_wait<kAhead - 2>();
            __syncwarp();                                     // all lanes have this stage, and are done with the one that is filled again
            request(base + (kAhead - 1) * stride + sub, (stage + kAhead - 1) % kAhead);
            stage = (stage + 1) % kAhead;
#pragma unroll
            for (int j = 0; j < NG; ++j) {
                clear_four(z[j]);
                if (expert(j, 0) < E) z[j] = ring[(here * NG + j) * 32 + lane];
            }
            const float* s = tail + here * 96 + lane;
            row_lse = s[0];
            row_dw = s[32];
            row_idx = in_range && l < k ? __float_as_int(s[64]) : -1;
        }
        auto logit = [&](int e) {
            if constexpr (V) {
                const int f = e / 4;
                return to_float(reinterpret_cast<const T*>(ring + (here * NG + f / L) * 32 + sub * L + f % L)[e % 4]);
            } else {
                return to_float(in[e]);
            }
        };
        const int first_idx = row_idx;
        const bool on = __shfl_sync(0xffffffffu, row_idx, sub * L) >= 0;      // a row that took no part may hold anything
        const float lse = on ? row_lse : 0.f, first_dw = row_dw;
        float2 v[NG][2], dots = make_float2(0.f, 0.f);
#pragma unroll
        for (int j = 0; j < NG; ++j) {
            if (!on) clear_four(z[j]);                        // p = 0, and so is all that follows
            unpack_four(z[j], v[j]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                v[j][i] = mul2(add2(v[j][i], make_float2(-lse, -lse)), make_float2(kLog2e, kLog2e));
                v[j][i] = make_float2(ex2(v[j][i].x), ex2(v[j][i].y));
                dots = fma2(v[j][i], g[j][i], dots);
            }
        }
        float dot = dots.x + dots.y;                          // sum of p g, plus that of the selected where weights are p
        float w_first = 0.f;                                  // p of this lane's first choice
        if (a.has_d_weights && on && (unsigned)first_idx < (unsigned)E) w_first = ex2((logit(first_idx) - lse) * kLog2e);
        if constexpr (!V) fetch(base + stride + sub);
        // p = v / sum of the row's v.  That is 1 but for lse's rounding to its last bit, by which every v is off alike: 2^-22 of itself at most where
        // |lse| < kNearLse, as much as the exponential, but 3e-5 for logits around 1000 and a factor of E where all are the lowest number.  So
        // rows farther out are divided by it; for all of them it costs 131072 x 128 bf16 1.6 us of 24.
        const bool far = on && !(fabsf(lse) < kNearLse);
        float unite = 1.f;
        if (__any_sync(0xffffffffu, far)) {
            float2 sums = make_float2(0.f, 0.f);
#pragma unroll
            for (int j = 0; j < NG; ++j) sums = add2(sums, add2(v[j][0], v[j][1]));
            float sum = sums.x + sums.y;
#pragma unroll
            for (int o = L / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (far) unite = __fdividef(1.f, sum);
        }
        if (a.has_d_weights) {
            // of renormalised weights' gradients only differences count: taken from that of the first choice, a weight next to 1 keeps the
            // accuracy of what the others leave it
            const float from = a.renormalise ? __shfl_sync(0xffffffffu, (unsigned)first_idx < (unsigned)E ? first_dw : 0.f, sub * L) : 0.f;
            float w_sum = w_first, wdw = w_first != 0.f ? w_first * (first_dw - from) : 0.f;
            for (int i = l + L; i < k; i += L) {
                const int e = on ? a.idx[row * k + i] : -1;
                if ((unsigned)e < (unsigned)E) {
                    const float w = ex2((logit(e) - lse) * kLog2e);
                    w_sum += w;
                    wdw = fmaf(w, a.d_weights[row * k + i] - from, wdw);
                }
            }
#pragma unroll
            for (int o = L / 2; o > 0; o >>= 1) {
                w_sum += __shfl_xor_sync(0xffffffffu, w_sum, o);
                wdw += __shfl_xor_sync(0xffffffffu, wdw, o);
            }
            const float inv = a.renormalise ? __fdividef(1.f, w_sum) : unite, mean = a.renormalise ? wdw * inv : 0.f;
            if (on && (unsigned)first_idx < (unsigned)E) put(mine + first_idx, w_first * inv * (first_dw - from - mean));
            for (int i = l + L; i < k; i += L) {
                const int e = on ? a.idx[row * k + i] : -1;
                if ((unsigned)e < (unsigned)E)
                    put(mine + e, ex2((logit(e) - lse) * kLog2e) * inv * (a.d_weights[row * k + i] - from - mean));
            }
            if (!a.renormalise) dot += wdw / L;
            __syncwarp();
        }
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
        // where lse^2 passes fp32 the z loss is infinite, and its part stays v lse
        const float shift = fmaf(zc * lse, fabsf(lse) < 0x1p64f ? unite : 1.f, -dot * unite * unite);
#pragma unroll
        for (int j = 0; j < NG; ++j) {
            float2 m[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
            if (a.has_d_weights) {
                if (V) {
                    if (expert(j, 0) < E) {
                        const float4 q = *reinterpret_cast<const float4*>(mine + expert(j, 0));
                        m[0] = make_float2(q.x, q.y);
                        m[1] = make_float2(q.z, q.w);
                        *reinterpret_cast<float4*>(mine + expert(j, 0)) = make_float4(0.f, 0.f, 0.f, 0.f);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (expert(j, i) < E) {
                            (i & 1 ? m[i / 2].y : m[i / 2].x) = mine[expert(j, i)];
                            mine[expert(j, i)] = 0.f;
                        }
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) m[i] = fma2(v[j][i], fma2(g[j][i], make_float2(unite, unite), make_float2(shift, shift)), m[i]);
            const float d[4] = {m[0].x, m[0].y, m[1].x, m[1].y};
            if (in_range) group_store4<T, L, V>(out, j, l, E, d);
        }
        if constexpr (!V) __syncwarp();
    }
}

int router_blocks(int rows, int warps, int sms) {
    const int most = sms * 2, need = (int)(((int64_t)rows + warps - 1) / warps);
    return need < 1 ? 1 : need < most ? need : most;
}

template <typename T, int NG, bool V>
cudaError_t router_launch(const RouterArgs& a, int sms, cudaStream_t st) {
    constexpr int W = kWarpsOf<NG>;
    return launch_plain(router_kernel<T, NG, V>, dim3(router_blocks(a.rows, W, sms)), dim3(W * 32), 0, st, a);
}
template <typename T, bool V>
cudaError_t router_typed(const RouterArgs& a, int sms, cudaStream_t st) {
    if (a.experts <= kManyExperts && a.top_k <= kManyK && a.rows >= kManyRows) {
        const int warps = a.experts <= 128 ? kManyWarps<1> : a.experts <= 256 ? kManyWarps<2> : kManyWarps<4>;
        const int64_t need = ((int64_t)a.rows + kTileRows - 1) / kTileRows;
        return launch_plain(a.experts <= 128 ? router_many_kernel<T, V, 1> : a.experts <= 256 ? router_many_kernel<T, V, 2> : router_many_kernel<T, V, 4>,
                            dim3((unsigned)(need < sms ? need : sms)), dim3(warps * 32), (size_t)warps * kTileRows * many_pitch(a.experts) * 4, st, a);
    }
    if (a.experts <= 128) return router_launch<T, 1, V>(a, sms, st);
    if (a.experts <= 256) return router_launch<T, 2, V>(a, sms, st);
    if (a.experts <= 512) return router_launch<T, 4, V>(a, sms, st);
    return router_launch<T, 8, V>(a, sms, st);
}
template <typename T, int L, int NG, bool V>
cudaError_t router_grad_launch(const RouterGradArgs& a, int sms, cudaStream_t st) {
    constexpr int R = 32 / L;
    const int64_t need = ((int64_t)a.rows + 8 * R - 1) / (8 * R), most = (int64_t)sms * kGradBlocks<T, NG>;
    const size_t smem = grad_smem<T, L, NG, V>(a.experts);
    return launch_plain(router_grad_kernel<T, L, NG, V>, dim3((unsigned)(need < most ? need : most)), dim3(256), smem, st, a);
}
// Sixteen experts for a lane where a row has as many; a row for a whole warp beyond 256.
template <typename T, bool V>
cudaError_t router_grad_typed(const RouterGradArgs& a, int sms, cudaStream_t st) {
    if (a.experts <= 32) return router_grad_launch<T, 4, 2, V>(a, sms, st);
    if (a.experts <= 128) return router_grad_launch<T, 8, 4, V>(a, sms, st);
    if (a.experts <= 256) return router_grad_launch<T, 16, 4, V>(a, sms, st);
    if (a.experts <= 512) return router_grad_launch<T, 32, 4, V>(a, sms, st);
    return router_grad_launch<T, 32, 8, V>(a, sms, st);
}

template <typename T, bool V>
cudaError_t router_init() {
    cudaError_t e = init_all(kManyWarps<1> * kTileRows * many_pitch(128) * 4, router_many_kernel<T, V, 1>);
    if (e == cudaSuccess) e = init_all(kManyWarps<2> * kTileRows * many_pitch(256) * 4, router_many_kernel<T, V, 2>);
    if (e == cudaSuccess) e = init_all(kManyWarps<4> * kTileRows * many_pitch(512) * 4, router_many_kernel<T, V, 4>);
    if (e != cudaSuccess) return e;
    e = init_all(0, router_kernel<T, 1, V>, router_kernel<T, 2, V>, router_kernel<T, 4, V>, router_kernel<T, 8, V>);
    if (e == cudaSuccess) e = init_all(grad_smem<T, 4, 2, V>(32), router_grad_kernel<T, 4, 2, V>);
    if (e == cudaSuccess) e = init_all(grad_smem<T, 8, 4, V>(128), router_grad_kernel<T, 8, 4, V>);
    if (e == cudaSuccess) e = init_all(grad_smem<T, 16, 4, V>(256), router_grad_kernel<T, 16, 4, V>);
    if (e == cudaSuccess) e = init_all(grad_smem<T, 32, 4, V>(512), router_grad_kernel<T, 32, 4, V>);
    if (e == cudaSuccess) e = init_all(grad_smem<T, 32, 8, V>(kRouterMaxExperts), router_grad_kernel<T, 32, 8, V>);
    return e;
}

}  // namespace

cudaError_t init_router_kernels() {
    const cudaError_t all[6] = {router_init<float, false>(), router_init<float, true>(), router_init<__nv_bfloat16, false>(),
                                router_init<__nv_bfloat16, true>(), router_init<__half, false>(), router_init<__half, true>()};
    for (cudaError_t e : all)
        if (e != cudaSuccess) return e;
    return cudaSuccess;
}

int router_max_blocks(int sms) { return (sms < kTrainSms ? sms : kTrainSms) * 2; }

cudaError_t launch_router(const RouterArgs& a, int type, bool vector, int sms, cudaStream_t st) {
    if (type == 0) return vector ? router_typed<float, true>(a, sms, st) : router_typed<float, false>(a, sms, st);
    if (type == 1) return vector ? router_typed<__nv_bfloat16, true>(a, sms, st) : router_typed<__nv_bfloat16, false>(a, sms, st);
    return vector ? router_typed<__half, true>(a, sms, st) : router_typed<__half, false>(a, sms, st);
}
cudaError_t launch_router_grad(const RouterGradArgs& a, int type, bool vector, int sms, cudaStream_t st) {
    if (type == 0) return vector ? router_grad_typed<float, true>(a, sms, st) : router_grad_typed<float, false>(a, sms, st);
    if (type == 1) return vector ? router_grad_typed<__nv_bfloat16, true>(a, sms, st) : router_grad_typed<__nv_bfloat16, false>(a, sms, st);
    return vector ? router_grad_typed<__half, true>(a, sms, st) : router_grad_typed<__half, false>(a, sms, st);
}

}  // namespace mars
