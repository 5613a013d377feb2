// Rotation of the heads of q and k by their positions:
//   (a, b) -> scale (a cos t - b sin t, b cos t + a sin t),  t = position x frequency of the pair,
// pairs (i, i + rotary / 2) or (2i, 2i + 1) of the first `rotary` values of a head, the rest of it passes.  The inverse (sign -1)
// is the transposed matrix and so the gradient.
// Bound by HBM: q and k are read and written once.  A thread keeps one place in the head (eight pairs of the half layout, four
// of the interleaved one, in 16-byte pieces; or one pair) for a token, so that the sines of a place are taken once for
// all heads it passes over.  Angles are in turns: position x turns in fp64 minus the nearest whole number.  The table's entries are rounded
// once, from 64 bits, and so is the product: together they are off by 2^-52 of the number of turns (4e-11 of a turn at position 10^6, 8e-8 at
// 2^31).  The fraction is rounded to fp32 for sincospif: 1.5e-8 of a turn, 9.4e-8 of a radian, about the error of the functions themselves.
// Measured (B200, copy rate 6463 GB/s): 65536 tokens x 36 heads x 128 bf16 187 us, at the copy rate; 2048 tokens 10.3 us, of which the data
// would take 6: launch, the chain position - sines - loads, and the store.  Asking for the first heads before the sines are taken costs
// registers, 183 -> 206 us for 65536 tokens; whether it would gain in one wave of blocks is not measured.
#include "train.h"
#include "train_types.cuh"

namespace mars {

namespace {

constexpr int kBatch = 3;            // heads whose loads a thread has in flight together (80 registers, three blocks on an SM)

__device__ __forceinline__ void sines(const RopeArgs& a, int pos, int pair, float& c, float& s) {
    const double t = (double)pos * a.turns[pair];
    const float f = (float)(t - rint(t));
    sincospif(2.f * f, &s, &c);
    c *= a.scale;
    s *= a.scale * a.sign;
}

// Threads of a token: `units` places in a head x `slots` heads side by side.
template <typename T, bool INTER>
__global__ void __launch_bounds__(256) rope_vec_kernel(const RopeArgs a, const int units, const int slots) {
    const int per = units * slots, tokens_here = blockDim.x / per;
    const int local = threadIdx.x / per, rest = threadIdx.x - local * per;
    const int64_t token = (int64_t)blockIdx.x * tokens_here + local;
    if (local >= tokens_here || token >= a.tokens) return;
    const int slot = rest / units, u = rest - slot * units;
    const int half = a.rotary / 2, turning = INTER ? a.rotary / 8 : half / 8;
    const bool pass = u >= turning;
    constexpr int P = INTER ? 4 : 8;
    float c[P], s[P];
    int at, at2 = 0;                                           // places in the head
    if (pass) {
        at = a.rotary + (u - turning) * 8;
    } else {
        at = u * 8;
        at2 = half + u * 8;
        const int pos = a.positions[token];
#pragma unroll
        for (int i = 0; i < P; ++i) sines(a, pos, u * P + i, c[i], s[i]);
    }
    const int heads = a.heads[0] + a.heads[1];
    const T *in_q = static_cast<const T*>(a.in[0]) + token * a.ld_in[0], *in_k = static_cast<const T*>(a.in[1]) + token * a.ld_in[1];
    T *out_q = static_cast<T*>(a.out[0]) + token * a.ld_out[0], *out_k = static_cast<T*>(a.out[1]) + token * a.ld_out[1];
    for (int h0 = slot; h0 < heads; h0 += kBatch * slots) {
        Raw8<T> x[kBatch], y[kBatch];
        T* out[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            int h = h0 + b * slots;
            out[b] = nullptr;
            if (h < heads) {
                const int w = h >= a.heads[0];
                h -= w ? a.heads[0] : 0;
                const T* in = (w ? in_k : in_q) + (int64_t)h * a.head_dim;
                out[b] = (w ? out_k : out_q) + (int64_t)h * a.head_dim;
                if (pass && in == out[b]) {
                    out[b] = nullptr;
                } else {
                    x[b] = load8(in + at);
                    if (!INTER && !pass) y[b] = load8(in + at2);
                }
            }
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            if (!out[b]) continue;
            if (!pass) {
                float v[8];
                unpack8<T>(x[b], v);
                if (INTER) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p = v[2 * i], q = v[2 * i + 1];
                        v[2 * i] = p * c[i] - q * s[i];
                        v[2 * i + 1] = q * c[i] + p * s[i];
                    }
                } else {
                    float w[8];
                    unpack8<T>(y[b], w);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float p = v[i], q = w[i];
                        v[i] = p * c[i % P] - q * s[i % P];
                        w[i] = q * c[i % P] + p * s[i % P];
                    }
                    store8(out[b] + at2, pack8<T>(w));
                }
                x[b] = pack8<T>(v);
            }
            store8(out[b] + at, x[b]);
        }
    }
}

// Any alignment and number of pairs: one pair, or one value that passes, for each thread; 2 or 4 bytes a load (20000 tokens x 36 heads x 80
// bf16, 40 values turned: 137 us, 1.7 TB/s).
template <typename T>
__global__ void __launch_bounds__(512) rope_kernel(const RopeArgs a, const int units, const int slots) {
    const int per = units * slots, tokens_here = blockDim.x / per;
    const int local = threadIdx.x / per, rest = threadIdx.x - local * per;
    const int64_t token = (int64_t)blockIdx.x * tokens_here + local;
    if (local >= tokens_here || token >= a.tokens) return;
    const int slot = rest / units, u = rest - slot * units, half = a.rotary / 2;
    const bool pass = u >= half;
    const int at = pass ? a.rotary + (u - half) : a.interleaved ? 2 * u : u, at2 = a.interleaved ? 2 * u + 1 : u + half;
    float c = 0.f, s = 0.f;
    if (!pass) sines(a, a.positions[token], u, c, s);
    const int heads = a.heads[0] + a.heads[1];
    const T *in_q = static_cast<const T*>(a.in[0]) + token * a.ld_in[0], *in_k = static_cast<const T*>(a.in[1]) + token * a.ld_in[1];
    T *out_q = static_cast<T*>(a.out[0]) + token * a.ld_out[0], *out_k = static_cast<T*>(a.out[1]) + token * a.ld_out[1];
    for (int h0 = slot; h0 < heads; h0 += kBatch * slots) {
        T x[kBatch], y[kBatch];
        T* out[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            int h = h0 + b * slots;
            out[b] = nullptr;
            if (h < heads) {
                const int w = h >= a.heads[0];
                h -= w ? a.heads[0] : 0;
                const T* in = (w ? in_k : in_q) + (int64_t)h * a.head_dim;
                out[b] = (w ? out_k : out_q) + (int64_t)h * a.head_dim;
                x[b] = in[at];
                if (!pass) y[b] = in[at2];
            }
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            if (!out[b]) continue;
            if (pass) {
                out[b][at] = x[b];
            } else {
                const float p = to_float(x[b]), q = to_float(y[b]);
                out[b][at] = from_float<T>(p * c - q * s);
                out[b][at2] = from_float<T>(q * c + p * s);
            }
        }
    }
}

template <typename T>
cudaError_t rope_typed(const RopeArgs& a, bool vector, int sms, cudaStream_t st) {
    const int heads = a.heads[0] + a.heads[1];
    const int turning = vector ? (a.interleaved ? a.rotary / 8 : a.rotary / 16) : a.rotary / 2;
    const int units = turning + (a.head_dim - a.rotary) / (vector ? 8 : 1);
    // One to three batches of heads for a thread: three share its sines best, one gives the most threads.  The waves of blocks (768 threads
    // on an SM), each as long as the batches and one more for start and sines, decide: 2048 tokens of 36 x 128 bf16 one batch (two waves)
    // 12.3 us, two (one wave) 10.6, three 10.7; 512 tokens 5.0 / - / 5.5; 4096 tokens 19.8 / 16.9 / 17.9; 32768 125 / - / 94.
    int slots = 1;
    int64_t least = INT64_MAX;
    for (int batches = 1; batches <= 3; ++batches) {
        const int s = (heads + batches * kBatch - 1) / (batches * kBatch);
        const int64_t waves = ((int64_t)a.tokens * units * s + sms * 768 - 1) / (sms * 768), cost = waves * (batches + 1);
        if (cost <= least) { least = cost; slots = s; }
    }
    if (slots * units > 256) slots = units < 256 ? 256 / units : 1;
    const int per = units * slots;
    const int block = per > 256 ? (per + 31) / 32 * 32 : 256, tokens_here = block / per;
    const dim3 grid((unsigned)(((int64_t)a.tokens + tokens_here - 1) / tokens_here));
    if (!vector) return launch_plain(rope_kernel<T>, grid, dim3(block), 0, st, a, units, slots);
    if (a.interleaved) return launch_plain(rope_vec_kernel<T, true>, grid, dim3(block), 0, st, a, units, slots);
    return launch_plain(rope_vec_kernel<T, false>, grid, dim3(block), 0, st, a, units, slots);
}

template <typename T>
cudaError_t rope_init() { return init_all(0, rope_vec_kernel<T, false>, rope_vec_kernel<T, true>, rope_kernel<T>); }

}  // namespace

cudaError_t init_rope_kernels() {
    const cudaError_t a = rope_init<float>(), b = rope_init<__nv_bfloat16>(), c = rope_init<__half>();
    return a != cudaSuccess ? a : b != cudaSuccess ? b : c;
}

cudaError_t launch_rope(const RopeArgs& a, int type, bool vector, int sms, cudaStream_t st) {
    if (type == 0) return rope_typed<float>(a, vector, sms, st);
    if (type == 1) return rope_typed<__nv_bfloat16>(a, vector, sms, st);
    return rope_typed<__half>(a, vector, sms, st);
}

}  // namespace mars
