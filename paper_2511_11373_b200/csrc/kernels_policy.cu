// Clipped policy loss with a KL term towards a reference policy, and its gradient to the log-probs.  Of every token with a
// target, r = exp(logp - old):
//   term = -min(r A, clip(r, 1 - low, 1 + high) A) + kl (exp(x) - x - 1),  x = ref - logp
//   d term / d logp = -A r where the first of the two is the smaller (or they are equal), + kl (1 - exp(x))
// weighted by 1 / live tokens, by 1 / (live sequences x the sequence's live tokens), or not at all, times `scale`.
// Bound by HBM for long batches (16 to 24 bytes a token) and by latency for short ones.  No gradient may be written before
// the tokens are counted, so a first kernel counts them (targets alone, which then lie in L2) with integer atomics, whose order
// changes nothing; sums of terms are fp64 of a thread's own tokens in order, then of the blocks in order by the last one to
// finish: the same call gives the same bits.  Which side of a border a ratio is on is decided in fp64 on logp - old, against
// the borders' logarithms.  A token's sequence is found by all threads of a block together (256 offsets a step).
#include "train.h"
#include "train_types.cuh"

namespace mars {

namespace {

constexpr int kThreads = 256, kTile = kThreads * 4;

// Number of the offsets seq_off[1 ..] in [lo, lo + len) that are at most t, plus lo; all threads of the block call it.
__device__ __forceinline__ int find_sequence(const int32_t* seq_off, int lo, int len, int t) {
    while (len > 0) {
        const int step = (len + kThreads - 1) / kThreads, p = ((int)threadIdx.x + 1) * step - 1;
        const int passed = __syncthreads_count(p < len && seq_off[1 + lo + p] <= t);
        lo += passed * step;
        len = min(step - 1, len - passed * step);
    }
    return lo;
}
__device__ __forceinline__ int find_here(const int32_t* seq_off, int lo, int hi, int t) {     // first s in [lo, hi] with t < off[s + 1], else hi
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (seq_off[1 + mid] <= t) lo = mid + 1; else hi = mid;
    }
    return lo;
}

// Sequences of a tile of tokens: [first, last] (last = seqs where the tile reaches behind the last sequence).
struct TileSeqs { int first, last; };
__device__ __forceinline__ TileSeqs tile_sequences(const PolicyArgs& a, int t0, int t1) {
    TileSeqs s;
    s.first = find_sequence(a.seq_off, 0, a.seqs, t0);
    s.last = s.first;
    if (s.first < a.seqs && a.seq_off[1 + s.first] <= t1) s.last = find_sequence(a.seq_off, s.first, a.seqs - s.first, t1);
    return s;
}

__global__ void __launch_bounds__(kThreads) policy_count_kernel(const PolicyArgs a) {
    __shared__ int last, sum[kThreads / 32], seqs[kThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, begin = a.seq_off[0];
    for (int64_t base = (int64_t)blockIdx.x * kTile; base < a.tokens; base += (int64_t)gridDim.x * kTile) {
        const int t0 = (int)base, t1 = (int)min((int64_t)a.tokens, base + kTile) - 1;
        const TileSeqs s = tile_sequences(a, t0, t1);
        const int t = t0 + (int)threadIdx.x * 4;
        int count = 0, at = -1, bound = 0;
        for (int i = 0; i < 4; ++i) {
            if (t + i > t1 || t + i < begin || a.targets[t + i] < 0) continue;
            if (at < 0 || t + i >= bound) {
                if (count) atomicAdd(a.seq_live + at, count);
                count = 0;
                at = find_here(a.seq_off, s.first, s.last, t + i);
                if (at >= a.seqs) break;                      // behind the last sequence
                bound = a.seq_off[1 + at];
            }
            ++count;
        }
        if (s.first == s.last) {                              // one sequence: one addition for each warp
            const int all = __reduce_add_sync(0xffffffffu, count);
            if (lane == 0 && all) atomicAdd(a.seq_live + s.first, all);
        } else if (count) {
            atomicAdd(a.seq_live + at, count);
        }
    }
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(a.ticket, 1) == (int)gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    int n = 0, held = 0;
    for (int s = threadIdx.x; s < a.seqs; s += kThreads) {
        const int c = __ldcg(a.seq_live + s);
        n += c;
        held += c > 0;
    }
    n = __reduce_add_sync(0xffffffffu, n);
    held = __reduce_add_sync(0xffffffffu, held);
    if (lane == 0) { sum[warp] = n; seqs[warp] = held; }
    __syncthreads();
    if (threadIdx.x == 0) {
        n = held = 0;
        for (int w = 0; w < kThreads / 32; ++w) { n += sum[w]; held += seqs[w]; }
        a.totals[0] = n;
        a.totals[1] = held;
        a.ticket[0] = 0;
    }
}

// exp(x) - 1 - x without cancellation: the series below 1/2, where the difference would lose two bits and more.
__device__ __forceinline__ float exp_minus_line(float x, float em1) {
    if (!(fabsf(x) < 0.5f)) return em1 - x;
    float s = 1.f / 40320.f;
    s = fmaf(s, x, 1.f / 5040.f);
    s = fmaf(s, x, 1.f / 720.f);
    s = fmaf(s, x, 1.f / 120.f);
    s = fmaf(s, x, 1.f / 24.f);
    s = fmaf(s, x, 1.f / 6.f);
    s = fmaf(s, x, 0.5f);
    return s * x * x;
}

__global__ void __launch_bounds__(kThreads, 4) policy_loss_kernel(const PolicyArgs a) {
    __shared__ double reduce[kThreads / 32][4];
    __shared__ int last;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, begin = a.seq_off[0];
    const int live = a.totals[0], held = a.totals[1];
    double sums[4] = {0., 0., 0., 0.};                        // loss, kl, cut ratios, ratios
    for (int64_t base = (int64_t)blockIdx.x * kTile; base < a.tokens; base += (int64_t)gridDim.x * kTile) {
        const int t0 = (int)base, t1 = (int)min((int64_t)a.tokens, base + kTile) - 1;
        const TileSeqs s = tile_sequences(a, t0, t1);
        const int t = t0 + (int)threadIdx.x * 4;
        int at = -1, bound = 0;
        double share = 0.;
        float adv = 0.f;
        for (int i = 0; i < 4; ++i) {
            if (t + i > t1) break;
            float d = 0.f;
            if (t + i >= begin && a.targets[t + i] >= 0) {
                if (at < 0 || t + i >= bound) {
                    at = find_here(a.seq_off, s.first, s.last, t + i);
                    if (at < a.seqs) {
                        bound = a.seq_off[1 + at];
                        share = a.scale;
                        if (a.reduce == 0) share /= live;
                        if (a.reduce == 1) share /= (double)held * __ldcg(a.seq_live + at);
                        if (!a.per_token) adv = a.adv[at];
                    } else {
                        bound = INT32_MAX;
                    }
                }
                if (at < a.seqs) {
                    const float lp = a.lp[t + i], A = a.per_token ? a.adv[t + i] : adv;
                    const double dd = (double)lp - (double)a.old_lp[t + i];
                    const float r = expf((float)dd);
                    const bool over = dd > a.log_high, under = dd < a.log_low;
                    const bool cut = (over && A > 0.f) || (under && A < 0.f);
                    float term = -(cut ? (over ? a.high : a.low) : r) * A;
                    d = cut ? 0.f : -A * r;
                    if (a.has_ref) {
                        const float x = (float)((double)a.ref[t + i] - (double)lp), em1 = expm1f(x), kl = exp_minus_line(x, em1);
                        if (a.kl != 0.f) {
                            term = fmaf(a.kl, kl, term);
                            d = fmaf(-a.kl, em1, d);
                        }
                        sums[1] += kl;
                    }
                    sums[0] += share * term;
                    sums[2] += cut;
                    sums[3] += r;
                    d = (float)(share * d);
                }
            }
            if (a.d_lp) a.d_lp[t + i] = d;
        }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) sums[q] = warp_sum_double(sums[q]);
    if (lane == 0)
        for (int q = 0; q < 4; ++q) reduce[warp][q] = sums[q];
    __syncthreads();
    if (threadIdx.x < 4) {
        double v = 0.;
        for (int w = 0; w < kThreads / 32; ++w) v += reduce[w][threadIdx.x];
        a.parts[(int64_t)blockIdx.x * 4 + threadIdx.x] = v;
    }
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(a.ticket + 1, 1) == (int)gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    for (int s = threadIdx.x; s < a.seqs; s += kThreads) a.seq_live[s] = 0;
    // thread = 4 x run of blocks + sum
    double v = 0.;
    for (int b = threadIdx.x >> 2; b < (int)gridDim.x; b += kThreads / 4) v += __ldcg(a.parts + (int64_t)b * 4 + (threadIdx.x & 3));
#pragma unroll
    for (int o = 16; o >= 4; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if (lane < 4) reduce[warp][lane] = v;
    __syncthreads();
    if (threadIdx.x < 4) {
        v = 0.;
        for (int w = 0; w < kThreads / 32; ++w) v += reduce[w][threadIdx.x];
        a.stats[threadIdx.x] = (float)(threadIdx.x == 0 ? v : live ? v / live : 0.);
        if (threadIdx.x == 0) {
            a.stats[4] = (float)live;
            a.stats[5] = (float)held;
            a.ticket[1] = 0;
        }
    }
}

int policy_blocks(int tokens, int sms) {
    const int64_t tiles = ((int64_t)tokens + kTile - 1) / kTile;
    const int most = policy_max_blocks(sms);
    return (int)(tiles < 1 ? 1 : tiles < most ? tiles : most);
}

}  // namespace

cudaError_t init_policy_kernels() { return init_all(0, policy_count_kernel, policy_loss_kernel); }

int policy_max_blocks(int sms) { return (sms < kTrainSms ? sms : kTrainSms) * 8; }

cudaError_t launch_policy_loss(const PolicyArgs& a, int sms, cudaStream_t st) {
    const dim3 grid(policy_blocks(a.tokens, sms)), block(kThreads);
    const cudaError_t e = launch_plain(policy_count_kernel, grid, block, 0, st, a);
    if (e != cudaSuccess) return e;
    return launch_plain(policy_loss_kernel, grid, block, 0, st, a);
}

}  // namespace mars
