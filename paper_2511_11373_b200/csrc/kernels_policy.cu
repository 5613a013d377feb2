// Clipped policy loss with a KL term towards a reference policy, and its gradient to the log-probs.  Of every token with a
// target, r = exp(logp - old):
//   term = -min(r A, clip(r, 1 - low, 1 + high) A) + kl (exp(x) - x - 1),  x = ref - logp
//   d term / d logp = -A r where the first of the two is the smaller (or they are equal), + kl (1 - exp(x))
// weighted by 1 / live tokens, by 1 / (live sequences x the sequence's live tokens), or not at all, times `scale`.
// Bound by HBM for long batches (16 to 24 bytes a token) and by latency for short ones.  No gradient may be written before
// the tokens are counted, so a first kernel counts them (targets alone, which then lie in L2) with integer atomics, whose order
// changes nothing; the second kernel turns the counts into weights.  Terms are added in fp32 over the four neighbouring tokens of a thread,
// in fp64 beyond, and the blocks' sums in order by the last one to finish: the same call gives the same bits.  Which side of a border a
// ratio is on is decided on logp - old against the borders' logarithms, in fp64 where fp32 is too near.  A warp has one piece of all
// tokens and goes through it in runs; it finds the sequences of a run together, 32 offsets a step, where the run leaves the last one.
// Measured (B200): 4 M tokens of 1024 sequences with a reference 34 us (13 + 24 alone, 37 one after the other; 10 at the copy rate);
// with a search for every block and quad of tokens 58.  What is left are two launches, the first loads, and 80 instructions a token in
// the second kernel; two or four blocks on an SM instead of three 46 and 40 us; the first kernel asking for the second one's lines in L2 + 3.
// Four tokens of one sequence go the short way where |ref - logp| < 1/2 for all of them; others, and advantages for each token, take the general
// one, with their whole warp.  ref = logp + N(0, s): s = 0.1 33 us, 0.15 34, 0.2 40, 0.3 and more 43; advantages for each token 40; no reference 30.
// A sum (MARS_SUM) takes as long as a mean: its weights need no count, its statistics do.
#include "train.h"
#include "train_types.cuh"

namespace mars {

namespace {

constexpr int kThreads = 256, kSmallThreads = 512, kRun = 128;      // a warp works on runs of 128 tokens, four for each lane
// Up to here one block does everything.  One block / two kernels: 256 tokens 6.6 / 8.8 us, 2048 8.4 / 15.3, 4096 12.4 / 15.9, 8192 19.4 / 17.1.
constexpr int kSmallTokens = 4096;

// Four neighbouring values, `fill` behind the last token.
template <typename T>
__device__ __forceinline__ void load_quad(const T* p, int t, int tokens, int vector, T fill, T (&v)[4]) {
    if (vector && t + 4 <= tokens) {
        const int4 w = *reinterpret_cast<const int4*>(p + t);
        const int u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const T*>(&u[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = t + i < tokens ? p[t + i] : fill;
    }
}

// Number of the offsets seq_off[1 ..] in [lo, lo + len) that are at most t, plus lo; all lanes of a warp look for the same t.
__device__ __forceinline__ int find_sequence(const int32_t* seq_off, int lo, int len, int t) {
    const int lane = threadIdx.x & 31;
    while (len > 0) {
        const int step = (len + 31) / 32, p = (lane + 1) * step - 1;
        const int passed = __popc(__ballot_sync(0xffffffffu, p < len && seq_off[1 + lo + min(p, len - 1)] <= t));
        lo += passed * step;
        len = min(step - 1, len - passed * step);
    }
    return lo;
}
// The same by one lane: the first s in [lo, hi] whose end lies behind t, else hi.
__device__ __forceinline__ int find_here(const int32_t* seq_off, int lo, int hi, int t) {
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (seq_off[1 + mid] <= t) lo = mid + 1; else hi = mid;
    }
    return lo;
}

// The tokens of a warp: a piece [begin, end) of all, in whole runs.
struct Piece { int begin, end; };
__device__ __forceinline__ Piece warp_piece(int tokens, int run, int warp, int warps) {
    const int64_t runs = ((int64_t)tokens + run - 1) / run;
    Piece p;
    p.begin = (int)min((int64_t)tokens, runs * warp / warps * run);
    p.end = (int)min((int64_t)tokens, runs * (warp + 1) / warps * run);
    return p;
}
// Moves first to the sequence of token t0 and returns that of token t1 (seqs: behind the last one).
__device__ __forceinline__ int advance(const PolicyArgs& a, int& first, int t0, int t1) {
    if (first < a.seqs && a.seq_off[1 + first] <= t0) first = find_sequence(a.seq_off, first, a.seqs - first, t0);
    if (first < a.seqs && a.seq_off[1 + first] <= t1) return find_sequence(a.seq_off, first, a.seqs - first, t1);
    return first;
}

// Adds live tokens to a sequence; whoever finds it without any has found one more sequence that has some.
__device__ __forceinline__ void add_live(const PolicyArgs& a, int seq, int count, int& held) {
    if (count && seq < a.seqs) held += atomicAdd(a.seq_live + seq, count) == 0;
}
// live, held: what this warp found (held: sequences that nobody had found before).
template <int QUADS>
__device__ __forceinline__ void count_tokens(const PolicyArgs& a, int warp, int warps, int& live, int& held) {
    constexpr int kLong = kRun * QUADS;                       // tokens whose loads are in flight together
    const int lane = threadIdx.x & 31;
    const Piece p = warp_piece(a.tokens, kLong, warp, warps);
    live = held = 0;
    if (p.begin >= p.end) return;
    int pending = 0, first = -1, begin = 0;         // pending: live tokens of `first` that are not added yet
    for (int t0 = p.begin; t0 < p.end; t0 += kLong) {
        int target[QUADS][4];
#pragma unroll
        for (int q = 0; q < QUADS; ++q) load_quad(a.targets, t0 + q * kRun + lane * 4, a.tokens, a.vector, -1, target[q]);
        if (first < 0) {
            begin = a.seq_off[0];
            first = find_sequence(a.seq_off, 0, a.seqs, t0);
        }
        const int before = first, last = advance(a, first, t0, min(a.tokens, t0 + kLong) - 1);
        if (first != before) {
            pending = __reduce_add_sync(0xffffffffu, pending);
            if (lane == 0) {
                add_live(a, before, pending, held);
                live += before < a.seqs ? pending : 0;
            }
            pending = 0;
        }
        if (first == last && t0 >= begin) {                   // one sequence
#pragma unroll
            for (int q = 0; q < QUADS; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i) pending += target[q][i] >= 0;
            continue;
        }
        int count = 0, at = first, bound = at < a.seqs && first != last ? a.seq_off[1 + at] : INT32_MAX;
        auto add = [&]() {
            if (at == first) {
                pending += count;
            } else if (at < a.seqs) {
                add_live(a, at, count, held);
                live += count;
            }
            count = 0;
        };
#pragma unroll
        for (int q = 0; q < QUADS; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = t0 + q * kRun + lane * 4 + i;
                if (target[q][i] < 0 || t < begin) continue;
                if (t >= bound) {
                    add();
                    at = find_here(a.seq_off, at, last, t);
                    bound = at < a.seqs ? a.seq_off[1 + at] : INT32_MAX;
                }
                ++count;
            }
        add();
    }
    pending = __reduce_add_sync(0xffffffffu, pending);
    if (lane == 0) {
        add_live(a, first, pending, held);
        live += first < a.seqs ? pending : 0;
    }
    live = __reduce_add_sync(0xffffffffu, live);
    held = __reduce_add_sync(0xffffffffu, held);
}
// The block's counts into the totals: one addition each.
template <int WARPS>
__device__ __forceinline__ void add_totals(const PolicyArgs& a, int live, int held) {
    __shared__ int sums[2][WARPS];
    if ((threadIdx.x & 31) == 0) {
        sums[0][threadIdx.x >> 5] = live;
        sums[1][threadIdx.x >> 5] = held;
    }
    __syncthreads();
    if (threadIdx.x < 2) {
        int n = 0;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) n += sums[threadIdx.x][w];
        if (n) atomicAdd(a.totals + threadIdx.x, n);
    }
}

// exp(x) - 1 and exp(x) - 1 - x without cancellation: the series below 1/2, where the differences would lose two bits and more.
__device__ __forceinline__ float exp_series(float x) {
    float s = 1.f / 40320.f;
    s = fmaf(s, x, 1.f / 5040.f);
    s = fmaf(s, x, 1.f / 720.f);
    s = fmaf(s, x, 1.f / 120.f);
    s = fmaf(s, x, 1.f / 24.f);
    s = fmaf(s, x, 1.f / 6.f);
    s = fmaf(s, x, 0.5f);
    return s * x * x;
}
__device__ __forceinline__ void exp_differences(float x, float& em1, float& rest) {
    rest = exp_series(x);
    em1 = rest + x;
    if (!(fabsf(x) < 0.5f)) {
        em1 = expf(x) - 1.f;
        rest = em1 - x;
    }
}

// Sums of a lane's terms.
struct Terms {
    float term = 0.f, kl = 0.f, ratio = 0.f;
    int cut = 0;
};
// Adds a token's term and returns its derivative.  Tokens that are not live come with lp = old = ref and A = 0.
template <bool REF>
__device__ __forceinline__ float policy_term(const PolicyArgs& a, float log_low, float log_high, bool live, float lp, float old, float ref,
                                             float A, Terms& s) {
    const float x = lp - old;
    // 2^(x log2 e) with log2 e in two parts: what is left is the rounding of the product and of the function
    const float r = exp2f(fmaf(x, 1.44269502f, x * 1.92596299e-8f));
    const bool up = A > 0.f;
    const float border = up ? log_high : log_low;
    bool cut = up ? x > border : x < border;
    // next to a border the fp32 difference and border, each off by 2^-24 of itself, do not decide
    if (fabsf(x - border) <= 2.4e-7f * fabsf(x)) {
        const double exact = (double)lp - (double)old;
        cut = up ? exact > a.log_high : exact < a.log_low;
    }
    cut = cut && A != 0.f;
    float d = cut ? 0.f : -A * r, term = -A * (cut ? (up ? a.high : a.low) : r);
    if (REF) {
        float em1, kl;
        exp_differences(ref - lp, em1, kl);
        s.kl += kl;
        if (a.kl != 0.f) {
            term = fmaf(a.kl, kl, term);
            d = fmaf(-a.kl, em1, d);
        }
    }
    s.term += term;
    s.cut += cut;
    s.ratio += live ? r : 0.f;
    return d;
}

struct Inputs {
    int target[4];
    float lp[4], old[4], ref[4];
};
template <bool REF>
__device__ __forceinline__ Inputs load_inputs(const PolicyArgs& a, int t) {
    Inputs v;
    if (a.vector && t + 4 <= a.tokens) {
        const int4 g = *reinterpret_cast<const int4*>(a.targets + t);
        const float4 l = *reinterpret_cast<const float4*>(a.lp + t), o = *reinterpret_cast<const float4*>(a.old_lp + t);
        const float4 r = REF ? *reinterpret_cast<const float4*>(a.ref + t) : l;
        v.target[0] = g.x; v.target[1] = g.y; v.target[2] = g.z; v.target[3] = g.w;
        v.lp[0] = l.x; v.lp[1] = l.y; v.lp[2] = l.z; v.lp[3] = l.w;
        v.old[0] = o.x; v.old[1] = o.y; v.old[2] = o.z; v.old[3] = o.w;
        v.ref[0] = r.x; v.ref[1] = r.y; v.ref[2] = r.z; v.ref[3] = r.w;
    } else {
        load_quad(a.targets, t, a.tokens, 0, -1, v.target);
        load_quad(a.lp, t, a.tokens, 0, 0.f, v.lp);
        load_quad(a.old_lp, t, a.tokens, 0, 0.f, v.old);
        if (REF) load_quad(a.ref, t, a.tokens, 0, 0.f, v.ref);
    }
    return v;
}

// The same for four tokens of one sequence, where no ratio is next to a border and |ref - lp| < 1/2: false, and nothing changed, elsewhere.
template <bool REF>
__device__ __forceinline__ bool plain_terms(const PolicyArgs& a, float log_low, float log_high, const Inputs& v, float A, float share, Terms& sum,
                                            float (&d)[4]) {
    // over the border: side * x - edge > 0
    const float side = A > 0.f ? 1.f : -1.f, edge = A > 0.f ? log_high : A < 0.f ? -log_low : INFINITY, limit = A > 0.f ? a.high : a.low;
    const float near = fabsf(edge) < INFINITY ? 3e-7f * fabsf(edge) : 0.f;
    Terms s = sum;
    bool ok = true;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool on = v.target[i] >= 0;
        const float x = on ? v.lp[i] - v.old[i] : 0.f, B = on ? -A : 0.f;
        const float r = ex2(fmaf(x, 1.44269502f, x * 1.92596299e-8f)), over = fmaf(side, x, -edge);
        const bool cut = over > 0.f;
        ok = ok && !(fabsf(over) <= near && on);
        s.term = fmaf(B, cut ? limit : r, s.term);
        d[i] = cut ? 0.f : B * r;
        s.cut += cut;
        s.ratio += on ? r : 0.f;
        if (REF) {
            const float y = on ? v.ref[i] - v.lp[i] : 0.f, kl = exp_series(y);
            ok = ok && fabsf(y) < 0.5f;
            s.kl += kl;
            if (a.kl != 0.f) {
                s.term = fmaf(a.kl, kl, s.term);
                d[i] = fmaf(-a.kl, kl + y, d[i]);
            }
        }
        d[i] *= share;
    }
    if (ok) sum = s;
    return ok;
}

// Weight of a term of a sequence.
__device__ __forceinline__ double term_share(const PolicyArgs& a, int live, int held, int seq) {
    if (a.reduce == 0) return a.scale / max(1, live);
    if (a.reduce == 1) return seq < a.seqs ? a.scale / ((double)max(1, held) * max(1, __ldcg(a.seq_live + seq))) : 0.;
    return a.scale;
}

// Terms and derivatives of a warp's tokens; sums: loss, kl, cut ratios, ratios.
// SECOND: of the second kernel, which waits for the first one's counts.
template <bool REF, bool SECOND>
__device__ __forceinline__ void loss_tokens(const PolicyArgs& a, int warp, int warps, double (&sums)[4]) {
    const int lane = threadIdx.x & 31, begin = a.seq_off[0];
    const Piece p = warp_piece(a.tokens, kRun, warp, warps);
    if (p.begin >= p.end) {
        if (SECOND) pdl_wait();
        return;
    }
    Inputs v = load_inputs<REF>(a, p.begin + lane * 4);
    int live = 0, held = 0;
    auto counts = [&]() {
        live = __ldcg(a.totals);
        held = __ldcg(a.totals + 1);
    };
    if (!SECOND) counts();                                    // on their way during the search
    int first = find_sequence(a.seq_off, 0, a.seqs, p.begin), of = -1;      // of: the sequence of share and seq_adv
    if (SECOND) {
        pdl_wait();
        counts();
    }
    const float log_low = (float)a.log_low, log_high = (float)a.log_high;
    double share = 0.;
    float seq_adv = 0.f;
    for (int t0 = p.begin; t0 < p.end; t0 += kRun) {
        Inputs next = v;
        if (t0 + kRun < p.end) next = load_inputs<REF>(a, t0 + kRun + lane * 4);     // on its way while this run is worked on
        const int t = t0 + lane * 4, last = advance(a, first, t0, min(a.tokens, t0 + kRun) - 1);
        int at = first == last ? first : find_here(a.seq_off, first, last, t);
        int bound = at < a.seqs && first != last ? a.seq_off[1 + at] : INT32_MAX;
        auto enter = [&](int seq) {                           // share and advantage of the sequence
            if (seq != of) {
                share = term_share(a, live, held, seq);
                if (!a.per_token && seq < a.seqs) seq_adv = a.adv[seq];
                of = seq;
            }
        };
        enter(at);
        Terms sum;
        float adv[4], d[4];
        if (a.per_token) load_quad(a.adv, t, a.tokens, a.vector, 0.f, adv);
        if (first != last || t0 < begin || a.per_token || first >= a.seqs || !plain_terms<REF>(a, log_low, log_high, v, seq_adv, (float)share, sum, d))
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool counts = v.target[i] >= 0 && t + i >= begin;
            if (counts && t + i >= bound) {                   // the next sequence with a token here
                sums[0] += share * sum.term;
                sum.term = 0.f;
                at = find_here(a.seq_off, at, last, t + i);
                bound = at < a.seqs ? a.seq_off[1 + at] : INT32_MAX;
                enter(at);
            }
            const bool on = counts && at < a.seqs;
            const float A = a.per_token ? adv[i] : seq_adv;
            d[i] = policy_term<REF>(a, log_low, log_high, on, on ? v.lp[i] : 0.f, on ? v.old[i] : 0.f, on && REF ? v.ref[i] : 0.f, on ? A : 0.f, sum);
            d[i] *= on ? (float)share : 0.f;
        }
        sums[0] += share * sum.term;
        sums[1] += sum.kl;
        sums[2] += sum.cut;
        sums[3] += sum.ratio;
        if (a.d_lp) {
            if (a.vector && t + 4 <= a.tokens) {
                *reinterpret_cast<float4*>(a.d_lp + t) = make_float4(d[0], d[1], d[2], d[3]);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (t + i < a.tokens) a.d_lp[t + i] = d[i];
            }
        }
        v = next;
    }
}
// The block's sums, by the first four threads.
template <int WARPS>
__device__ __forceinline__ double block_sums(double (&sums)[4], double (&reduce)[WARPS][4]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int q = 0; q < 4; ++q) sums[q] = warp_sum_double(sums[q]);
    if (lane == 0)
        for (int q = 0; q < 4; ++q) reduce[warp][q] = sums[q];
    __syncthreads();
    double v = 0.;
    if (threadIdx.x < 4)
        for (int w = 0; w < WARPS; ++w) v += reduce[w][threadIdx.x];
    return v;
}
// What the call reports, and counters back at zero.
__device__ __forceinline__ void write_stats(const PolicyArgs& a, double v) {
    const int live = __ldcg(a.totals), held = __ldcg(a.totals + 1);
    if (threadIdx.x < 4) a.stats[threadIdx.x] = (float)(threadIdx.x == 0 ? v : live ? v / live : 0.);
    for (int s = threadIdx.x; s < a.seqs; s += blockDim.x) a.seq_live[s] = 0;
    __syncthreads();
    if (threadIdx.x == 0) {
        a.stats[4] = (float)live;
        a.stats[5] = (float)held;
        a.totals[0] = a.totals[1] = a.ticket[0] = 0;
    }
}

__global__ void __launch_bounds__(kThreads) policy_count_kernel(const PolicyArgs a) {
    asm volatile("griddepcontrol.launch_dependents;");        // all blocks have started: those of the second kernel come in as these end
    int live, held;
    count_tokens<4>(a, blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), gridDim.x * (kThreads / 32), live, held);
    add_totals<kThreads / 32>(a, live, held);
}

template <bool REF>
__global__ void __launch_bounds__(kThreads, 3) policy_loss_kernel(const PolicyArgs a) {
    __shared__ double reduce[kThreads / 32][4];
    __shared__ int last;
    double sums[4] = {0., 0., 0., 0.};
    loss_tokens<REF, true>(a, blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), gridDim.x * (kThreads / 32), sums);
    double v = block_sums<kThreads / 32>(sums, reduce);
    if (threadIdx.x < 4) {
        a.parts[(int64_t)blockIdx.x * 4 + threadIdx.x] = v;
        __threadfence();
    }
    __syncthreads();
    if (threadIdx.x == 0) last = atomicAdd(a.ticket, 1) == (int)gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    // thread = 4 x run of blocks + sum
    v = 0.;
#pragma unroll 8
    for (int b = threadIdx.x >> 2; b < (int)gridDim.x; b += kThreads / 4) v += __ldcg(a.parts + (int64_t)b * 4 + (threadIdx.x & 3));
#pragma unroll
    for (int o = 16; o >= 4; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if ((threadIdx.x & 31) < 4) reduce[threadIdx.x >> 5][threadIdx.x & 3] = v;
    __syncthreads();
    v = 0.;
    if (threadIdx.x < 4)
        for (int w = 0; w < kThreads / 32; ++w) v += reduce[w][threadIdx.x];
    write_stats(a, v);
}

// Short batches: one block counts, waits for its own counts and goes on.
template <bool REF>
__global__ void __launch_bounds__(kSmallThreads) policy_small_kernel(const PolicyArgs a) {
    __shared__ double reduce[kSmallThreads / 32][4];
    int live, held;
    count_tokens<1>(a, threadIdx.x >> 5, kSmallThreads / 32, live, held);
    add_totals<kSmallThreads / 32>(a, live, held);
    __threadfence();
    __syncthreads();
    double sums[4] = {0., 0., 0., 0.};
    loss_tokens<REF, false>(a, threadIdx.x >> 5, kSmallThreads / 32, sums);
    write_stats(a, block_sums<kSmallThreads / 32>(sums, reduce));
}

}  // namespace

cudaError_t init_policy_kernels() {
    return init_all(0, policy_count_kernel, policy_loss_kernel<false>, policy_loss_kernel<true>, policy_small_kernel<false>, policy_small_kernel<true>);
}

// Three blocks of 256 threads on every SM.
int policy_max_blocks(int sms) { return (sms < kTrainSms ? sms : kTrainSms) * 3; }

cudaError_t launch_policy_loss(const PolicyArgs& a, int sms, cudaStream_t st) {
    if (a.tokens <= kSmallTokens)
        return launch_plain(a.has_ref ? policy_small_kernel<true> : policy_small_kernel<false>, dim3(1), dim3(kSmallThreads), 0, st, a);
    const int64_t need = ((int64_t)a.tokens + kThreads / 32 * kRun - 1) / (kThreads / 32 * kRun), most = policy_max_blocks(sms);
    const int64_t counting = (need + 3) / 4 < (int64_t)sms * 6 ? (need + 3) / 4 : (int64_t)sms * 6;
    const dim3 grid((unsigned)(need < most ? need : most)), block(kThreads);
    const cudaError_t e = launch_plain(policy_count_kernel, dim3((unsigned)counting), block, 0, st, a);
    if (e != cudaSuccess) return e;
    return launch_second(a.has_ref ? policy_loss_kernel<true> : policy_loss_kernel<false>, grid, block, 0, st, a);
}

}  // namespace mars
