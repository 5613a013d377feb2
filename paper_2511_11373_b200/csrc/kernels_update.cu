// Contractions of the policy update on the 5th-generation tensor cores (tcgen05 + TMEM):
//   log-prob of known tokens      logits = h W^T, softmax statistics in the epilogue        (K-major x K-major)
//   its gradient, per piece       d = g/T ([v = t] - softmax) from the logits again          (K-major x K-major)
//                                 d_hidden += d W_piece                                      (K-major x MN-major)
//                                 d_lm_head_piece = d^T h                                    (MN-major x MN-major)
//   expert products               y_e = x_e w_e^T, dx_e = dy_e w_e, dw_e = dy_e^T x_e        (the same three forms)
// One persistent kernel template serves all of them.  A CTA walks 128 x 256 output tiles:
//   warp 0 (one lane)  TMA producer, 64 contraction indexes per stage, 128-byte swizzle, mbarrier ring that
//                      runs on across tiles;
//   warp 1             one lane issues tcgen05.mma (K 16) into one of two TMEM accumulators;
//   warps 2..5         epilogue of the previous tile (a thread owns a row of it) while the next is computed.
// A K-major operand is a [rows][k] matrix (boxes of 128 rows x 64 k), an MN-major one a [k][columns] matrix
// (boxes of 64 k x 64 columns), so no transposed copy of anything is made.  Ragged groups: rows of a tile
// behind the group's end are computed and not stored; in dw_e, where the rows are the contraction, the stage
// that holds the end has the rows behind it cleared in shared memory (they belong to the next expert and may
// hold anything, NaN included), in whole steps of 16 the rest is not issued at all.
// Every wait is bounded; one that gives up sets the status word, the CTA stops issuing, waits for its copies
// in flight, frees its TMEM and returns.
#include "common.cuh"
#include "kernels.h"
#include "update.h"

namespace mars {

namespace {

constexpr int kTileN = 256, kStageK = 64, kThreads = 192;
constexpr uint32_t kSpin = 1u << 22;
constexpr int kMnBox = 64 * kStageK * 2;                     // 8 KB: 64 contraction rows of 128 B

template <int CG>
struct Cfg {
    static constexpr int kTileM = 128 * CG;
    static constexpr int kBRows = kTileN / CG;               // B columns held by one CTA
    static constexpr int kABytes = 128 * kStageK * 2;
    static constexpr int kBBytes = kBRows * kStageK * 2;
    static constexpr int kStageBytes = kABytes + kBBytes;
    static constexpr int kStages = CG == 1 ? 4 : 6;          // 192 KB of ring
    static constexpr int kGroupWords = 2 * (kUpMaxExperts + 1);
    static constexpr size_t smem_bytes(bool groups) {
        return (size_t)kStages * kStageBytes + 1024 + (groups ? kGroupWords * 4 : 0);
    }
};

enum Sched { kDense, kGroupRows, kGroupK };
enum Epi { kStats, kDlogits, kStore };

__device__ __forceinline__ void mb_init(uint64_t* bar, int count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count));
}
__device__ __forceinline__ void mb_expect(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mb_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// Bounded wait: at most kSpin polls and about two seconds.  CLUSTER: acquires plain writes of the other CTA too
// (a copy's or an MMA's arrival needs no such scope).
template <bool CLUSTER = false>
__device__ __forceinline__ bool mb_wait(uint64_t* bar, uint32_t parity) {
    uint64_t begin = 0;
    for (uint32_t i = 0; i < kSpin; ++i) {
        uint32_t ok;
        if (CLUSTER)
            asm volatile(
                "{\n\t.reg .pred p;\n\t"
                "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
                "selp.u32 %0, 1, 0, p;\n\t}"
                : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
        else
            asm volatile(
                "{\n\t.reg .pred p;\n\t"
                "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
                "selp.u32 %0, 1, 0, p;\n\t}"
                : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
        if (ok) return true;
        if ((i & 1023) == 1023) {
            uint64_t t;
            asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
            if (!begin) begin = t;
            else if (t - begin > 2000000000ull) return false;
        }
    }
    return false;
}
// Address of the same shared-memory object in CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t in_cta(const void* p, uint32_t rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ void mb_arrive_at(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// One lane of a converged warp.  The loops around it stay warp-uniform, so that the compiler keeps stage
// counters, addresses and descriptors in uniform registers, which the copy and MMA instructions take: with the
// whole loop under `if (lane == 0)` an MMA cost its issuing lane about twice its time on the tensor cores.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// CG = 2: the barrier may be the other CTA's (`bar`: cluster address).
template <int CG>
__device__ __forceinline__ void tma_2d(uint32_t dst, const CUtensorMap* tm, int x, int y, uint32_t bar) {
    if (CG == 1)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"((uint64_t)tm), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"((uint64_t)tm), "r"(x), "r"(y), "r"(bar) : "memory");
}
template <int CG>
__device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap* tm, int x, int y, int z, uint32_t bar) {
    if (CG == 1)
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
            ::"r"(dst), "l"((uint64_t)tm), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
            ::"r"(dst), "l"((uint64_t)tm), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// Shared-memory matrix descriptor (version 1, 128-byte swizzle).  K-major: rows of 128 B, groups of 8 rows 1024 B
// apart (stride offset), the leading offset unused.  MN-major: a row of 128 B holds 64 consecutive columns of one
// contraction index, 8 indexes are 1024 B apart, the next 64 columns one box further (leading offset).
template <bool MN>
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr) {
    uint64_t d = (uint64_t)((addr >> 4) & 0x3fffu);
    d |= (uint64_t)(MN ? kMnBox >> 4 : 1) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}
template <bool MN> constexpr uint32_t kDescStep = MN ? 16 * 128 / 16 : 32 / 16;    // 16 contraction indexes, in 16 bytes

// fp32 accumulator, bf16 operands, bit 15 / 16: A / B is MN-major
template <int CG, bool A_MN, bool B_MN>
constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | ((A_MN ? 1u : 0u) << 15) | ((B_MN ? 1u : 0u) << 16) |
                            ((uint32_t)(kTileN >> 3) << 17) | ((uint32_t)(Cfg<CG>::kTileM >> 4) << 24);

template <int CG>
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate) {
    if (CG == 1)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
            ::"r"(d), "l"(da), "l"(db), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "setp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
            ::"r"(d), "l"(da), "l"(db), "r"(idesc), "r"(accumulate) : "memory");
}
// Arrives on the barrier (of both CTAs, at the same place, for a pair) once the MMAs issued so far are done.
template <int CG>
__device__ __forceinline__ void commit(uint64_t* bar) {
    if (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float (&v)[32]) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
}
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// One output tile and its contraction.
struct Tile {
    int a_row, b_col;         // first row / column in the operands' coordinates
    int m_valid, n_valid;     // rows / columns that exist
    int k0, k_len;            // contraction range
    int expert;               // third coordinate of the expert stack
    int col_tile;
    int64_t out;              // element offset of the tile's corner in the output
};

// The tiles of a call, numbered the same way in every role.  `off`, `first`: group bounds and the number of
// tiles before each group, in shared memory.
template <int CG, int SCHED>
struct TileMap {
    const UpParams& p;
    const int* off;
    const int* first;
    int m, k, tiles_m, tiles_n, count;

    __device__ __forceinline__ TileMap(const UpParams& q, const int* o, const int* f) : p(q), off(o), first(f) {
        constexpr int TM = Cfg<CG>::kTileM;
        tiles_n = (p.n + kTileN - 1) / kTileN;
        m = p.m; k = p.k;
        if (SCHED == kDense) {
            if (p.m_live) m = *p.m_live;
            if (p.k_live) k = *p.k_live;
            tiles_m = (m + TM - 1) / TM;
            count = tiles_m * tiles_n * p.splits;
        } else if (SCHED == kGroupRows) {
            tiles_m = 0;
            count = first[p.experts];
        } else {
            tiles_m = (m + TM - 1) / TM;
            count = p.experts * tiles_m * tiles_n;
        }
    }
    __device__ __forceinline__ Tile at(int t) const {
        constexpr int TM = Cfg<CG>::kTileM;
        Tile r;
        int tm;
        if (SCHED == kDense) {                       // rows fastest: neighbours share the columns' operand in L2
            const int per = tiles_m * tiles_n, split = t / per, u = t - split * per;
            r.col_tile = u / tiles_m;
            tm = u - r.col_tile * tiles_m;
            const int stages = (k + kStageK - 1) / kStageK;
            const int s0 = (int)((int64_t)stages * split / p.splits), s1 = (int)((int64_t)stages * (split + 1) / p.splits);
            r.k0 = s0 * kStageK;
            r.k_len = min(k, s1 * kStageK) - r.k0;
            r.expert = 0;
            r.a_row = tm * TM;
            r.m_valid = m - r.a_row;
            r.out = (int64_t)split * p.e.split_stride + (int64_t)r.a_row * p.e.ld;
        } else if (SCHED == kGroupRows) {
            int lo = 0, hi = p.experts - 1;          // the last group whose first tile is <= t and that has tiles
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (first[mid] <= t) lo = mid; else hi = mid - 1;
            }
            const int rows = off[lo + 1] - off[lo], per = (rows + TM - 1) / TM, u = t - first[lo];
            r.col_tile = u / per;
            tm = u - r.col_tile * per;
            r.k0 = 0; r.k_len = k; r.expert = lo;
            r.a_row = off[lo] + tm * TM;
            r.m_valid = rows - tm * TM;
            r.out = (int64_t)r.a_row * p.e.ld;
        } else {
            const int per = tiles_m * tiles_n, e = t / per, u = t - e * per;
            r.col_tile = u / tiles_m;
            tm = u - r.col_tile * tiles_m;
            r.expert = e;
            r.k0 = off[e];
            r.k_len = off[e + 1] - off[e];
            r.a_row = tm * TM;
            r.m_valid = m - r.a_row;
            r.out = ((int64_t)e * m + r.a_row) * p.e.ld;
        }
        r.b_col = r.col_tile * kTileN;
        r.n_valid = min(kTileN, p.n - r.b_col);
        r.out += r.b_col;
        return r;
    }
};

// Group bounds in shared memory: clamped to [0, rows] and made non-decreasing, so that no offset array leads
// outside the operands; first[e] = tiles of the groups before e.  One warp.
template <int TM>
__device__ __forceinline__ void load_groups(const UpParams& p, int* off, int* first, int tiles_n, int lane) {
    const int E = p.experts, per = (E + 1 + 31) / 32, b = min(lane * per, E + 1), e = min(b + per, E + 1);
    int top = 0;
    for (int i = b; i < e; ++i) {
        top = max(top, min(max(p.expert_off[i], 0), p.rows));
        off[i] = top;
    }
    int run = top;                                    // running maximum over the lanes before
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run = max(run, v);
    }
    int before = __shfl_up_sync(0xffffffffu, run, 1);
    if (lane == 0) before = 0;
    for (int i = b; i < e; ++i) off[i] = max(off[i], before);
    __syncwarp();
    int sum = 0;
    for (int i = b; i < min(e, E); ++i) sum += (off[i + 1] - off[i] + TM - 1) / TM * tiles_n;
    int pre = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, pre, o);
        if (lane >= o) pre += v;
    }
    pre -= sum;
    for (int i = b; i < e; ++i) {
        first[i] = pre;
        if (i < E) pre += (off[i + 1] - off[i] + TM - 1) / TM * tiles_n;
    }
    __syncwarp();
}

// ---------------------------------------------------------------------------------------- epilogues
// `taddr`: this thread's lane of the accumulator, column 0.  row: row of the tile.

// Store the tile: bf16 (rounded once from the fp32 accumulator) or fp32, optionally on top of what is there.
__device__ __forceinline__ void store_tile(const UpEpilogue& e, const Tile& t, int row, uint32_t taddr, bool zero) {
    const bool live = row < t.m_valid;
#pragma unroll 1
    for (int c = 0; c < t.n_valid; c += 32) {
        float v[32];
        if (zero) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = 0.f;
        } else {
            tmem_ld32(taddr + c, v);
        }
        if (!live) continue;
        const int64_t at = t.out + (int64_t)row * e.ld + c;
        if (e.out_f32) {
            float* dst = reinterpret_cast<float*>(e.out) + at;
#pragma unroll
            for (int j = 0; j < 32; j += 4)
                if (c + j < t.n_valid) {
                    float4 w = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                    if (e.accumulate) {
                        const float4 o = *reinterpret_cast<const float4*>(dst + j);
                        w.x += o.x; w.y += o.y; w.z += o.z; w.w += o.w;
                    }
                    *reinterpret_cast<float4*>(dst + j) = w;
                }
        } else {
            __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(e.out) + at;
#pragma unroll
            for (int j = 0; j < 32; j += 8)
                if (c + j < t.n_valid) {
                    if (e.accumulate) {
                        const uint4 o = *reinterpret_cast<const uint4*>(dst + j);
                        const uint32_t ow[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                        for (int q = 0; q < 4; ++q) { v[j + 2 * q] += bf16_lo(ow[q]); v[j + 2 * q + 1] += bf16_hi(ow[q]); }
                    }
                    *reinterpret_cast<uint4*>(dst + j) =
                        make_uint4(pack_bf16(v[j], v[j + 1]), pack_bf16(v[j + 2], v[j + 3]), pack_bf16(v[j + 4], v[j + 5]),
                                   pack_bf16(v[j + 6], v[j + 7]));
                }
        }
    }
}

// Softmax statistics of the tile's columns: the largest logit M (before the temperature) and
// sum exp((logit - M) / T), one pass with a running maximum; differences are taken before the scaling, so the
// exponents carry no rounding of large values.  The row's own target logit is stored on the way.
__device__ __forceinline__ void stats_tile(const UpEpilogue& e, const Tile& t, int row, uint32_t taddr, int tiles_n) {
    const bool live = row < t.m_valid;
    const int r = t.a_row + row;
    const int tgt = live ? e.target[r] - t.b_col : -1;        // column of the target, if it is in this tile
    const float scale = e.inv_temp * 1.4426950408889634f;
    float mx = -INFINITY, sum = 0.f, zt = 0.f;
#pragma unroll 1
    for (int c = 0; c < t.n_valid; c += 32) {
        float v[32];
        tmem_ld32(taddr + c, v);
        if (!live) continue;
        const int left = t.n_valid - c;
        float nm = mx;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            if (j >= left) v[j] = -INFINITY;
            nm = fmaxf(nm, v[j]);
        }
        const float ref = nm == -INFINITY ? 0.f : nm;          // nothing but -inf so far: all terms are 0
        float add = 0.f;
#pragma unroll
        for (int j = 0; j < 32; ++j) add += exp2_approx((v[j] - ref) * scale);
        sum = sum * exp2_approx((mx - ref) * scale) + add;
        mx = nm;
        if (tgt >= c && tgt < c + 32) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (c + j == tgt) zt = v[j];
        }
    }
    if (!live) return;
    e.stats[(int64_t)r * tiles_n + t.col_tile] = make_float2(mx, sum);
    if (tgt >= 0 && tgt < t.n_valid) e.target_logit[r] = zt;
}

// Gradient of the logits: d = w ([v = t] - p), p = exp(z - lse), w = g / T, rounded once to bf16 (relative
// 2^-8 at most, independent from entry to entry) because it is an operand of two tensor-core products.
// The target's own 1 - p is -expm1(z - lse): no cancellation where p is close to 1.  Rows and columns behind
// the end are written as zeros: they are contraction indexes of those products.
__device__ __forceinline__ void dlogits_tile(const UpEpilogue& e, const Tile& t, int row, uint32_t taddr) {
    const bool live = row < t.m_valid;
    const int r = t.a_row + row;
    const int tgt = live ? e.target[r] - e.v0 - t.b_col : -1;
    const float w = live ? e.weight[r] : 0.f, lse = live ? e.lse[r] : 0.f;
    const float scale = e.inv_temp * 1.4426950408889634f, shift = -lse * 1.4426950408889634f;
    const int left0 = e.vocab - e.v0 - t.b_col;
    __nv_bfloat16* dst = e.dlogits + (int64_t)r * e.ld + t.b_col;
#pragma unroll 1
    for (int c = 0; c < t.n_valid; c += 32) {
        float v[32];
        tmem_ld32(taddr + c, v);
        const int left = left0 - c;
        const bool own = tgt >= c && tgt < c + 32;
        float dt = 0.f;
        if (own) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (c + j == tgt) dt = v[j];
            dt = -w * expm1f(fmaf(dt, e.inv_temp, -lse));
        }
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const float d = -w * exp2_approx(fmaf(v[j], scale, shift));
            v[j] = live && j < left ? (own && c + j == tgt ? dt : d) : 0.f;
        }
#pragma unroll
        for (int j = 0; j < 32; j += 8)
            *reinterpret_cast<uint4*>(dst + c + j) =
                make_uint4(pack_bf16(v[j], v[j + 1]), pack_bf16(v[j + 2], v[j + 3]), pack_bf16(v[j + 4], v[j + 5]),
                           pack_bf16(v[j + 6], v[j + 7]));
    }
}

template <int CG, bool A_MN, bool B_MN, int SCHED, int EPI>
__global__ void __launch_bounds__(kThreads, 1)
contract_kernel(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b,
                const __grid_constant__ UpParams p) {
    using C = Cfg<CG>;
    extern __shared__ unsigned char up_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>(((uintptr_t)up_raw + 1023) & ~(uintptr_t)1023);
    int* off = reinterpret_cast<int*>(smem + C::kStages * C::kStageBytes);
    int* first = off + kUpMaxExperts + 1;
    __shared__ __align__(8) uint64_t full[C::kStages], empty[C::kStages], tail[C::kStages], acc_full[2], acc_empty[2];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int dead;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int rank = CG == 2 ? (int)(blockIdx.x & 1) : 0;      // place in the pair; rank 0 leads
    const int worker = blockIdx.x / CG, workers = gridDim.x / CG;
    // a stage of kGroupK is full after two arrivals: the leader's own two, or one of each CTA that cleared rows
    constexpr int kFullCount = SCHED == kGroupK ? 2 : 1;

    if (tid == 0) {
        for (int i = 0; i < C::kStages; ++i) { mb_init(&full[i], kFullCount); mb_init(&empty[i], 1); mb_init(&tail[i], 1); }
        for (int i = 0; i < 2; ++i) { mb_init(&acc_full[i], 1); mb_init(&acc_empty[i], 4 * CG); }
        dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 2) {
        if (CG == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(2 * kTileN));
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(2 * kTileN));
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    pdl_wait();
    if (SCHED != kDense && warp == 3) load_groups<C::kTileM>(p, off, first, (p.n + kTileN - 1) / kTileN, lane);
    __syncwarp();
    if (CG == 2) cluster_sync(); else __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_d = tmem_slot;
    const TileMap<CG, SCHED> map(p, off, first);
    const uint32_t ring = smem_u32(smem);

    if (warp == 0) {
        const bool elected = elect_one();
        uint32_t it = 0;
        int s = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int tile = worker; ok && tile < map.count; tile += workers) {
            const Tile t = map.at(tile);
            const int nk = (t.k_len + kStageK - 1) / kStageK;
            const int a_row = t.a_row + rank * 128, b_col = t.b_col + rank * C::kBRows;
            for (int ks = 0; ks < nk; ++ks) {
                ok = !dead && mb_wait(&empty[s], phase ^ 1);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const uint32_t sa = ring + (uint32_t)s * C::kStageBytes, sb = sa + C::kABytes;
                const int k = t.k0 + ks * kStageK;
                const bool ragged = SCHED == kGroupK && (t.k_len - ks * kStageK) < kStageK && t.k_len % 16;
                // a ragged stage is reported by warp 1 once it has cleared rows, any other by the copies to the leader
                const uint32_t bar = ragged ? (CG == 2 ? in_cta(&tail[s], rank) : smem_u32(&tail[s]))
                                            : (CG == 2 ? in_cta(&full[s], 0) : smem_u32(&full[s]));
                if (elected) {
                    if (ragged) {
                        mb_expect(&tail[s], C::kStageBytes);
                    } else if (rank == 0) {
                        if (kFullCount == 2) mb_arrive(&full[s]);
                        mb_expect(&full[s], CG * C::kStageBytes);
                    }
                    if (A_MN) {
#pragma unroll
                        for (int b = 0; b < 2; ++b) tma_2d<CG>(sa + b * kMnBox, &tm_a, a_row + b * 64, k, bar);
                    } else {
                        tma_2d<CG>(sa, &tm_a, k, a_row, bar);
                    }
                    if (B_MN) {
#pragma unroll
                        for (int b = 0; b < C::kBRows / 64; ++b) {
                            if (SCHED == kGroupRows) tma_3d<CG>(sb + b * kMnBox, &tm_b, b_col + b * 64, k, t.expert, bar);
                            else tma_2d<CG>(sb + b * kMnBox, &tm_b, b_col + b * 64, k, bar);
                        }
                    } else {
#pragma unroll
                        for (int b = 0; b < C::kBRows / 128; ++b) {
                            if (SCHED == kGroupRows) tma_3d<CG>(sb + b * 16384, &tm_b, k, b_col + b * 128, t.expert, bar);
                            else tma_2d<CG>(sb + b * 16384, &tm_b, k, b_col + b * 128, bar);
                        }
                    }
                }
                __syncwarp();
                ++it;
                if (++s == C::kStages) { s = 0; phase ^= 1; }
            }
        }
        // Copies in flight must land before the shared memory is given up: the stages' release says so in the
        // regular case (the last accumulator is waited for); after a wait that gave up they are waited for here.
        if (!ok && lane == 0) {
            dead = 1;
            atomicOr(p.err, kErrTimeout);
            if (rank == 0)
                for (uint32_t w = it > C::kStages ? it - C::kStages : 0; w < it; ++w) mb_wait(&full[w % C::kStages], (w / C::kStages) & 1);
        }
    } else if (warp == 1) {
        // the leader's warp issues the MMAs; for kGroupK the other CTA's walks along to clear rows of its own half
        if (SCHED == kGroupK || rank == 0) {
            const bool elected = elect_one();
            uint32_t tails = 0;                               // parity of every stage's tail barrier
            int s = 0, local = 0;
            uint32_t phase = 0;
            bool ok = true;
            const uint64_t desc_a = smem_desc<A_MN>(ring), desc_b = smem_desc<B_MN>(ring + C::kABytes);
            for (int tile = worker; ok && tile < map.count; tile += workers) {
                const Tile t = map.at(tile);
                const int nk = (t.k_len + kStageK - 1) / kStageK;
                if (nk <= 0) continue;                        // nothing to contract: the epilogue writes zeros
                const int buf = local & 1;
                if (rank == 0) {
                    ok = !dead && mb_wait<CG == 2>(&acc_empty[buf], ((local >> 1) & 1) ^ 1);
                    ok = __all_sync(0xffffffffu, ok);
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                }
                const uint32_t acc = tmem_d + (uint32_t)(buf * kTileN);
                for (int ks = 0; ok && ks < nk; ++ks) {
                    const int left = t.k_len - ks * kStageK;
                    const int steps = left >= kStageK ? 4 : (left + 15) / 16;
                    if (SCHED == kGroupK && left < kStageK && left % 16) {
                        ok = !dead && mb_wait(&tail[s], (tails >> s) & 1);
                        ok = __all_sync(0xffffffffu, ok);
                        if (!ok) break;
                        tails ^= 1u << s;
                        constexpr int kBoxes = (C::kABytes + C::kBBytes) / kMnBox;
                        unsigned char* st = smem + (size_t)s * C::kStageBytes;
                        const int n_rows = steps * 16 - left;     // rows behind the group's end, up to the step's 16
                        for (int i = lane; i < n_rows * kBoxes * 8; i += 32) {
                            const int piece = i & 7, row = left + (i >> 3) % n_rows, box = (i >> 3) / n_rows;
                            *reinterpret_cast<uint4*>(st + (size_t)box * kMnBox + row * 128 + piece * 16) = make_uint4(0, 0, 0, 0);
                        }
                        asm volatile("fence.proxy.async;" ::: "memory");
                        __syncwarp();
                        if (elected) {
                            if (CG == 1) { mb_arrive(&full[s]); mb_arrive(&full[s]); }
                            else mb_arrive_at(in_cta(&full[s], 0));
                        }
                        __syncwarp();
                    }
                    if (rank == 0) {
                        ok = !dead && mb_wait<CG == 2 && SCHED == kGroupK>(&full[s], phase);
                        ok = __all_sync(0xffffffffu, ok);
                        if (!ok) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint64_t da = desc_a + (uint64_t)(s * (C::kStageBytes >> 4)), db = desc_b + (uint64_t)(s * (C::kStageBytes >> 4));
                        if (elected) {
                            if (steps == 4) {
#pragma unroll
                                for (int kk = 0; kk < 4; ++kk)
                                    mma_f16<CG>(acc, da + kDescStep<A_MN> * kk, db + kDescStep<B_MN> * kk, kIdesc<CG, A_MN, B_MN>, kk == 0 ? ks != 0 : 1u);
                            } else {
                                for (int kk = 0; kk < steps; ++kk)
                                    mma_f16<CG>(acc, da + kDescStep<A_MN> * kk, db + kDescStep<B_MN> * kk, kIdesc<CG, A_MN, B_MN>, (ks | kk) != 0);
                            }
                            commit<CG>(&empty[s]);
                            if (ks == nk - 1) commit<CG>(&acc_full[buf]);
                        }
                        __syncwarp();
                    }
                    if (++s == C::kStages) { s = 0; phase ^= 1; }
                }
                ++local;
            }
            if (!ok && lane == 0) { dead = 1; atomicOr(p.err, kErrTimeout); }
        }
    } else {
        const int quarter = warp & 3, row = quarter * 32 + lane;
        int local = 0;
        for (int tile = worker; tile < map.count; tile += workers) {
            Tile t = map.at(tile);
            if (CG == 2) { t.a_row += rank * 128; t.m_valid -= rank * 128; t.out += (int64_t)rank * 128 * p.e.ld; }
            if (t.k_len <= 0) {
                if (EPI == kStore && !p.e.accumulate) store_tile(p.e, t, row, 0, true);
                continue;
            }
            const int buf = local & 1;
            if (lane == 0 && !dead && !mb_wait(&acc_full[buf], (local >> 1) & 1)) { dead = 1; atomicOr(p.err, kErrTimeout); }
            __syncwarp();
            if (!__all_sync(0xffffffffu, !dead)) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t taddr = tmem_d + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(buf * kTileN);
            if (EPI == kStats) stats_tile(p.e, t, row, taddr, map.tiles_n);
            else if (EPI == kDlogits) dlogits_tile(p.e, t, row, taddr);
            else store_tile(p.e, t, row, taddr, false);
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                if (CG == 1) mb_arrive(&acc_empty[buf]);
                else mb_arrive_at(in_cta(&acc_empty[buf], 0));
            }
            ++local;
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    // neither CTA of a pair leaves while the other may still signal its barriers or read its operands
    __syncwarp();
    if (CG == 2) cluster_sync(); else __syncthreads();
    if (warp == 2) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (CG == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_d), "r"(2 * kTileN));
        else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_d), "r"(2 * kTileN));
    }
}

constexpr int kCG = 2;

template <bool A_MN, bool B_MN, int SCHED, int EPI>
cudaError_t launch(const CUtensorMap& a, const CUtensorMap& b, const UpParams& p, int64_t tiles, int sms, cudaStream_t st) {
    const int64_t want = tiles < 1 ? 1 : tiles;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(want < sms / kCG ? want : sms / kCG) * kCG);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Cfg<kCG>::smem_bytes(SCHED != kDense);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kCG;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, contract_kernel<kCG, A_MN, B_MN, SCHED, EPI>, a, b, p);
}
template <bool A_MN, bool B_MN, int SCHED, int EPI>
cudaError_t init_one() {
    return cudaFuncSetAttribute(contract_kernel<kCG, A_MN, B_MN, SCHED, EPI>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                (int)Cfg<kCG>::smem_bytes(SCHED != kDense));
}
int64_t tiles_of(int64_t m, int64_t n) {
    return ((m + Cfg<kCG>::kTileM - 1) / Cfg<kCG>::kTileM) * ((n + kTileN - 1) / kTileN);
}
}  // namespace

cudaError_t init_update_kernels() {
    cudaError_t e = init_one<false, false, kDense, kStats>();
    if (e == cudaSuccess) e = init_one<false, false, kDense, kDlogits>();
    if (e == cudaSuccess) e = init_one<false, true, kDense, kStore>();
    if (e == cudaSuccess) e = init_one<true, true, kDense, kStore>();
    if (e == cudaSuccess) e = init_one<false, false, kGroupRows, kStore>();
    if (e == cudaSuccess) e = init_one<false, true, kGroupRows, kStore>();
    if (e == cudaSuccess) e = init_one<true, true, kGroupK, kStore>();
    return e;
}

cudaError_t launch_logit_stats(const CUtensorMap& h, const CUtensorMap& w, const UpParams& p, int sms, cudaStream_t st) {
    return launch<false, false, kDense, kStats>(h, w, p, tiles_of(p.m, p.n), sms, st);
}
cudaError_t launch_dlogits(const CUtensorMap& h, const CUtensorMap& w, const UpParams& p, int sms, cudaStream_t st) {
    return launch<false, false, kDense, kDlogits>(h, w, p, tiles_of(p.m, p.n), sms, st);
}
cudaError_t launch_dhidden(const CUtensorMap& d, const CUtensorMap& w, const UpParams& p, int sms, cudaStream_t st) {
    return launch<false, true, kDense, kStore>(d, w, p, tiles_of(p.m, p.n) * p.splits, sms, st);
}
cudaError_t launch_dhead(const CUtensorMap& d, const CUtensorMap& h, const UpParams& p, int sms, cudaStream_t st) {
    return launch<true, true, kDense, kStore>(d, h, p, tiles_of(p.m, p.n), sms, st);
}
cudaError_t launch_expert_fwd(const CUtensorMap& x, const CUtensorMap& w, const UpParams& p, int sms, cudaStream_t st) {
    return launch<false, false, kGroupRows, kStore>(x, w, p, sms, sms, st);
}
cudaError_t launch_expert_dx(const CUtensorMap& dy, const CUtensorMap& w, const UpParams& p, int sms, cudaStream_t st) {
    return launch<false, true, kGroupRows, kStore>(dy, w, p, sms, sms, st);
}
cudaError_t launch_expert_dw(const CUtensorMap& dy, const CUtensorMap& x, const UpParams& p, int sms, cudaStream_t st) {
    return launch<true, true, kGroupK, kStore>(dy, x, p, tiles_of(p.m, p.n) * p.experts, sms, st);
}

// Parts of the d_hidden contraction (over the vocabulary piece, `stages` stages of 64): few rows give few output
// tiles, and a piece is long, so it is cut until the tiles fill the SMs' rounds; at least 8 stages remain.
int dhidden_splits(int rows, int hidden, int stages, int sms) {
    const int64_t tiles = tiles_of(rows, hidden), slots = sms / kCG;
    int best = 1;
    double best_fill = 0.;
    for (int s = 1; s <= 16 && (s == 1 || stages / s >= 8); ++s) {
        const int64_t units = tiles * s, rounds = (units + slots - 1) / slots;
        const double fill = (double)units / (double)(rounds * slots) - 0.01 * s;     // a part more costs its output's traffic
        if (fill > best_fill) { best_fill = fill; best = s; }
    }
    return best;
}

// --------------------------------------------------------------------------------- live rows and ends

constexpr int kLiveRowsPerBlock = 8, kLiveThreads = 256;

// Copies the live rows side by side.  Every block counts the live rows before its own range (targets and
// weights are a few bytes per row and sit in L2), so one launch does the whole compaction, in order.
__global__ void __launch_bounds__(kLiveThreads) live_rows_kernel(LiveRows a) {
    __shared__ int counts[kLiveThreads / 32];
    __shared__ int place[kLiveRowsPerBlock];
    pdl_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int row0 = blockIdx.x * kLiveRowsPerBlock, end = min(row0 + kLiveRowsPerBlock, a.n);
    auto live = [&](int i) {
        const int t = a.targets[i];
        return t >= 0 && t < a.vocab && (!a.weight || a.weight[i] != 0.f);
    };
    int c = 0;
    for (int i = tid; i < row0; i += kLiveThreads) c += live(i);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
    if (lane == 0) counts[warp] = c;
    __syncthreads();
    if (tid == 0) {
        int at = 0;
        for (int i = 0; i < kLiveThreads / 32; ++i) at += counts[i];
        for (int i = row0; i < end; ++i) place[i - row0] = live(i) ? at++ : -1;
        counts[0] = at;
        if (blockIdx.x == gridDim.x - 1) *a.n_live = at;
    }
    __syncthreads();
    for (int i = row0 + warp; i < end; i += kLiveThreads / 32) {      // a warp copies a row
        const int to = place[i - row0];
        if (to < 0) {
            if (lane == 0) {
                if (a.logp_out) { a.logp_out[i] = 0.f; a.lse_out[i] = 0.f; }
                if (a.targets[i] >= a.vocab) atomicOr(a.err, kErrBadToken);
            }
            if (a.d_hidden)
                for (int j = lane; j < a.H / 8; j += 32)
                    reinterpret_cast<uint4*>(a.d_hidden + (int64_t)i * a.ld_d)[j] = make_uint4(0, 0, 0, 0);
            continue;
        }
        const uint4* src = reinterpret_cast<const uint4*>(a.hidden + (int64_t)i * a.ld);
        uint4* dst = reinterpret_cast<uint4*>(a.rows + (int64_t)to * a.H);
        for (int j = lane; j < a.H / 8; j += 32) dst[j] = src[j];
        if (lane == 0) {
            a.src[to] = i;
            a.target[to] = a.targets[i];
            if (a.weight) { a.scaled[to] = a.weight[i] * a.inv_temp; a.lse[to] = a.lse_in[i]; }
        }
    }
    if (blockIdx.x == gridDim.x - 1) {       // zero rows up to the tile: contraction indexes of d_lm_head
        const int total = counts[0], pad = (total + kUpTile - 1) / kUpTile * kUpTile;
        const int64_t n = (int64_t)(pad - total) * (a.H / 8);
        uint4* dst = reinterpret_cast<uint4*>(a.rows + (int64_t)total * a.H);
        for (int64_t j = tid; j < n; j += kLiveThreads) dst[j] = make_uint4(0, 0, 0, 0);
    }
}

cudaError_t launch_live_rows(const LiveRows& r, cudaStream_t st) {
    const int blocks = (r.n + kLiveRowsPerBlock - 1) / kLiveRowsPerBlock;
    return launch_chained(live_rows_kernel, dim3(blocks < 1 ? 1 : blocks), dim3(kLiveThreads), 0, st, r);
}

// One warp joins the column tiles' (largest logit, sum) of a row: lse = M / T + log sum, logp = (z_t - M) / T - log sum.
__global__ void __launch_bounds__(256) logprob_finish_kernel(const float2* stats, int tiles, int tiles_ld, const float* zt,
                                                             const int32_t* src, const int32_t* n_live, float inv_temp,
                                                             float* logp, float* lse) {
    pdl_wait();
    const int r = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (r >= *n_live) return;
    const float2* row = stats + (int64_t)r * tiles_ld;
    const float scale = inv_temp * 1.4426950408889634f;
    float mx = -INFINITY;
    for (int i = lane; i < tiles; i += 32) mx = fmaxf(mx, row[i].x);
    mx = warp_max(mx);
    float sum = 0.f;
    for (int i = lane; i < tiles; i += 32) {
        const float2 v = row[i];
        sum += v.y * exp2_approx((v.x - mx) * scale);
    }
    sum = warp_sum(sum);
    if (lane == 0) {
        const float l = logf(sum);
        lse[src[r]] = fmaf(mx, inv_temp, l);
        logp[src[r]] = (zt[r] - mx) * inv_temp - l;
    }
}

cudaError_t launch_logprob_finish(const float2* stats, int tiles, int tiles_ld, const float* target_logit, const int32_t* src,
                                  const int32_t* n_live, int n, float inv_temp, float* logp, float* lse, cudaStream_t st) {
    return launch_chained(logprob_finish_kernel, dim3((n + 7) / 8), dim3(256), 0, st, stats, tiles, tiles_ld, target_logit, src,
                          n_live, inv_temp, logp, lse);
}

// d_hidden of the live rows: the splits' fp32 parts added in order, rounded once, scattered to the original rows.
__global__ void __launch_bounds__(256) dhidden_finish_kernel(const float* parts, int splits, int64_t split_stride,
                                                             const int32_t* src, const int32_t* n_live, int H,
                                                             __nv_bfloat16* out, int64_t ld) {
    pdl_wait();
    const int r = blockIdx.x;
    if (r >= *n_live) return;
    const float* p = parts + (int64_t)r * H;
    __nv_bfloat16* dst = out + (int64_t)src[r] * ld;
    for (int j = threadIdx.x * 4; j < H; j += 1024) {
        float4 v = *reinterpret_cast<const float4*>(p + j);
        for (int s = 1; s < splits; ++s) {
            const float4 w = *reinterpret_cast<const float4*>(p + s * split_stride + j);
            v.x += w.x; v.y += w.y; v.z += w.z; v.w += w.w;
        }
        *reinterpret_cast<uint2*>(dst + j) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
    }
}

cudaError_t launch_dhidden_finish(const float* parts, int splits, int64_t split_stride, const int32_t* src,
                                  const int32_t* n_live, int n, int H, __nv_bfloat16* d_hidden, int64_t ld, cudaStream_t st) {
    return launch_chained(dhidden_finish_kernel, dim3(n), dim3(256), 0, st, parts, splits, split_stride, src, n_live, H,
                          d_hidden, ld);
}

}  // namespace mars
