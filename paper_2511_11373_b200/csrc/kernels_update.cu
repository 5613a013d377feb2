// Contractions of the policy update on the 5th-generation tensor cores (tcgen05 + TMEM), all of the form
// sum_k A(m, k) B(n, k), M being the TMEM lanes:
//   log-prob of known tokens    logits: A = lm_head (M vocabulary), B = hidden rows; softmax statistics in the epilogue
//   its gradient, per piece     d = g/T ([v = t] - softmax): the same contraction again, d stored as bf16
//                               d_hidden += W_piece^T d: A = lm_head (M hidden, MN-major), B = d
//                               d_lm_head_piece = d^T h: A = d (M vocabulary, MN-major), B = hidden rows (MN-major)
//   expert products             y: A = w_e, B = x;   dx: A = w_e (MN-major), B = dy;   dw_e: A = dy, B = x (both MN-major)
// One persistent kernel template serves all of them.  A pair of CTAs (cta_group::2) works on one tile of 256 x
// up to 256: each CTA holds 128 rows of A and half of B's rows, its tensor core reads the other half from its
// peer, so a 64-deep stage brings 32 KB into each SM where single-CTA 128 x 256 tiles bring 48 (those ran at the
// 11.5 TB/s that the L2 delivers: 758 us against 665 us for 131072 expert rows x 2048 -> 1536, bursts on equal groups).
// The N width of a tile is a multiple of 32 chosen from the rows there are (see cut): tokens sit on N, so ragged
// groups and short calls cost what they hold (a group of 4 rows a 32-wide tile, 270 rows one of 160 and one of 128),
// and a call of few rows is a plain stream of the weights.
//   warp 0      TMA producer, 64 contraction indexes per stage, 128-byte swizzle, mbarrier ring of 4 to 12
//               stages that runs on across tiles;
//   warp 1      of the leading CTA: issues tcgen05.mma (M 256, K 16) into one of two TMEM accumulators;
//   warps 2..9  epilogue of the previous tile (a thread owns one M index, half of the columns) meanwhile;
//   warp 10     dw_e: clears rows of ragged stages (below).
// A K-major operand is a [rows][k] matrix, an MN-major one a [k][columns] matrix (boxes of 64 k x 64 columns),
// so no transposed copy of anything is made.  Ragged groups: N rows of a tile behind the group's end are
// computed and not stored; in dw_e, where the rows are the contraction, the stage that holds the end has the
// rows behind it cleared in shared memory (they belong to the next expert and may hold anything, NaN included).
// Long contractions are cut into parts that are added in fp32 (kPartStages).
// Every wait is bounded; one that gives up sets the status word, the CTA stops issuing, waits for its copies
// in flight, frees its TMEM and returns.
#include <algorithm>

#include "common.cuh"
#include "kernels.h"
#include "update.h"

namespace mars {

namespace {

enum Sched { kDense, kGroupRows, kGroupK };
enum Epi { kStats, kDlogits, kStore, kStoreRows };      // kStore: out[n][m], kStoreRows: out[m][n]

constexpr int kTileM = 256, kTileN = 256, kStageK = 64;
constexpr int kEpiWarps = 8, kThreads = 64 + 32 * kEpiWarps + 32;
constexpr uint32_t kSpin = 1u << 22;
constexpr int kMnBox = 64 * kStageK * 2;                     // 8 KB: 64 contraction rows of 128 B
constexpr int kABytes = 128 * kStageK * 2;                   // one CTA's half of a tile's A rows
constexpr int kBBytes = 128 * kStageK * 2;                   // one CTA's half of the widest tile's B rows
// 192 KB of ring, 160 KB where a 4 KB stage for each epilogue warp stands beside it: 6 or 5 stages of full width (3: 10 %
// slower).  For log-prob rows a stage has as much room for B as the call's tiles take: 10 stages for a few rows (64 scored
// rows 120 -> 117 us), 4 for pairs of full tiles.  Expert groups keep full stages (one token: 20.2 us, 20.8 with 10).
template <int EPI> constexpr int kRingBytes = (EPI == kStoreRows ? 5 : 6) * 32768;
constexpr int kMaxStages = 12;
// The tensor cores' fp32 sums drop low bits, always towards zero, so their error grows with the number of steps: one group
// of positive rows in dw, relative to fp64: 700 rows 1.2e-6, 32768 rows 1.8e-4, 2^20 rows 6.8e-3, more than a rounding to
// bf16.  Kernels with PARTS therefore contract at most 64 stages (4096 indexes, 256 steps: 1.4e-5 in that example, at any
// length) in one go; the epilogue adds these parts, rounding to nearest, in the other accumulator (add_part), which takes
// about 1 us beside the 24 of a full part.  It also bounds how long an accumulator is waited for.  A call has it where its
// contraction can be longer than a part: d_lm_head and dw of more than 4096 rows, y and dx of wider experts (in every call
// it cost 131072 rows of y 10 %, 735 -> 815 us).  The logits contract the hidden size, and d_hidden, rounded to bf16, a part
// of a vocabulary piece (151936 entries in one go: 2e-4): they do without.
constexpr int kPartStages = 64;
bool in_parts(int64_t k) { return k > kPartStages * kStageK; }
constexpr int kGroupWords = 2 * (kUpMaxExperts + 1);
// statistics of two tiles, or the tokens' values of a chunk per warp; output stages
template <int EPI> constexpr int kEpiBytes = EPI == kStoreRows ? kEpiWarps * 4096 : 2 * 4 * kTileN * 8;
template <int EPI>
constexpr size_t smem_bytes(bool groups) {
    return (size_t)kRingBytes<EPI> + kEpiBytes<EPI> + 1024 + (groups ? kGroupWords * 4 : 0);
}

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
            else if ((int64_t)(t - begin) > 2000000000ll) return false;
        }
    }
    return false;
}
// The same for a whole warp: every lane polls for itself, all go on together or none does.
template <bool CLUSTER = false>
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, const volatile int& dead) {
    const bool ok = !dead && mb_wait<CLUSTER>(bar, parity);
    return __all_sync(0xffffffffu, ok) != 0;
}
// The same for the epilogue's warps, whose wait is long: 256 polling lanes get in the way of the producer's and the MMA
// warp's own polls (131072 expert rows: 729 us, 612 with one polling lane per warp), so lane 0 looks first.  What a warp
// goes on by is still what each of its lanes has seen: all of them test the barrier once lane 0 has found it ready.
__device__ __forceinline__ bool warp_wait_long(uint64_t* bar, uint32_t parity, int lane, const volatile int& dead) {
    if (lane == 0 && !dead) mb_wait(bar, parity);
    __syncwarp();
    return warp_wait(bar, parity, dead);
}
// A wait for the end of a contraction of nk stages: two seconds more for every 1024 of them (0.4 ms of work).
__device__ __forceinline__ bool warp_wait_stages(uint64_t* bar, uint32_t parity, int nk, const volatile int& dead) {
    for (int i = 0; i <= nk >> 10; ++i) {
        if (warp_wait(bar, parity, dead)) return true;
        if (__any_sync(0xffffffffu, dead)) return false;
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
// The barrier (`bar`: cluster address) may be the other CTA's.
__device__ __forceinline__ void tma_2d(uint32_t dst, const CUtensorMap* tm, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"((uint64_t)tm), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap* tm, int x, int y, int z, uint32_t bar) {
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

// fp32 accumulator, bf16 operands, bit 15 / 16: A / B is MN-major; the N width is added per tile
template <bool A_MN, bool B_MN>
constexpr uint32_t kIdesc = (1u << 4) | (1u << 7) | (1u << 10) | ((A_MN ? 1u : 0u) << 15) | ((B_MN ? 1u : 0u) << 16) |
                            ((uint32_t)(kTileM >> 4) << 24);

__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(da), "l"(db), "r"(idesc), "r"(accumulate) : "memory");
}
// Arrives on the barrier, of both CTAs at the same place, once the MMAs issued so far are done.
__device__ __forceinline__ void commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
}
// 32 columns of this thread's TMEM lane: the request, and the wait after which the values may be used (they pass
// through it, so that no use can be moved in front).
__device__ __forceinline__ void tmem_request(uint32_t taddr, float (&v)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
                   "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
                   "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]),
                   "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
                 : "r"(taddr));
}
__device__ __forceinline__ void tmem_wait(float (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                   "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]),
                   "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]),
                   "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])
                 :
                 : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float (&v)[32]) {
    tmem_request(taddr, v);
    tmem_wait(v);
}
__device__ __forceinline__ void tmem_store(uint32_t taddr, const float (&v)[32]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
                 ::"r"(taddr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]),
                   "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]),
                   "f"(v[16]), "f"(v[17]), "f"(v[18]), "f"(v[19]), "f"(v[20]), "f"(v[21]), "f"(v[22]), "f"(v[23]),
                   "f"(v[24]), "f"(v[25]), "f"(v[26]), "f"(v[27]), "f"(v[28]), "f"(v[29]), "f"(v[30]), "f"(v[31])
                 : "memory");
}
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// One output tile and its contraction.
struct Tile {
    int a_row, b_row;         // first M / N index in the operands' coordinates
    int m_valid, n_valid;     // M / N indexes that exist
    int width;                // N width of the MMA, a multiple of 32
    int k0, k_len;            // contraction range
    int expert;               // third coordinate of the expert stack
    int m_tile;
    int64_t out;              // element offset of the tile's corner in the output
    int width2;               // not 0: a second tile beside it in N works on the same A (PAIRS)
    int b_row2, n_valid2;
};

// Cuts an extent into `tiles` (= n / 256 rounded up) widths that differ by one unit at most: 32, the MMA's granularity, or
// 64 for out[m][n] (128-byte rows).  300 rows make tiles of 160 and 160, 270 rows 160 and 128.
template <int UNIT>
__device__ __forceinline__ void cut(int n, int tiles, int i, int* start, int* width) {
    const int units = (n + UNIT - 1) / UNIT, each = units / tiles, more = units - each * tiles;
    *start = (each * i + min(i, more)) * UNIT;
    *width = (each + (i < more ? 1 : 0)) * UNIT;
}

// Two N tiles side by side as one unit of work (PAIRS, for d_hidden of up to 512 rows): a stage holds A once and both tiles' B, so that
// 288 token rows, say, bring 34 KB per stage into an SM where two units bring 50 (one SM takes 75 - 85 GB/s from L2):
// 271 rows x 151936 entries 192 us single, 134 us as pairs.  The price is that both accumulators are taken and the
// epilogue does not hide behind the next unit, so it is for long contractions: for the logits (32 stages) pairs were
// slower, 194 us against 177, and more than two tiles fill the rounds better one by one (4096 rows: 771 us per piece as
// pairs, 575 single).
__device__ __forceinline__ int n_units(int n, bool pairs) {
    const int tiles = (n + kTileN - 1) / kTileN;
    return pairs ? (tiles + 1) / 2 : tiles;
}
// Room for B in a stage, in units of 2 KB (half of 32 rows, 128 bytes each): the widest unit of an extent.
__device__ __forceinline__ int b_room(int n, bool pairs) {
    const int most = pairs ? 16 : 8;
    return n <= most * 32 ? max(1, (n + 31) >> 5) : most;
}

// The units of work of a call, numbered the same way in every role.  `off`, `first`: group bounds and the number of
// units before each group, in shared memory.
template <int SCHED, bool ROWS, bool PAIRS>
struct TileMap {
    const UpParams& p;
    const int* off;
    const int* first;
    int n, k, tiles_m, units_n, count;

    __device__ __forceinline__ TileMap(const UpParams& q, const int* o, const int* f) : p(q), off(o), first(f) {
        n = p.n; k = p.k;
        if (SCHED == kDense) {
            if (p.n_live) n = *p.n_live;
            if (p.k_live) k = *p.k_live;
        }
        tiles_m = (p.m + kTileM - 1) / kTileM;
        units_n = n_units(n, PAIRS);
        count = SCHED == kGroupRows ? first[p.experts] : tiles_m * units_n * (SCHED == kGroupK ? p.experts : p.splits);
    }
    // Unit u of `per` N units x the M tiles: N fastest, so that neighbours share A, but in blocks of N whose B stays in
    // L2 while the M tiles pass (one group of 131072 rows x 2048, 537 MB of rows,
    // to 1536: 869 us without blocks, 690 us).
    __device__ __forceinline__ void in_blocks(Tile& r, int u, int per, int& tn) const {
        int first_n = 0, size = per;
        if (per > p.n_block) {
            const int b = u / (p.n_block * tiles_m);
            first_n = b * p.n_block;
            size = min(p.n_block, per - first_n);
            u -= first_n * tiles_m;
        }
        r.m_tile = u / size;
        tn = first_n + u - r.m_tile * size;
    }
    // N columns of unit tn of an extent of n that begins at row `base`.
    __device__ __forceinline__ static void columns(Tile& r, int n, int tn, int base) {
        const int tiles = (n + kTileN - 1) / kTileN, i = PAIRS ? 2 * tn : tn;
        int start;
        cut<ROWS ? 64 : 32>(n, tiles, i, &start, &r.width);
        r.b_row = base + start;
        r.n_valid = min(r.width, n - start);
        r.width2 = 0;
        if (PAIRS && i + 1 < tiles) {
            cut<ROWS ? 64 : 32>(n, tiles, i + 1, &start, &r.width2);
            r.b_row2 = base + start;
            r.n_valid2 = min(r.width2, n - start);
        }
    }
    // The second tile of a unit.
    __device__ __forceinline__ Tile second(Tile r) const {
        r.out += (int64_t)(r.b_row2 - r.b_row) * (ROWS ? 1 : p.e.ld);
        r.b_row = r.b_row2; r.width = r.width2; r.n_valid = r.n_valid2;
        r.width2 = 0;
        return r;
    }
    __device__ __forceinline__ Tile at(int t) const {
        Tile r;
        int tn;
        if (SCHED == kGroupRows) {
            int lo = 0, hi = p.experts - 1;          // the last group whose first tile is <= t: it has tiles
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (first[mid] <= t) lo = mid; else hi = mid - 1;
            }
            const int rows = off[lo + 1] - off[lo];
            in_blocks(r, t - first[lo], n_units(rows, PAIRS), tn);
            r.k0 = 0; r.k_len = k; r.expert = lo;
            columns(r, rows, tn, off[lo]);
            r.out = 0;
        } else {
            const int per = tiles_m * units_n, group = t / per, u = t - group * per;
            in_blocks(r, u, units_n, tn);
            columns(r, n, tn, 0);
            if (SCHED == kGroupK) {
                r.expert = group;
                r.k0 = off[group];
                r.k_len = off[group + 1] - off[group];
                r.out = (int64_t)group * p.e.split_stride;
            } else {
                const int stages = (k + kStageK - 1) / kStageK;
                const int s0 = (int)((int64_t)stages * group / p.splits), s1 = (int)((int64_t)stages * (group + 1) / p.splits);
                r.expert = 0;
                r.k0 = s0 * kStageK;
                r.k_len = min(k, s1 * kStageK) - r.k0;
                r.out = (int64_t)group * p.e.split_stride;
            }
        }
        r.a_row = r.m_tile * kTileM;
        r.m_valid = p.m - r.a_row;
        r.out += ROWS ? (int64_t)r.a_row * p.e.ld + r.b_row : (int64_t)r.b_row * p.e.ld + r.a_row;
        return r;
    }
};

// Group bounds in shared memory: clamped to [0, rows] and made non-decreasing, so that no offset array leads
// outside the operands; first[e] = tiles of the groups before e.  One warp.
__device__ __forceinline__ void load_groups(const UpParams& p, int* off, int* first, int tiles_m, int lane) {
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
    for (int i = b; i < min(e, E); ++i) sum += n_units(off[i + 1] - off[i], false) * tiles_m;
    int pre = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, pre, o);
        if (lane >= o) pre += v;
    }
    pre -= sum;
    for (int i = b; i < e; ++i) {
        first[i] = pre;
        if (i < E) pre += n_units(off[i + 1] - off[i], false) * tiles_m;
    }
    __syncwarp();
}

// ---------------------------------------------------------------------------------------- epilogues
// `taddr`: this thread's lane of the accumulator, column 0; ch: its M index in the tile; c0 .. c1: its warp's columns.

// Two columns of a warp (32 M indexes each) as packed pairs: even lanes get (m, m + 1) of column j, odd lanes of
// column j + 1, so that a store instruction writes 64 contiguous bytes for each of two output rows.
__device__ __forceinline__ uint32_t pair_columns(float a, float b, bool odd) {
    const uint32_t mine = pack_bf16(a, b), other = __shfl_xor_sync(0xffffffffu, mine, 1);
    return __byte_perm(mine, other, odd ? 0x3276 : 0x5410);
}

// 32 columns of the tile, from column c on: bf16 (rounded once from the fp32 accumulator) or fp32, the latter optionally
// on top of what is there (the parts of d_hidden; nothing adds to bf16 here).
__device__ __forceinline__ void store_chunk(const UpEpilogue& e, const Tile& t, int ch, int c, int left, float (&v)[32]) {
    const bool live = ch < t.m_valid, odd = ch & 1;
    const bool whole = left >= 32 && (ch | 31) < t.m_valid;          // the same for the warp
    if (e.out_f32) {
        float* dst = reinterpret_cast<float*>(e.out) + t.out + (int64_t)c * e.ld + ch;
        if (whole && !e.accumulate) {
#pragma unroll
            for (int j = 0; j < 32; ++j, dst += e.ld) *dst = v[j];
            return;
        }
        if (e.accumulate) {
            const float* old = dst;
#pragma unroll
            for (int j = 0; j < 32; ++j, old += e.ld)
                if (live && j < left) v[j] += *old;
        }
#pragma unroll
        for (int j = 0; j < 32; ++j, dst += e.ld)
            if (live && j < left) *dst = v[j];
    } else {
        __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(e.out) + t.out + (int64_t)(c + odd) * e.ld + (ch - odd);
        const int64_t step = 2 * e.ld;
        if (whole) {
#pragma unroll
            for (int j = 0; j < 32; j += 2, dst += step) *reinterpret_cast<uint32_t*>(dst) = pair_columns(v[j], v[j + 1], odd);
            return;
        }
#pragma unroll
        for (int j = 0; j < 32; j += 2, dst += step) {
            const uint32_t w = pair_columns(v[j], v[j + 1], odd);
            if (live && j + odd < left) *reinterpret_cast<uint32_t*>(dst) = w;
        }
    }
}

// The same for out[m][n]: a thread owns an output row and its columns lie side by side.
__device__ __forceinline__ void store_rows_chunk(const UpEpilogue& e, const Tile& t, int row, int c, int left, float (&v)[32]) {
    if (row >= t.m_valid) return;
    const int64_t at = t.out + (int64_t)row * e.ld + c;
    if (e.out_f32) {
        float* dst = reinterpret_cast<float*>(e.out) + at;
        if (e.accumulate) {
#pragma unroll
            for (int j = 0; j < 32; j += 4)
                if (j < left) {
                    const float4 o = *reinterpret_cast<const float4*>(dst + j);
                    v[j] += o.x; v[j + 1] += o.y; v[j + 2] += o.z; v[j + 3] += o.w;
                }
        }
#pragma unroll
        for (int j = 0; j < 32; j += 8)
            if (j < left) {                                     // extents are multiples of 8
                *reinterpret_cast<float4*>(dst + j) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                *reinterpret_cast<float4*>(dst + j + 4) = make_float4(v[j + 4], v[j + 5], v[j + 6], v[j + 7]);
            }
    } else {
        __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(e.out) + at;
        if (e.accumulate) {
#pragma unroll
            for (int j = 0; j < 32; j += 8)
                if (j < left) {
                    const uint4 o = *reinterpret_cast<const uint4*>(dst + j);
                    const uint32_t ow[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                    for (int q = 0; q < 4; ++q) { v[j + 2 * q] += bf16_lo(ow[q]); v[j + 2 * q + 1] += bf16_hi(ow[q]); }
                }
        }
#pragma unroll
        for (int j = 0; j < 32; j += 8)
            if (j < left)
                *reinterpret_cast<uint4*>(dst + j) = make_uint4(pack_bf16(v[j], v[j + 1]), pack_bf16(v[j + 2], v[j + 3]),
                                                                pack_bf16(v[j + 4], v[j + 5]), pack_bf16(v[j + 6], v[j + 7]));
    }
}

// out[m][n] without adding, the way dw and d_lm_head leave the kernel: the contraction is short there and the output is
// the work, so the load/store pipe must not be the limit (dw of 128 x 1536 x 2048 with few rows: 250 us with pair stores
// and exchanges, 292 us with 32-byte stores per thread, 196 us this way, which is what writing 805 MB takes: a fill of
// that size runs at 3.9 TB/s, 207 us).  A warp lays 32 rows of 128 bytes side by side in shared memory (128-byte swizzle,
// no bank conflicts) and a bulk tensor copy takes them out; rows and columns behind the matrix's end are clipped by it.
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* tm, uint32_t src, int x, int y, int z) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
                 ::"l"((uint64_t)tm), "r"(src), "r"(x), "r"(y), "r"(z) : "memory");
}
template <typename F>
__device__ __forceinline__ void store_tile_bulk(const UpEpilogue& e, const CUtensorMap* tm, const Tile& t, int row0, int c0, int c1,
                                                uint32_t taddr, unsigned char* stage, int lane, bool elected, F release) {
    const int end = min(c1, t.n_valid);
    const bool rows = row0 < t.m_valid;                              // the same for the warp
    unsigned char* mine = stage + lane * 128;
    const int turn = lane & 7;
    const uint32_t src = smem_u32(stage);
    const auto hand_over = [&](int x) {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (elected) {
            if (rows) tma_store_3d(tm, src, x, t.a_row + row0, t.expert);
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
    };
    const auto reclaim = [&] {                                       // the copy before has read the stage
        if (elected) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
    };
    float v[32], w[32];
#pragma unroll 1
    for (int c = c0; c < end; c += 64) {
        tmem_request(taddr + c, v);
        tmem_wait(v);
        tmem_request(taddr + c + 32, w);
        reclaim();
        if (e.out_f32) {
#pragma unroll
            for (int q = 0; q < 8; ++q)
                *reinterpret_cast<float4*>(mine + ((q ^ turn) * 16)) = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
            hand_over(t.b_row + c);
            tmem_wait(w);
            if (c + 64 >= end) release();
            reclaim();
#pragma unroll
            for (int q = 0; q < 8; ++q)
                *reinterpret_cast<float4*>(mine + ((q ^ turn) * 16)) = make_float4(w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
            if (c + 32 < end) hand_over(t.b_row + c + 32);
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<uint4*>(mine + ((q ^ turn) * 16)) =
                    make_uint4(pack_bf16(v[8 * q], v[8 * q + 1]), pack_bf16(v[8 * q + 2], v[8 * q + 3]), pack_bf16(v[8 * q + 4], v[8 * q + 5]),
                               pack_bf16(v[8 * q + 6], v[8 * q + 7]));
            tmem_wait(w);
            if (c + 64 >= end) release();
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<uint4*>(mine + (((q + 4) ^ turn) * 16)) =
                    make_uint4(pack_bf16(w[8 * q], w[8 * q + 1]), pack_bf16(w[8 * q + 2], w[8 * q + 3]), pack_bf16(w[8 * q + 4], w[8 * q + 5]),
                               pack_bf16(w[8 * q + 6], w[8 * q + 7]));
            hand_over(t.b_row + c);
        }
    }
    if (c0 >= end) release();
}

// The tile's columns c0 .. c1, the next 32 requested from TMEM while the ones before are stored; `release` is called as
// soon as the accumulator has been read.
template <bool ROWS, typename F>
__device__ __forceinline__ void store_tile(const UpEpilogue& e, const Tile& t, int ch, int c0, int c1, uint32_t taddr, F release) {
    const int end = min(c1, t.n_valid);
    float v[32], w[32];
    if (c0 < end) {
        tmem_request(taddr + c0, v);
        tmem_wait(v);
    }
#pragma unroll 1
    for (int c = c0; c < end; c += 64) {
        const bool second = c + 32 < end, third = c + 64 < end;
        if (second) tmem_request(taddr + c + 32, w);
        else release();
        if (ROWS) store_rows_chunk(e, t, ch, c, end - c, v); else store_chunk(e, t, ch, c, end - c, v);
        if (!second) return;
        tmem_wait(w);
        if (third) tmem_request(taddr + c + 64, v);
        else release();
        if (ROWS) store_rows_chunk(e, t, ch, c + 32, end - c - 32, w); else store_chunk(e, t, ch, c + 32, end - c - 32, w);
        if (!third) return;
        tmem_wait(v);
    }
    release();          // no column of this warp exists
}
template <bool ROWS>
__device__ __forceinline__ void store_zeros(const UpEpilogue& e, const Tile& t, int ch, int c0, int c1) {
    const int end = min(c1, t.n_valid);
#pragma unroll 1
    for (int c = c0; c < end; c += 32) {
        float v[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = 0.f;
        if (ROWS) store_rows_chunk(e, t, ch, c, end - c, v); else store_chunk(e, t, ch, c, end - c, v);
    }
}

// A part of a long contraction (kPartStages) on top of the parts before it: columns c0 .. end of this warp, `sum` written and
// read by the same threads only.
__device__ __forceinline__ void add_part(uint32_t part, uint32_t sum, int c0, int end, bool first) {
#pragma unroll 1
    for (int c = c0; c < end; c += 32) {
        float v[32];
        tmem_ld32(part + c, v);
        if (!first) {
            float w[32];
            tmem_ld32(sum + c, w);
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] += w[j];
        }
        tmem_store(sum + c, v);
    }
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ float redux_max(float v) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}

// Softmax statistics of the tile's vocabulary entries for every token, the token's own target left out (its
// logit is computed apart, in fp32): the largest logit M (before the temperature) and sum exp((logit - M) / T).
// Differences are taken before the scaling, so the exponents carry no rounding of large values.  A warp holds 32
// entries x 32 tokens at a time: the maximum of a token is one redux, the sums of 32 tokens take 31 exchanges
// (halving the number of columns a lane holds each time), after which lane l has token l's; the four warps of
// a column half meet in shared memory.
__device__ __forceinline__ void stats_tile(const UpEpilogue& e, const Tile& t, int ch, int c0, int c1, uint32_t taddr, float2* meet,
                                           int quarter, int half, int lane, int slot, int slots, const int* n_live) {
    const bool live = ch < t.m_valid;
    const int v_row = t.a_row + ch, end = min(c1, t.n_valid);
    const float scale = e.inv_temp * 1.4426950408889634f;
#pragma unroll 1
    for (int c = c0; c < end; c += 32) {
        float v[32];
        tmem_ld32(taddr + c, v);
        const int tok = t.b_row + c + lane;
        const int tgt = tok < *n_live ? e.target[tok] - (v_row - lane) : -1;           // its lane, if the warp holds the target
        const uint32_t hits = __ballot_sync(0xffffffffu, (unsigned)tgt < 32u);
        if (hits) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if ((hits >> j) & 1) {
                    if (__shfl_sync(0xffffffffu, tgt, j) == lane) v[j] = -INFINITY;
                }
        }
        float mine = -INFINITY;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            if (!live) v[j] = -INFINITY;
            const float m = redux_max(v[j]);
            if (lane == j) mine = m;
            v[j] = exp2_approx((v[j] - (m == -INFINITY ? 0.f : m)) * scale);       // nothing but -inf: all terms are 0
        }
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) {
            const bool up = lane & o;
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (j < o) {
                    const float give = up ? v[j] : v[j + o], keep = up ? v[j + o] : v[j];
                    v[j] = keep + __shfl_xor_sync(0xffffffffu, give, o);
                }
        }
        meet[quarter * kTileN + c + lane] = make_float2(mine, v[0]);
    }
    __syncwarp();
    asm volatile("bar.sync %0, 128;" ::"r"(1 + half) : "memory");
    const int col = c0 + quarter * 32 + lane;
    if (col < end) {
        float mx = -INFINITY, sum = 0.f;
#pragma unroll
        for (int q = 0; q < 4; ++q) mx = fmaxf(mx, meet[q * kTileN + col].x);
        const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float2 s = meet[q * kTileN + col];
            sum += s.y * exp2_approx((s.x - ref) * scale);
        }
        e.stats[(int64_t)(t.b_row + col) * slots + slot] = make_float2(mx, sum);
    }
}

// Gradient of the logits: d = w ([v = t] - p), p = exp(z - lse), w = g / T, rounded to bf16 (relative 2^-8 at
// most, independent from entry to entry) because it is an operand of two tensor-core products; for calls of few
// rows, which are streams of the lm_head anyway, what the rounding took off is stored as a second bf16 row.  The
// target's own value w (1 - p) is prepared per row (live_rows_kernel).  Tokens and
// entries behind the end are written as zeros: they are contraction indexes of those products.
// The factor is taken into the exponent, w p = sign exp2(z log2 e / T + log2 |w| - lse log2 e), so that a token's share
// of the work on its 32 entries is one number out of shared memory (read four tokens at a time: the MMAs of the next
// tile need that memory's bandwidth) and a sign out of a mask; a target is found by one ballot for 32 tokens.
__device__ __forceinline__ void dlogits_tile(const UpEpilogue& e, const Tile& t, int ch, int c0, int c1, uint32_t taddr, float* tokens,
                                             int lane, const int* n_live) {
    const int v_row = e.v0 + t.a_row + ch, end = min(c1, t.width), n = *n_live;
    const bool live = v_row < e.vocab, odd = ch & 1;
    const float scale = e.inv_temp * 1.4426950408889634f;
#pragma unroll 1
    for (int c = c0; c < end; c += 32) {
        float v[32];
        tmem_request(taddr + c, v);
        const int tok = t.b_row + c + lane;
        const bool here = tok < n;
        float k = -INFINITY, w = 0.f;
        int tgt = -1;
        if (here) {
            w = e.weight[tok];
            k = fmaf(e.lse[tok], -1.4426950408889634f, log2f(fabsf(w)));
            tgt = e.target[tok] - (v_row - lane);                    // its lane, if the warp holds the target
        }
        __syncwarp();
        tokens[lane] = k;
        const uint32_t minus = __ballot_sync(0xffffffffu, w > 0.f), hits = __ballot_sync(0xffffffffu, (unsigned)tgt < 32u);
        tmem_wait(v);
        __syncwarp();
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float4 k4 = reinterpret_cast<const float4*>(tokens)[q];
            const float ks[4] = {k4.x, k4.y, k4.z, k4.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = 4 * q + i;
                v[j] = __uint_as_float(__float_as_uint(exp2_approx(fmaf(v[j], scale, ks[i]))) ^ ((minus << (31 - j)) & 0x80000000u));
            }
        }
        if (hits) {
            const float d = (unsigned)tgt < 32u ? e.target_d[tok] : 0.f;
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if ((hits >> j) & 1) {
                    const float dj = __shfl_sync(0xffffffffu, d, j);
                    if (__shfl_sync(0xffffffffu, tgt, j) == lane) v[j] = dj;
                }
        }
        const int left = n - (t.b_row + c);
        if (left < 32 || v_row - lane + 32 > e.vocab) {              // tokens or entries behind the end
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = live && j < left ? v[j] : 0.f;
        }
        __nv_bfloat16* dst = e.dlogits + (int64_t)(t.b_row + c + odd) * e.ld + (t.a_row + ch - odd);
        const int64_t step = 2 * e.ld, lo = (int64_t)e.lo_rows * e.ld;
#pragma unroll
        for (int j = 0; j < 32; j += 2, dst += step) {
            const uint32_t u = pair_columns(v[j], v[j + 1], odd);
            *reinterpret_cast<uint32_t*>(dst) = u;
            if (lo) {
                const float got = __shfl_xor_sync(0xffffffffu, odd ? v[j] : v[j + 1], 1);
                *reinterpret_cast<uint32_t*>(dst + lo) = pack_bf16((odd ? got : v[j]) - bf16_lo(u), (odd ? v[j + 1] : got) - bf16_hi(u));
            }
        }
    }
}

// The work of one pair of CTAs, number `worker` of `workers` on this contraction.
template <bool A_MN, bool B_MN, int SCHED, int EPI, bool PAIRS, bool PARTS>
__device__ __forceinline__ void contract(const UpMaps& maps, const UpParams& p, const int worker, const int workers) {
    extern __shared__ unsigned char up_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>(((uintptr_t)up_raw + 1023) & ~(uintptr_t)1023);
    unsigned char* epi = smem + kRingBytes<EPI>;
    int* off = reinterpret_cast<int*>(epi + kEpiBytes<EPI>);
    int* first = off + kUpMaxExperts + 1;
    __shared__ __align__(8) uint64_t full[kMaxStages], empty[kMaxStages], tail[kMaxStages], acc_full[2], acc_empty[2];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int dead;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int rank = (int)(blockIdx.x & 1);                    // place in the pair; rank 0 leads
    // a stage of kGroupK is full after two arrivals: the leader's own two, or one of each CTA that cleared rows
    constexpr int kFullCount = SCHED == kGroupK ? 2 : 1;

    if (tid < kMaxStages) {
        mb_init(&full[tid], kFullCount);
        mb_init(&empty[tid], 1);
        mb_init(&tail[tid], 1);
        if (tid < 2) { mb_init(&acc_full[tid], 1); mb_init(&acc_empty[tid], 2 * kEpiWarps); }
        dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(2 * kTileN));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    pdl_wait();
    if (SCHED != kDense && warp == 3) load_groups(p, off, first, (p.m + kTileM - 1) / kTileM, lane);
    __syncwarp();
    cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem_d = tmem_slot;
    const TileMap<SCHED, EPI == kStoreRows, PAIRS> map(p, off, first);
    const uint32_t ring = smem_u32(smem);
    constexpr bool kFullStages = B_MN || SCHED != kDense;
    const uint32_t stage_bytes = kABytes + (kFullStages ? kBBytes : b_room(map.n, PAIRS) * 2048);
    const int stages = kFullStages ? kRingBytes<EPI> / (kABytes + kBBytes) : min(kMaxStages, (int)(kRingBytes<EPI> / 2048u / (stage_bytes >> 11)));

    if (warp == 0) {
        const bool elected = elect_one();
        uint32_t it = 0;
        int s = 0;
        uint32_t phase = 0;
        bool ok = true;
        for (int tile = worker; ok && tile < map.count; tile += workers) {
            const Tile t = map.at(tile);
            const int nk = (t.k_len + kStageK - 1) / kStageK;
            const int half = t.width / 2, a_row = t.a_row + rank * 128, b_row = t.b_row + rank * half;
            const int half2 = PAIRS ? t.width2 / 2 : 0, b_row2 = t.b_row2 + rank * half2;
            // B, K-major: the half's rows in boxes of 128, or of 64, 32 and 16; MN-major: one or two boxes of 64 columns
            const uint32_t b_bytes = B_MN ? (uint32_t)((half + 63) / 64 * kMnBox) : (uint32_t)(half + half2) * 128u;
            const auto load_rows = [&](uint32_t dst, int k, int row, int n, uint32_t bar) {
                if (n == 128) {
                    tma_2d(dst, &maps.b[3], k, row, bar);
                    return;
                }
                const int r32 = n & 64, r16 = n & 96;
                if (n & 64) tma_2d(dst, &maps.b[2], k, row, bar);
                if (n & 32) tma_2d(dst + r32 * 128, &maps.b[1], k, row + r32, bar);
                if (n & 16) tma_2d(dst + r16 * 128, &maps.b[0], k, row + r16, bar);
            };
            for (int ks = 0; ks < nk; ++ks) {
                ok = warp_wait(&empty[s], phase ^ 1, dead);
                if (!ok) break;
                const uint32_t sa = ring + (uint32_t)s * stage_bytes, sb = sa + kABytes;
                const int k = t.k0 + ks * kStageK;
                const bool ragged = SCHED == kGroupK && (t.k_len - ks * kStageK) < kStageK && t.k_len % 16;
                // a ragged stage is reported by the clearing warps, any other by the copies to the leader
                const uint32_t bar = ragged ? in_cta(&tail[s], rank) : in_cta(&full[s], 0);
                if (elected) {
                    if (ragged) {
                        mb_expect(&tail[s], kABytes + b_bytes);
                    } else if (rank == 0) {
                        if (kFullCount == 2) mb_arrive(&full[s]);
                        mb_expect(&full[s], 2 * (kABytes + b_bytes));
                    }
                    if (A_MN) {
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            if (SCHED == kGroupRows) tma_3d(sa + b * kMnBox, &maps.a, a_row + b * 64, k, t.expert, bar);
                            else tma_2d(sa + b * kMnBox, &maps.a, a_row + b * 64, k, bar);
                        }
                    } else {
                        if (SCHED == kGroupRows) tma_3d(sa, &maps.a, k, a_row, t.expert, bar);
                        else tma_2d(sa, &maps.a, k, a_row, bar);
                    }
                    if (B_MN) {
                        tma_2d(sb, &maps.b[0], b_row, k, bar);
                        if (half > 64) tma_2d(sb + kMnBox, &maps.b[0], b_row + 64, k, bar);
                    } else {
                        load_rows(sb, k, b_row, half, bar);
                        if (PAIRS && half2) load_rows(sb + half * 128, k, b_row2, half2, bar);
                    }
                }
                __syncwarp();
                ++it;
                if (++s == stages) { s = 0; phase ^= 1; }
            }
        }
        // The last stages' release is waited for as well: it says that the copies into them and the MMAs on them are
        // done, and it is a signal from the leader's MMAs into this CTA's shared memory, which must not be given up
        // before (the epilogue's accumulator signal is another one and need not come later).  After a wait that
        // gave up the copies in flight are waited for instead.
        const uint32_t st = (uint32_t)stages, from = it > st ? it - st : 0;
        for (uint32_t w = from; ok && w < it; ++w) ok = warp_wait(&empty[w % st], (w / st) & 1, dead);
        if (!ok) {
            if (lane == 0) { dead = 1; atomicOr(p.err, kErrTimeout); }
            if (rank == 0)
                for (uint32_t w = from; w < it; ++w) mb_wait(&full[w % st], (w / st) & 1);
        }
    } else if (warp == 1) {
        if (rank == 0) {
            const bool elected = elect_one();
            int s = 0, buf = 0;                               // stage; accumulator (they take turns)
            uint32_t phase = 0, uses = 0;                     // uses: parity of each accumulator's next use
            bool ok = true;
            const uint64_t desc_a = smem_desc<A_MN>(ring), desc_b = smem_desc<B_MN>(ring + kABytes);
            for (int tile = worker; ok && tile < map.count; tile += workers) {
                const Tile t = map.at(tile);
                const int nk = (t.k_len + kStageK - 1) / kStageK;
                if (nk <= 0) continue;                        // nothing to contract: the epilogue writes zeros
                const bool two = PAIRS && t.width2, parts = PARTS && nk > kPartStages, both = two || parts;
                ok = warp_wait<true>(&acc_empty[buf], ((uses >> buf) & 1) ^ 1, dead);
                if (both && ok) ok = warp_wait<true>(&acc_empty[buf ^ 1], ((uses >> (buf ^ 1)) & 1) ^ 1, dead);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t acc = tmem_d + (uint32_t)(buf * kTileN), acc2 = tmem_d + (uint32_t)((buf ^ 1) * kTileN);
                const uint32_t idesc = kIdesc<A_MN, B_MN> | ((uint32_t)(t.width >> 3) << 17);
                const uint32_t idesc2 = kIdesc<A_MN, B_MN> | ((uint32_t)((PAIRS ? t.width2 : 0) >> 3) << 17);
                int from = 0, last = PARTS ? min(nk, kPartStages) - 1 : nk - 1;      // stages of the part
                for (int ks = 0; ok && ks < nk; ++ks) {
                    const int left = t.k_len - ks * kStageK;
                    const int steps = left >= kStageK ? 4 : (left + 15) / 16;
                    ok = warp_wait<SCHED == kGroupK>(&full[s], phase, dead);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t da = desc_a + (uint64_t)(s * (stage_bytes >> 4)), db = desc_b + (uint64_t)(s * (stage_bytes >> 4));
                    if (elected) {
                        if (steps == 4) {
#pragma unroll
                            for (int kk = 0; kk < 4; ++kk)
                                mma_f16(acc, da + kDescStep<A_MN> * kk, db + kDescStep<B_MN> * kk, idesc, kk == 0 ? ks != from : 1u);
                        } else {
                            for (int kk = 0; kk < steps; ++kk)
                                mma_f16(acc, da + kDescStep<A_MN> * kk, db + kDescStep<B_MN> * kk, idesc, ks != from || kk);
                        }
                        if (two) {                            // half the first tile's rows x 128 bytes further, in units of 16
                            const uint64_t db2 = db + (uint64_t)(t.width * 4);
                            for (int kk = 0; kk < steps; ++kk)
                                mma_f16(acc2, da + kDescStep<A_MN> * kk, db2 + kDescStep<B_MN> * kk, idesc2, ks != from || kk);
                        }
                        commit(&empty[s]);
                        if (ks == last) {
                            commit(&acc_full[buf]);
                            if (both && ks == nk - 1) commit(&acc_full[buf ^ 1]);
                        }
                    }
                    __syncwarp();
                    if (PARTS && ks == last && ks != nk - 1) {       // the next part, once this one has been taken
                        from = ks + 1;
                        last = min(nk, from + kPartStages) - 1;
                        uses ^= 1u << buf;
                        ok = warp_wait<true>(&acc_empty[buf], ((uses >> buf) & 1) ^ 1, dead);
                    }
                    if (++s == stages) { s = 0; phase ^= 1; }
                }
                uses ^= both ? 3u : 1u << buf;
                if (!both) buf ^= 1;
            }
            if (!ok && lane == 0) { dead = 1; atomicOr(p.err, kErrTimeout); }
        }
    } else if (warp == 2 + kEpiWarps) {
        // kGroupK, a warp of either CTA: the rows behind a group's end, up to the step's 16, are cleared in the stage
        // that holds the end; the MMA warp finds the stage full once both CTAs have done so.
        if (SCHED == kGroupK) {
            const bool elected = elect_one();
            uint32_t tails = 0;                               // parity of every stage's tail barrier
            int s = 0;
            bool ok = true;
            for (int tile = worker; ok && tile < map.count; tile += workers) {
                const Tile t = map.at(tile);
                const int nk = (t.k_len + kStageK - 1) / kStageK;
                if (nk <= 0) continue;
                const int last = (s + nk - 1) % stages, left = t.k_len - (nk - 1) * kStageK;
                s = (s + nk) % stages;
                if (left % 16 == 0) continue;
                ok = warp_wait_stages(&tail[last], (tails >> last) & 1, nk, dead);
                if (!ok) break;
                tails ^= 1u << last;
                unsigned char* st = smem + (size_t)last * stage_bytes + (lane & 7) * 16;
                const int boxes = 2 + (t.width / 2 + 63) / 64, end = (left + 15) & ~15;
                for (int row = left + (lane >> 3); row < end; row += 4)
                    for (int box = 0; box < boxes; ++box)
                        *reinterpret_cast<uint4*>(st + (size_t)box * kMnBox + row * 128) = make_uint4(0, 0, 0, 0);
                asm volatile("fence.proxy.async;" ::: "memory");
                __syncwarp();
                if (elected) mb_arrive_at(in_cta(&full[last], 0));
                __syncwarp();
            }
            if (!ok && lane == 0) { dead = 1; atomicOr(p.err, kErrTimeout); }
        }
    } else {
        // a warp may touch the TMEM lanes 32 (warp % 4) .. + 31; the first four warps take the left half of the columns
        const int quarter = warp & 3, half = (warp - 2) >> 2, ch = rank * 128 + quarter * 32 + lane;
        const bool elected = elect_one();
        int buf = 0;
        uint32_t uses = 0;
        bool ok = true;
        const uint32_t lanes = tmem_d + ((uint32_t)(quarter * 32) << 16);
        const auto release_acc = [&](int b) {           // this warp has read its part of the accumulator
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) mb_arrive_at(in_cta(&acc_empty[b], 0));
        };
        for (int tile = worker, which = 0; ok && tile < map.count; tile += which ? 0 : workers) {
            Tile t = map.at(tile);
            if (PAIRS) {                  // the two tiles of a unit, one after the other
                if (which) t = map.second(t);
                which = !which && t.width2;
            }
            constexpr int kCols = EPI == kStoreRows ? 64 : 32;
            const int mid = (t.width / 2 + kCols - 1) & ~(kCols - 1), c0 = half ? mid : 0, c1 = half ? t.width : mid;
            if (t.k_len <= 0) {
                if ((EPI == kStore || EPI == kStoreRows) && !p.e.accumulate) store_zeros<EPI == kStoreRows>(p.e, t, ch, c0, c1);
                continue;
            }
            const int nk = (t.k_len + kStageK - 1) / kStageK;
            const bool parts = PARTS && nk > kPartStages;
            if (parts) {
                for (int ks = 0; ks < nk; ks += kPartStages) {
                    ok = warp_wait_long(&acc_full[buf], (uses >> buf) & 1, lane, dead);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    add_part(lanes + (uint32_t)(buf * kTileN), lanes + (uint32_t)((buf ^ 1) * kTileN), c0, min(c1, t.n_valid), ks == 0);
                    release_acc(buf);
                    uses ^= 1u << buf;
                }
                if (!ok) break;
            }
            const int acc = parts ? buf ^ 1 : buf;       // what is stored
            ok = EPI == kStats ? warp_wait(&acc_full[acc], (uses >> acc) & 1, dead) : warp_wait_long(&acc_full[acc], (uses >> acc) & 1, lane, dead);
            if (EPI == kStats) {          // the warps of a column half meet on a barrier: all of them go on, or none
                uint32_t all_ok;
                __syncwarp();
                asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.and.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                             : "=r"(all_ok) : "r"((uint32_t)ok), "r"(1 + half) : "memory");
                ok = all_ok != 0;
            }
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t taddr = lanes + (uint32_t)(acc * kTileN);
            const auto release = [&] { release_acc(acc); };
            if (EPI == kStats) {
                stats_tile(p.e, t, ch, c0, c1, taddr, reinterpret_cast<float2*>(epi) + acc * 4 * kTileN, quarter, half, lane,
                           t.m_tile * 2 + rank, map.tiles_m * 2, p.n_live);
                release();
            } else if (EPI == kDlogits) {
                dlogits_tile(p.e, t, ch, c0, c1, taddr, reinterpret_cast<float*>(epi) + (warp - 2) * 32, lane, p.e.n_live);
                release();
            } else if (EPI == kStoreRows && p.e.bulk) {
                store_tile_bulk(p.e, &maps.out, t, ch - lane, c0, c1, taddr, epi + (warp - 2) * 4096, lane, elected, release);
            } else {
                store_tile<EPI == kStoreRows>(p.e, t, ch, c0, c1, taddr, release);
            }
            uses ^= 1u << acc;
            if (!parts) buf ^= 1;
        }
        if (!ok && lane == 0) { dead = 1; atomicOr(p.err, kErrTimeout); }
        if (EPI == kStoreRows && elected) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");     // copies out have read their stages
        __syncwarp();
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    // neither CTA of a pair leaves while the other may still signal its barriers or read its operands; after a wait
    // that gave up, what is in flight (copies, MMAs and their signals: microseconds) gets two milliseconds to land
    __syncwarp();
    if (__any_sync(0xffffffffu, dead))
        for (int i = 0; i < 2000; ++i) __nanosleep(1000);
    __syncwarp();
    cluster_sync();
    if (warp == 2) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem_d), "r"(2 * kTileN));
    }
}

template <bool A_MN, bool B_MN, int SCHED, int EPI, bool PAIRS, bool PARTS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
contract_kernel(const __grid_constant__ UpMaps maps, const __grid_constant__ UpParams p) {
    contract<A_MN, B_MN, SCHED, EPI, PAIRS, PARTS>(maps, p, blockIdx.x / 2, gridDim.x / 2);
}

// d_hidden and d_lm_head of a piece side by side, for small calls: the first pairs of CTAs work on the one, the others on
// the other.  Both need nothing but d, and neither fills the SMs then (37 rows x 264 x 1013, both calls: 45.7 us with a
// launch each, 39.3 us).  Where they do, each alone is bound by what one SM or HBM moves, and side by side takes as long
// (64 rows x 2048 x 151936: 103 + 196 us, together 300; 500 rows 507 us, 611).
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
both_gradients_kernel(const __grid_constant__ UpMaps hidden_maps, const __grid_constant__ UpParams hidden,
                      const __grid_constant__ UpMaps head_maps, const __grid_constant__ UpParams head, const int hidden_pairs) {
    const int pair = blockIdx.x / 2;
    if (pair < hidden_pairs) contract<true, false, kDense, kStore, true, false>(hidden_maps, hidden, pair, hidden_pairs);
    else contract<true, true, kDense, kStoreRows, false, false>(head_maps, head, pair - hidden_pairs, gridDim.x / 2 - hidden_pairs);
}

template <bool A_MN, bool B_MN, int SCHED, int EPI, bool PAIRS = false, bool PARTS = false>
cudaError_t launch(const UpMaps& m, const UpParams& p, int64_t tiles, int sms, cudaStream_t st) {
    const int64_t want = tiles < 1 ? 1 : tiles, pairs = sms / 2;
    return launch_chained(contract_kernel<A_MN, B_MN, SCHED, EPI, PAIRS, PARTS>, dim3((unsigned)(want < pairs ? want : pairs) * 2), dim3(kThreads),
                          smem_bytes<EPI>(SCHED != kDense), st, m, p);
}
template <bool A_MN, bool B_MN, int SCHED, int EPI, bool PAIRS = false, bool PARTS = false>
cudaError_t init_one() {
    return cudaFuncSetAttribute(contract_kernel<A_MN, B_MN, SCHED, EPI, PAIRS, PARTS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                (int)smem_bytes<EPI>(SCHED != kDense));
}
constexpr size_t kBothBytes = std::max(smem_bytes<kStore>(false), smem_bytes<kStoreRows>(false));
int64_t tiles_of(int64_t m, int64_t n) { return ((m + kTileM - 1) / kTileM) * ((n + kTileN - 1) / kTileN); }
}  // namespace

cudaError_t init_update_kernels() {
    cudaError_t e = init_one<false, false, kDense, kStats>();
    if (e == cudaSuccess) e = init_one<false, false, kDense, kDlogits>();
    if (e == cudaSuccess) e = init_one<true, false, kDense, kStore>();
    if (e == cudaSuccess) e = init_one<true, false, kDense, kStore, true>();
    if (e == cudaSuccess) e = cudaFuncSetAttribute(both_gradients_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kBothBytes);
    if (e == cudaSuccess) e = init_one<true, true, kDense, kStoreRows>();
    if (e == cudaSuccess) e = init_one<true, true, kDense, kStoreRows, false, true>();
    if (e == cudaSuccess) e = init_one<false, false, kGroupRows, kStore>();
    if (e == cudaSuccess) e = init_one<false, false, kGroupRows, kStore, false, true>();
    if (e == cudaSuccess) e = init_one<true, false, kGroupRows, kStore>();
    if (e == cudaSuccess) e = init_one<true, false, kGroupRows, kStore, false, true>();
    if (e == cudaSuccess) e = init_one<true, true, kGroupK, kStoreRows>();
    if (e == cudaSuccess) e = init_one<true, true, kGroupK, kStoreRows, false, true>();
    return e;
}

cudaError_t launch_logit_stats(const UpMaps& m, const UpParams& p, int sms, cudaStream_t st) {
    return launch<false, false, kDense, kStats>(m, p, tiles_of(p.m, p.n), sms, st);
}
cudaError_t launch_dlogits(const UpMaps& m, const UpParams& p, int sms, cudaStream_t st) {
    return launch<false, false, kDense, kDlogits>(m, p, tiles_of(p.m, p.n), sms, st);
}
// Pairs of CTAs for d_hidden where d_lm_head leaves at least half of them: all that have no tile of it.  0: a launch each.
int both_hidden_pairs(int rows, int width, int hidden, int slots) {
    const int64_t tiles = tiles_of(width, hidden);
    return rows <= kUpBothRows && 2 * tiles <= slots ? (int)(slots - tiles) : 0;
}
cudaError_t launch_both_gradients(const UpMaps& hidden_maps, const UpParams& hidden, const UpMaps& head_maps, const UpParams& head,
                                  int hidden_pairs, int sms, cudaStream_t st) {
    const int64_t units = (int64_t)(hidden.m + kTileM - 1) / kTileM * hidden.splits, tiles = tiles_of(head.m, head.n);
    const int64_t first = std::min<int64_t>(units, hidden_pairs), second = std::min<int64_t>(tiles, sms / 2 - first);
    return launch_chained(both_gradients_kernel, dim3((unsigned)(first + second) * 2), dim3(kThreads), kBothBytes, st, hidden_maps, hidden,
                          head_maps, head, (int)first);
}
cudaError_t launch_dhidden(const UpMaps& m, const UpParams& p, int sms, cudaStream_t st) {
    if (p.n <= kUpBothRows) return launch<true, false, kDense, kStore, true>(m, p, tiles_of(p.m, 1) * p.splits, sms, st);
    return launch<true, false, kDense, kStore>(m, p, tiles_of(p.m, p.n) * p.splits, sms, st);
}
cudaError_t launch_dhead(const UpMaps& m, const UpParams& p, int sms, cudaStream_t st) {
    if (in_parts(p.k)) return launch<true, true, kDense, kStoreRows, false, true>(m, p, tiles_of(p.m, p.n), sms, st);
    return launch<true, true, kDense, kStoreRows>(m, p, tiles_of(p.m, p.n), sms, st);
}
cudaError_t launch_expert_fwd(const UpMaps& m, const UpParams& p, int sms, cudaStream_t st) {
    if (in_parts(p.k)) return launch<false, false, kGroupRows, kStore, false, true>(m, p, sms, sms, st);
    return launch<false, false, kGroupRows, kStore>(m, p, sms, sms, st);
}
cudaError_t launch_expert_dx(const UpMaps& m, const UpParams& p, int sms, cudaStream_t st) {
    if (in_parts(p.k)) return launch<true, false, kGroupRows, kStore, false, true>(m, p, sms, sms, st);
    return launch<true, false, kGroupRows, kStore>(m, p, sms, sms, st);
}
cudaError_t launch_expert_dw(const UpMaps& m, const UpParams& p, int sms, cudaStream_t st) {
    if (in_parts(p.rows)) return launch<true, true, kGroupK, kStoreRows, false, true>(m, p, tiles_of(p.m, p.n) * p.experts, sms, st);
    return launch<true, true, kGroupK, kStoreRows>(m, p, tiles_of(p.m, p.n) * p.experts, sms, st);
}

// Parts of the d_hidden contraction (over the vocabulary piece, `stages` stages of 64): few rows give few units of
// work, and a piece is long, so it is cut until the units fill the pairs' rounds; at least 8 stages remain.  A part more
// costs the reading and writing of its fp32 sums, about 13 / stages of the contraction where that is bound by HBM.  Up to two tiles of rows the
// number of units is known; beyond, the live rows may be fewer than `rows`, and half a round is lost on average.
int dhidden_splits(int rows, int hidden, int stages, int slots) {
    const bool known = rows <= kUpBothRows;
    const int64_t units = (hidden + kTileM - 1) / kTileM * (known ? 1 : (rows + kTileN - 1) / kTileN);
    int best = 1;
    double best_fill = 0.;
    for (int s = 1; s <= 64 && (s == 1 || stages / s >= 8); ++s) {
        const double full = (double)(units * s) / (double)slots;
        const double fill = (known ? full / (double)((units * s + slots - 1) / slots) : full / (full + 0.5)) - std::min(0.01, 13. / stages) * s;
        if (fill > best_fill) { best_fill = fill; best = s; }
    }
    return best;
}

// --------------------------------------------------------------------------------- live rows and ends

constexpr int kLiveWarps = 8, kLiveThreads = 32 * kLiveWarps, kLiveHeld = 8;

// Copies the live rows side by side and takes each one's target logit as an fp32 dot product (the tensor cores'
// sums drop low bits on the way, always towards zero; a target that leads its row carries that error into its own
// log-prob in full).  The gradient's target entry is w (1 - p) = -w expm1(logp): from the caller's logp it keeps its relative
// accuracy at any p; without one logp is z / T - lse, and the rounding of lse, 2^-24 of its size, is an absolute error of
// 1 - p (at lse = 20 as large as a 1 - p of 1e-6 itself).  A warp takes a row; its pieces and those of the target's lm_head row, 2048 elements at a time, are
// requested together and before anything else is waited for (the lm_head row is a DRAM access of its own: one
// request after the other cost 19 us for 64 rows, now 6).  Meanwhile every block counts the live rows before its own
// (targets and weights are a few bytes per row and sit in L2), so one launch does the whole compaction, in order.
__global__ void __launch_bounds__(kLiveThreads) live_rows_kernel(LiveRows a) {
    __shared__ int counts[kLiveWarps], alive[kLiveWarps];
    pdl_wait();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int row0 = blockIdx.x * kLiveWarps, i = row0 + warp, pieces = a.H / 8;
    const bool exists = i < a.n;
    const int tgt = exists ? a.targets[i] : -1;
    const float weight = exists && a.weight ? a.weight[i] : 1.f;
    const bool live = tgt >= 0 && tgt < a.vocab && weight != 0.f;
    const uint4* src = reinterpret_cast<const uint4*>(a.hidden + (int64_t)(exists ? i : 0) * a.ld);
    const uint4* head = reinterpret_cast<const uint4*>(a.lm_head + (int64_t)(live ? tgt : 0) * a.H);
    uint4 x[kLiveHeld], w[kLiveHeld];
    const auto request = [&](int from) {
#pragma unroll
        for (int q = 0; q < kLiveHeld; ++q) {
            const int j = from + q * 32 + lane;
            x[q] = live && j < pieces ? src[j] : make_uint4(0, 0, 0, 0);
            w[q] = live && j < pieces && !a.logp_in ? head[j] : make_uint4(0, 0, 0, 0);
        }
    };
    request(0);
    int c = 0;
    for (int k = tid; k < row0; k += kLiveThreads) {
        const int t = a.targets[k];
        c += t >= 0 && t < a.vocab && (!a.weight || a.weight[k] != 0.f);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
    if (lane == 0) { counts[warp] = c; alive[warp] = live; }
    __syncthreads();
    int to = 0, total = 0;
#pragma unroll
    for (int q = 0; q < kLiveWarps; ++q) {
        to += counts[q] + (q < warp ? alive[q] : 0);
        total += counts[q] + alive[q];
    }
    const int64_t second = (int64_t)a.lo_rows * pieces;
    if (live) {
        uint4* dst = reinterpret_cast<uint4*>(a.rows + (int64_t)to * a.H);
        float dot = 0.f;
        for (int from = 0; from < pieces; from += kLiveHeld * 32) {
            if (from) request(from);
#pragma unroll
            for (int q = 0; q < kLiveHeld; ++q) {
                const int j = from + q * 32 + lane;
                if (j < pieces) {
                    dst[j] = x[q];
                    if (second) dst[second + j] = x[q];
                }
                const uint32_t xs[4] = {x[q].x, x[q].y, x[q].z, x[q].w}, ws[4] = {w[q].x, w[q].y, w[q].z, w[q].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    dot = fmaf(bf16_lo(xs[e]), bf16_lo(ws[e]), dot);
                    dot = fmaf(bf16_hi(xs[e]), bf16_hi(ws[e]), dot);
                }
            }
        }
        dot = warp_sum(dot);
        if (lane == 0) {
            a.src[to] = i;
            a.target[to] = tgt;
            a.target_logit[to] = dot;
            if (a.weight) {
                const float s = weight * a.inv_temp, l = a.lse_in[i];
                a.scaled[to] = s;
                a.lse[to] = l;
                a.target_d[to] = -s * expm1f(a.logp_in ? a.logp_in[i] : fmaf(dot, a.inv_temp, -l));
            }
        }
    } else if (exists) {
        if (lane == 0) {
            if (a.logp_out) { a.logp_out[i] = 0.f; a.lse_out[i] = 0.f; }
            if (tgt >= a.vocab) atomicOr(a.err, kErrBadToken);
        }
        if (a.d_hidden)
            for (int j = lane; j < pieces; j += 32) reinterpret_cast<uint4*>(a.d_hidden + (int64_t)i * a.ld_d)[j] = make_uint4(0, 0, 0, 0);
        // the k-th row that is not live clears compact row n - 1 - k, so that all rows from the last live one to n are
        // zeros: they are contraction indexes of d_lm_head (the last block clears what is left up to the padding)
        uint4* dst = reinterpret_cast<uint4*>(a.rows) + (int64_t)(a.n - 1 - (i - to)) * pieces;
        for (int j = lane; j < pieces; j += 32) {
            dst[j] = make_uint4(0, 0, 0, 0);
            if (second) dst[second + j] = make_uint4(0, 0, 0, 0);
        }
    }
    if (blockIdx.x == gridDim.x - 1) {
        if (tid == 0) *a.n_live = total;
        const int pad = a.lo_rows ? a.lo_rows : (a.n + 15) & ~15;
        for (int64_t j = (int64_t)a.n * pieces + tid; j < (int64_t)pad * pieces; j += kLiveThreads) {
            reinterpret_cast<uint4*>(a.rows)[j] = make_uint4(0, 0, 0, 0);
            if (second) reinterpret_cast<uint4*>(a.rows)[second + j] = make_uint4(0, 0, 0, 0);
        }
    }
}

cudaError_t launch_live_rows(const LiveRows& r, cudaStream_t st) {
    const int blocks = (r.n + kLiveWarps - 1) / kLiveWarps;
    return launch_chained(live_rows_kernel, dim3(blocks < 1 ? 1 : blocks), dim3(kLiveThreads), 0, st, r);
}

// One warp joins a row's (largest logit, sum of the others' exp) of all column tiles with its target's logit z:
// l = log(exp(z / T) + sum), logp = z / T - l, both taken from the larger of z and the maximum; where the target leads,
// logp = -log1p(sum exp(M - z)) keeps its relative accuracy down to probabilities next to 1.
__global__ void __launch_bounds__(256) logprob_finish_kernel(const float2* stats, int tiles, const float* zt, const int32_t* src,
                                                             const int32_t* n_live, float inv_temp, float* logp, float* lse) {
    pdl_wait();
    const int r = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (r >= *n_live) return;
    const float2* row = stats + (int64_t)r * tiles;
    const float scale = inv_temp * 1.4426950408889634f;
    float mx = -INFINITY;
    for (int i = lane; i < tiles; i += 32) mx = fmaxf(mx, row[i].x);
    mx = warp_max(mx);
    const float ref = mx == -INFINITY ? 0.f : mx;
    float sum = 0.f;
    for (int i = lane; i < tiles; i += 32) {
        const float2 v = row[i];
        sum += v.y * exp2_approx((v.x - ref) * scale);
    }
    sum = warp_sum(sum);
    if (lane == 0) {
        const float z = zt[r];
        float l, lp;
        if (z >= ref || mx == -INFINITY) {
            const float x = log1pf(sum * exp2_approx((mx - z) * scale));
            l = fmaf(z, inv_temp, x);
            lp = -x;
        } else {
            const float x = logf(sum + exp2_approx((z - mx) * scale));
            l = fmaf(mx, inv_temp, x);
            lp = (z - mx) * inv_temp - x;
        }
        lse[src[r]] = l;
        logp[src[r]] = lp;
    }
}

cudaError_t launch_logprob_finish(const float2* stats, int tiles, const float* target_logit, const int32_t* src,
                                  const int32_t* n_live, int n, float inv_temp, float* logp, float* lse, cudaStream_t st) {
    return launch_chained(logprob_finish_kernel, dim3((n + 7) / 8), dim3(256), 0, st, stats, tiles, target_logit, src, n_live,
                          inv_temp, logp, lse);
}

// d_hidden of the live rows: the splits' fp32 parts (and the second bf16 rows' share, lo_rows further) added in
// order, eight requests in flight, rounded once, scattered to the original rows.
__global__ void __launch_bounds__(256) dhidden_finish_kernel(const float* parts, int n_parts, int64_t split_stride, int64_t lo_stride,
                                                             const int32_t* src, const int32_t* n_live, int H,
                                                             __nv_bfloat16* out, int64_t ld) {
    pdl_wait();
    const int r = blockIdx.x, j = (blockIdx.y * 256 + threadIdx.x) * 4;
    if (r >= *n_live || j >= H) return;
    const float* p = parts + (int64_t)r * H + j;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = 0; s0 < n_parts; s0 += 8) {
        float4 w[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const int s = s0 + q;
            w[q] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (s < n_parts) w[q] = *reinterpret_cast<const float4*>(p + (lo_stride ? (s >> 1) * split_stride + (s & 1) * lo_stride : s * split_stride));
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) { v.x += w[q].x; v.y += w[q].y; v.z += w[q].z; v.w += w[q].w; }
    }
    *reinterpret_cast<uint2*>(out + (int64_t)src[r] * ld + j) = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
}

cudaError_t launch_dhidden_finish(const float* parts, int splits, int64_t split_stride, int lo_rows, const int32_t* src,
                                  const int32_t* n_live, int n, int H, __nv_bfloat16* d_hidden, int64_t ld, cudaStream_t st) {
    return launch_chained(dhidden_finish_kernel, dim3(n, (H + 1023) / 1024), dim3(256), 0, st, parts, lo_rows ? 2 * splits : splits,
                          split_stride, (int64_t)lo_rows * H, src, n_live, H, d_hidden, ld);
}

}  // namespace mars
