// Host-side declarations of the policy-update kernels: log-probability with its gradient, expert products with
// theirs (kernels_update.cu), gradient norm and clipping (kernels_grads.cu).
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace mars {

constexpr int kUpTile = 256;        // rows / columns by which workspace rows and vocabulary pieces are padded
constexpr int kUpMaxExperts = 1024;

constexpr int kUpBothRows = 512;    // two tiles of rows: d_hidden works on them as a pair
constexpr int kUpLoRows = 128;      // calls of at most this many rows keep d as two bf16 rows (see dlogits_tile)

// Tensor maps of a contraction's operands (bf16, 128-byte swizzle).  K-major: boxes of 64 contraction indexes x 128
// rows for A, x 16 << i rows for b[i]; MN-major: boxes of 64 contraction indexes x 64 columns (b[0] alone).
// out: [matrices][rows][columns] of an out[m][n] contraction, boxes of 128 bytes x 32 rows.
struct UpMaps {
    CUtensorMap a, b[4], out;
};

// What the epilogue of a contraction does with its accumulator tile (M index = TMEM lane).
struct UpEpilogue {
    // store: fp32 or bf16, optionally added to what is there
    void* out;
    int64_t ld;               // elements between rows of out (or of dlogits)
    int64_t split_stride;     // elements between the outputs of two splits of the contraction, or of two experts
    int out_f32, accumulate;
    int bulk;                 // out[m][n]: leaves by bulk copies through UpMaps::out (no accumulation)
    // log-prob rows (compact, live rows only)
    const int32_t* target;    // vocabulary entry of every row
    const float* lse;         // log sum exp of every row (gradient)
    const float* weight;      // d loss / d logp / T of every row (gradient)
    const float* target_d;    // gradient of the target's own logit
    const int32_t* n_live;    // rows that exist (gradient)
    float inv_temp;
    float2* stats;            // [row][2 tiles_m]: (largest logit, sum of exp((logit - largest) / T)) of 128 entries
    __nv_bfloat16* dlogits;   // [row][ld] of one vocabulary piece
    int lo_rows;              // not 0: distance of the second row that holds what the rounding took off
    int v0, vocab;            // first vocabulary entry of the piece, size of the vocabulary
};

// One contraction (or a family of them, one for each expert): sum_k A(m, k) B(n, k) as out[n][m], or out[m][n] for dw and
// d_lm_head.
struct UpParams {
    int m, n, k;
    const int32_t* n_live;    // device counts that replace n / k where not null (live rows of a log-prob call)
    const int32_t* k_live;
    int n_block;              // N tiles whose B is kept in L2 while the M tiles pass (see update_n_block)
    int splits;               // the contraction is cut into this many parts with outputs of their own
    const int32_t* expert_off;   // [experts + 1], device: groups of rows (expert products)
    int experts, rows;        // rows: extent of the row axis that the offsets refer to
    int32_t* err;
    UpEpilogue e;
};

// 32 MB of B rows of k elements, in tiles of 256.
inline int update_n_block(int64_t k) {
    const int64_t tiles = ((int64_t)32 << 20) / (512 * k);
    return (int)(tiles < 1 ? 1 : tiles > (1 << 20) ? 1 << 20 : tiles);
}

cudaError_t init_update_kernels();

cudaError_t launch_logit_stats(const UpMaps& m, const UpParams& p, int sms, cudaStream_t st);    // a = lm_head, b = rows
cudaError_t launch_dlogits(const UpMaps& m, const UpParams& p, int sms, cudaStream_t st);        // a = lm_head, b = rows
cudaError_t launch_dhidden(const UpMaps& m, const UpParams& p, int sms, cudaStream_t st);        // a = lm_head (MN), b = dlogits
cudaError_t launch_dhead(const UpMaps& m, const UpParams& p, int sms, cudaStream_t st);          // a = dlogits (MN), b = rows (MN)
cudaError_t launch_expert_fwd(const UpMaps& m, const UpParams& p, int sms, cudaStream_t st);     // a = w, b = x
cudaError_t launch_expert_dx(const UpMaps& m, const UpParams& p, int sms, cudaStream_t st);      // a = w (MN), b = dy
cudaError_t launch_expert_dw(const UpMaps& m, const UpParams& p, int sms, cudaStream_t st);      // a = dy (MN), b = x (MN)
// d_hidden and d_lm_head of a piece in one launch, where both_hidden_pairs is not 0
cudaError_t launch_both_gradients(const UpMaps& hidden_maps, const UpParams& hidden, const UpMaps& head_maps, const UpParams& head,
                                  int hidden_pairs, int sms, cudaStream_t st);
int both_hidden_pairs(int rows, int width, int hidden, int slots);
int dhidden_splits(int rows, int hidden, int stages, int slots);

// Live rows of a log-prob call: those with a target (and, for the gradient, a non-zero weight).
struct LiveRows {
    const __nv_bfloat16* hidden;   // [n][ld]
    int64_t ld;
    const __nv_bfloat16* lm_head;  // [vocab][H]
    const int32_t* targets;
    const float* weight;           // null: forward
    const float* lse_in;           // gradient: [n]
    const float* logp_in;          // gradient: [n] or null (1 - p of the target then comes from its logit and lse_in)
    int n, H, vocab;
    float inv_temp;
    __nv_bfloat16* rows;           // [padded][H] compact copies, zeros behind the last one up to n rounded up to 16 (or lo_rows)
    int lo_rows;                   // not 0: a second copy this many rows further, both zeroed up to there
    int32_t *src, *target, *n_live;   // compact: original row, target
    float *target_logit, *lse, *scaled, *target_d;   // compact: logit of the target, lse, weight / T, d of the target's logit
    float *logp_out, *lse_out;     // forward: 0 for rows without a target
    __nv_bfloat16* d_hidden;       // gradient: zeroed for rows that are not live
    int64_t ld_d;
    int32_t* err;
};
cudaError_t launch_live_rows(const LiveRows& r, cudaStream_t st);
cudaError_t launch_logprob_finish(const float2* stats, int tiles, const float* target_logit, const int32_t* src,
                                  const int32_t* n_live, int n, float inv_temp, float* logp, float* lse, cudaStream_t st);
cudaError_t launch_dhidden_finish(const float* parts, int splits, int64_t split_stride, int lo_rows, const int32_t* src,
                                  const int32_t* n_live, int n, int H, __nv_bfloat16* d_hidden, int64_t ld, cudaStream_t st);

// Gradient lists.
struct GradEntry {
    const void* src;
    void* dst;
    int64_t numel;
    int64_t first_chunk;    // chunks of the tensors before this one
    int32_t type, pad;
};
cudaError_t launch_grad_norm(const GradEntry* table, int n_tensors, int64_t n_chunks, double* partials, int32_t* ticket,
                             float max_norm, float* norm_out, double* scale, int blocks, cudaStream_t st);
cudaError_t launch_grad_scale(const GradEntry* table, int n_tensors, int64_t n_chunks, const double* scale, int blocks,
                              cudaStream_t st);
int64_t grad_chunks(const void* src, int64_t numel, int type);
int grad_blocks(int sms);

}  // namespace mars
