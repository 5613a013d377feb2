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

// What the epilogue of a contraction does with its accumulator tile (row = TMEM lane).
struct UpEpilogue {
    // store: out[row][col], fp32 or bf16, optionally added to what is there
    void* out;
    int64_t ld;               // elements between rows of out
    int64_t split_stride;     // elements between the outputs of two splits of the contraction
    int out_f32, accumulate;
    // log-prob rows (compact, live rows only)
    const int32_t* target;    // vocabulary entry of every row
    const float* lse;         // log sum exp of every row (gradient)
    const float* weight;      // d loss / d logp / T of every row (gradient)
    float inv_temp;
    float2* stats;            // [row][tiles_n]: (largest logit, sum of exp((logit - largest) / T)) of a column tile
    float* target_logit;      // [row]
    __nv_bfloat16* dlogits;   // [row][ld] of one vocabulary piece
    int v0, vocab;            // first vocabulary entry of the piece, size of the vocabulary
};

// One contraction (or a family of them, one for each expert): C[m, n] = sum_k A(m, k) B(n, k).
struct UpParams {
    int m, n, k;              // extents; for expert products see below
    const int32_t* m_live;    // device counts that replace m / k where not null (live rows of a log-prob call)
    const int32_t* k_live;
    int splits;               // the contraction is cut into this many parts with outputs of their own
    const int32_t* expert_off;   // [experts + 1], device: groups of rows (expert products)
    int experts, rows;        // rows: extent of the row axis that the offsets refer to
    int32_t* err;
    UpEpilogue e;
};

cudaError_t init_update_kernels();

// tensor maps: K-major operands have boxes of 64 x 128 rows, MN-major operands boxes of 64 x 64 rows
cudaError_t launch_logit_stats(const CUtensorMap& h, const CUtensorMap& w, const UpParams& p, int sms, cudaStream_t st);
cudaError_t launch_dlogits(const CUtensorMap& h, const CUtensorMap& w, const UpParams& p, int sms, cudaStream_t st);
cudaError_t launch_dhidden(const CUtensorMap& d, const CUtensorMap& w, const UpParams& p, int sms, cudaStream_t st);
cudaError_t launch_dhead(const CUtensorMap& d, const CUtensorMap& h, const UpParams& p, int sms, cudaStream_t st);
cudaError_t launch_expert_fwd(const CUtensorMap& x, const CUtensorMap& w, const UpParams& p, int sms, cudaStream_t st);
cudaError_t launch_expert_dx(const CUtensorMap& dy, const CUtensorMap& w, const UpParams& p, int sms, cudaStream_t st);
cudaError_t launch_expert_dw(const CUtensorMap& dy, const CUtensorMap& x, const UpParams& p, int sms, cudaStream_t st);
int dhidden_splits(int rows, int hidden, int stages, int sms);

// Live rows of a log-prob call: those with a target (and, for the gradient, a non-zero weight).
struct LiveRows {
    const __nv_bfloat16* hidden;   // [n][ld]
    int64_t ld;
    const int32_t* targets;
    const float* weight;           // null: forward
    const float* lse_in;           // gradient: [n]
    int n, H, vocab;
    float inv_temp;
    __nv_bfloat16* rows;           // [padded][H] compact copies, zeroed behind the last one up to a multiple of kUpTile
    int32_t *src, *target, *n_live;   // compact: original row, target
    float *lse, *scaled;           // compact: lse, weight / T
    float *logp_out, *lse_out;     // forward: 0 for rows without a target
    __nv_bfloat16* d_hidden;       // gradient: zeroed for rows that are not live
    int64_t ld_d;
    int32_t* err;
};
cudaError_t launch_live_rows(const LiveRows& r, cudaStream_t st);
cudaError_t launch_logprob_finish(const float2* stats, int tiles, int tiles_ld, const float* target_logit, const int32_t* src,
                                  const int32_t* n_live, int n, float inv_temp, float* logp, float* lse, cudaStream_t st);
cudaError_t launch_dhidden_finish(const float* parts, int splits, int64_t split_stride, const int32_t* src,
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
                             float max_norm, float* norm_out, float* scale, int blocks, cudaStream_t st);
cudaError_t launch_grad_scale(const GradEntry* table, int n_tensors, int64_t n_chunks, const float* scale, int blocks,
                              cudaStream_t st);
int64_t grad_chunks(const void* src, int64_t numel, int type);
int grad_blocks(int sms);

}  // namespace mars
