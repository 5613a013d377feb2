// Host-side declarations of the kernels of a training pass: norms (kernels_norm.cu), rotation of heads by their positions
// (kernels_rope.cu), the mixture's router with its losses (kernels_router.cu), policy loss (kernels_policy.cu).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace mars {

// A call's first launch is an ordinary one: the grid starts when the work before it on the stream is done.  The kernels are loaded when
// a handle is created (init_*_kernels), not at a first launch among other work.
template <typename... Params, typename... Args>
inline cudaError_t launch_plain(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<Args&&>(args)...);
}
// Launch of the second kernel of a call: its blocks may start while the first one, an ordinary launch of the same call, drains.  All of its threads
// pass pdl_wait() before they read what the first kernel writes, and before they write.
template <typename... Params, typename... Args>
inline cudaError_t launch_second(void (*kernel)(Params...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, Args&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<Args&&>(args)...);
}
// Loads kernels, and lets them use up to `smem` bytes of dynamic shared memory where that is more than they may anyway.
template <typename... K>
inline cudaError_t init_all(int smem, K... kernels) {
    cudaError_t e = cudaSuccess;
    cudaFuncAttributes attr;
    ((e = e != cudaSuccess ? e
          : smem > 0       ? cudaFuncSetAttribute((const void*)kernels, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)
                           : cudaFuncGetAttributes(&attr, (const void*)kernels)),
     ...);
    return e;
}
cudaError_t init_norm_kernels();
cudaError_t init_rope_kernels();
cudaError_t init_router_kernels();
cudaError_t init_policy_kernels();

constexpr int kTrainSms = 148;               // SMs for which workspaces are laid out; grids take no more
constexpr int kNormMaxWidth = 8192;
constexpr int kRouterMaxExperts = 1024, kRouterMaxK = 32;
constexpr int kPolicyStats = 6;

// ------------------------------------------------------------------------------------------------- norms
// A row is [width] elements at t * ld + h * width, t = row / heads, h = row % heads.
// Inputs that a call leaves out have a flag, and a pointer that is valid all the same (to another input): a load that the compiler moves
// ahead of its condition then meets memory.
struct NormArgs {
    int rows, heads, width, layer;           // rows = n * heads; layer: 1 = mean and bias, 0 = root mean square
    float eps;
    int w_type, has_add, has_bias;
    const void *x, *add, *weight, *bias;
    void *sum, *y;                           // sum: null or x + add, in x's type
    int64_t ld_x, ld_add, ld_sum, ld_y;
    float *mean, *rstd;                      // null or [rows]
};
struct NormGradArgs {
    int rows, heads, width, layer, w_type, has_d_sum;
    const void *dy, *x, *weight, *d_sum;
    void* dx;
    int64_t ld_dy, ld_x, ld_d_sum, ld_dx;
    const float *mean, *rstd;
    float *part_w, *part_b;                  // null or [blocks][width]
};
// vector: every row of every operand starts on a 16-byte boundary and has whole 16-byte pieces.
cudaError_t launch_norm(const NormArgs& a, int x_type, int y_type, bool vector, int sms, cudaStream_t st);
cudaError_t launch_norm_grad(const NormGradArgs& a, int x_type, int y_type, bool vector, int sms, void* dw, void* db, int dw_type,
                             int accumulate, cudaStream_t st);
size_t norm_grad_part_bytes(int max_width);

// ---------------------------------------------------------------------------------------------- rotation
struct RopeArgs {
    int tokens, head_dim, rotary, interleaved;
    float scale, sign;                       // sign: -1 turns back
    const int32_t* positions;
    const double* turns;                     // [rotary / 2] turns for one position
    const void* in[2];                       // q and k
    void* out[2];
    int64_t ld_in[2], ld_out[2];
    int heads[2];
};
cudaError_t launch_rope(const RopeArgs& a, int type, bool vector, int sms, cudaStream_t st);

// ------------------------------------------------------------------------------------------------ router
struct RouterArgs {
    int rows, experts, top_k, renormalise;
    const void* logits;
    int64_t ld;
    const uint8_t* live;                     // [rows] where has_live
    int has_live;
    int32_t* idx;                            // [rows][k]
    float *weights, *lse;                    // [rows][k], null or [rows]
    int32_t *counts, *offsets;               // null or [experts], [experts + 1]
    float *prob_sums, *losses;               // null or [experts], [2]
    int32_t* work_counts;                    // [experts], zero between calls
    float* parts;                            // [blocks][experts]
    double* z_parts;                         // [blocks]
    int32_t* ticket;                         // zero between calls
};
struct RouterGradArgs {
    int rows, experts, top_k, renormalise;
    const void* logits;
    int64_t ld;
    const int32_t *idx, *counts;
    const float *lse, *d_weights;            // [rows], [rows][k] where has_d_weights
    int has_d_weights;
    float balance, z;
    void* d_logits;
    int64_t ld_d;
};
cudaError_t launch_router(const RouterArgs& a, int type, bool vector, int sms, cudaStream_t st);
cudaError_t launch_router_grad(const RouterGradArgs& a, int type, bool vector, int sms, cudaStream_t st);
int router_max_blocks(int sms);

// ------------------------------------------------------------------------------------------- policy loss
struct PolicyArgs {
    int tokens, seqs, reduce, per_token;     // reduce: MARS_MEAN_TOKENS, MARS_MEAN_SEQUENCES, MARS_SUM
    int has_ref, vector;                     // vector: every array of a value for each token starts on a 16-byte boundary
    const float *lp, *old_lp, *ref, *adv;
    const int32_t *targets, *seq_off;
    double log_low, log_high;                // borders of log r
    float low, high, kl;                     // borders of r, KL coefficient
    double scale;
    float *stats, *d_lp;                     // d_lp: may be null
    int32_t* seq_live;                       // [seqs] live tokens, zero between calls
    int32_t* totals;                         // [0] live tokens, [1] sequences with one, zero between calls
    double* parts;                           // [blocks][4]
    int32_t* ticket;                         // zero between calls
};
cudaError_t launch_policy_loss(const PolicyArgs& a, int sms, cudaStream_t st);
int policy_max_blocks(int sms);

}  // namespace mars
