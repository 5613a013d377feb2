// Host side of the policy-update operators: argument checks, workspace layout, launch sequence.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "api_common.h"
#include "step.h"
#include "update.h"

using namespace mars;

namespace {

// The gradient of the logits is held for one vocabulary piece at a time: this many bytes of bf16, or 2048 entries of every
// row where that is more (above 131072 rows; 4 GB at 2^20).  Wide pieces mean few passes over the fp32 sums of d_hidden (one
// read and write of rows x hidden per piece).
constexpr size_t kPieceBytes = (size_t)512 << 20;
constexpr int kMinPiece = 2048;

struct Layout {
    int n, H, V, piece, pieces, splits;
    int64_t rows;              // n rounded up to the tile
};

Layout make_update_layout(int H, int V, int n, int sms) {
    Layout l;
    l = Layout{};
    l.n = n; l.H = H; l.V = V; l.splits = 1;
    if (n == 0) return l;             // a handle without an lm_head
    l.rows = (int64_t)align_up((size_t)n, kUpTile);
    const int64_t most = std::max<int64_t>(kMinPiece, (int64_t)(kPieceBytes / 2 / (size_t)l.rows) / kUpTile * kUpTile);
    const int64_t tiles = (V + kUpTile - 1) / kUpTile, per = std::max<int64_t>(1, most / kUpTile);
    l.pieces = (int)((tiles + per - 1) / per);
    l.piece = (int)((tiles + l.pieces - 1) / l.pieces) * kUpTile;
    l.splits = dhidden_splits(n, H, l.piece / 64, sms / 2);
    return l;
}

// K-major operand: `rows` rows of `inner` contraction indexes; boxes of 64 x box_rows.
mars_status_t map_k(CUtensorMap* tm, const void* p, uint64_t inner, uint64_t rows, uint64_t ld, uint32_t box_rows = 128) {
    const cuuint64_t dims[2] = {inner, rows}, strides[1] = {ld * 2};
    const cuuint32_t box[2] = {64u, box_rows};
    return make_tiled_map(tm, p, 2, dims, strides, box);
}
// The rows of a K-major B operand in boxes of 16, 32, 64 and 128, as far as a call of `most` rows can use them: one tile
// of up to 256 rows, of which each CTA loads half.
mars_status_t map_rows(UpMaps* m, const void* p, uint64_t inner, uint64_t rows, uint64_t ld, int64_t most) {
    const int64_t half = most > 256 ? 128 : (most + 31) / 32 * 16;
    for (int i = 0; i < 4 && (16 << i) <= half; ++i) {
        const mars_status_t s = map_k(&m->b[i], p, inner, rows, ld, 16u << i);
        if (s != MARS_OK) return s;
    }
    return MARS_OK;
}
// MN-major operand: `rows` contraction indexes of `inner` columns; boxes of 64 x 64.
mars_status_t map_mn(CUtensorMap* tm, const void* p, uint64_t inner, uint64_t rows, uint64_t ld) {
    return map_k(tm, p, inner, rows, ld, 64u);
}
// Stack of expert matrices [experts][rows][inner]: the third coordinate keeps a box inside its expert.
mars_status_t map_stack(CUtensorMap* tm, const void* p, uint64_t inner, uint64_t rows, uint64_t experts, uint32_t box_rows) {
    const cuuint64_t dims[3] = {inner, rows, experts}, strides[2] = {inner * 2, inner * rows * 2};
    const cuuint32_t box[3] = {64u, box_rows, 1u};
    return make_tiled_map(tm, p, 3, dims, strides, box);
}

// The sizes of a handle's workspace do not depend on the device: laid out for the splits of d_hidden that 148 SMs and
// max_tokens rows call for; a call takes as many as its own rows leave room for.
constexpr int kPlanSms = 148;

}  // namespace

struct mars_update {
    int device, sms;
    Layout l;
    int32_t* err;
    __nv_bfloat16 *rows, *dlogits;
    float* parts;
    float2* stats;
    float *target_logit, *lse, *scaled, *target_d;
    int32_t *src, *target, *n_live;
};

struct mars_grads {
    int device, sms, n;
    int64_t chunks;
    GradEntry* table;
    double* partials;
    int32_t* ticket;
    double* scale;
};

namespace {

size_t carve_update(const Layout& l, unsigned char* base, mars_update* u) {
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at = align_up(at + bytes, 256); return base ? base + o : nullptr; };
    mars_update t{};
    t.err = (int32_t*)take(256);
    t.n_live = (int32_t*)take(256);
    if (l.n > 0) {
        const size_t R = (size_t)l.rows, tiles = ((size_t)l.V + kUpTile - 1) / kUpTile;
        t.src = (int32_t*)take(R * 4);
        t.target = (int32_t*)take(R * 4);
        t.target_logit = (float*)take(R * 4);
        t.lse = (float*)take(R * 4);
        t.scaled = (float*)take(R * 4);
        t.target_d = (float*)take(R * 4);
        t.rows = (__nv_bfloat16*)take(R * l.H * 2);
        // the forward's statistics and the gradient's pieces are never alive together
        const size_t stats = R * tiles * 16, grads = align_up(R * l.piece * 2, 256) + (size_t)l.splits * R * l.H * 4;
        unsigned char* shared = take(std::max(stats, grads));
        t.stats = (float2*)shared;
        t.dlogits = (__nv_bfloat16*)shared;
        t.parts = base ? (float*)(shared + align_up(R * l.piece * 2, 256)) : nullptr;
    }
    if (u) {
        u->err = t.err; u->n_live = t.n_live; u->src = t.src; u->target = t.target; u->target_logit = t.target_logit;
        u->lse = t.lse; u->scaled = t.scaled; u->target_d = t.target_d; u->rows = t.rows; u->stats = t.stats; u->dlogits = t.dlogits; u->parts = t.parts;
    }
    return at;
}

bool update_shape_ok(int32_t hidden, int32_t vocab, int32_t max_tokens) {
    if (hidden == 0 && vocab == 0 && max_tokens == 0) return true;
    return hidden >= 8 && hidden % 8 == 0 && hidden <= (1 << 20) && vocab >= 1 && vocab <= (1 << 30) && max_tokens >= 1 &&
           max_tokens <= (1 << 20);
}

mars_status_t check_logprob(const mars_update* u, int32_t n, const void* hidden, int64_t ld, const void* lm_head,
                            const int32_t* targets, float temperature) {
    if (!u) return MARS_ERR_BAD_HANDLE;
    // the kernels scale logits by log2(e) / T: an infinite factor would make the largest logit's 0 x inf a NaN
    if (u->l.n < 1 || n < 0 || n > u->l.n || !(temperature > 0.f) || !std::isfinite(temperature) ||
        !std::isfinite(1.f / temperature * 1.4426950408889634f)) return MARS_ERR_INVALID_ARG;
    if (!lm_head || !aligned16(lm_head)) return MARS_ERR_INVALID_ARG;
    if (n > 0 && (!hidden || !targets || !aligned16(hidden) || !aligned4(targets) || ld < u->l.H || ld % 8))
        return MARS_ERR_INVALID_ARG;
    return MARS_OK;
}

mars_status_t check_experts(const mars_update* u, int32_t E, int32_t rows, int32_t d_in, int32_t d_out, const void* rows_in,
                            int64_t ld_in, int64_t cols_in, const int32_t* off) {
    if (!u) return MARS_ERR_BAD_HANDLE;
    // at most 2^30 of anything: extents are rounded up to tiles and stages in 32 bits
    if (E < 1 || E > kUpMaxExperts || rows < 0 || rows > (1 << 30) || d_in < 8 || d_out < 8 || d_in > (1 << 30) || d_out > (1 << 30) ||
        d_in % 8 || d_out % 8) return MARS_ERR_INVALID_ARG;
    if (!off || (uintptr_t)off % 4) return MARS_ERR_INVALID_ARG;
    if (rows > 0 && (!rows_in || !aligned16(rows_in) || ld_in < cols_in || ld_in % 8)) return MARS_ERR_INVALID_ARG;
    return MARS_OK;
}
size_t out_bytes(int type) { return type == MARS_F32 ? 4 : 2; }
// Output stack [matrices][rows][columns]: boxes of 128 bytes x 32 rows of one matrix.
mars_status_t map_out(CUtensorMap* tm, void* p, uint64_t columns, uint64_t rows, uint64_t matrices, int type) {
    const uint64_t eb = out_bytes(type);
    const cuuint64_t dims[3] = {columns, rows, matrices}, strides[2] = {columns * eb, columns * rows * eb};
    const cuuint32_t box[3] = {(cuuint32_t)(128 / eb), 32u, 1u};
    return make_tiled_map(tm, p, 3, dims, strides, box, type == MARS_F32);
}

}  // namespace

extern "C" {

size_t mars_update_workspace_bytes(int32_t hidden, int32_t vocab, int32_t max_tokens) {
    if (!update_shape_ok(hidden, vocab, max_tokens)) return 0;
    return carve_update(make_update_layout(hidden, vocab, max_tokens, kPlanSms), nullptr, nullptr);
}

mars_status_t mars_update_create(int32_t hidden, int32_t vocab, int32_t max_tokens, void* workspace, size_t workspace_bytes,
                                 mars_update_t** out) {
    if (!workspace || !out || (uintptr_t)workspace % 256) return MARS_ERR_INVALID_ARG;
    if (!update_shape_ok(hidden, vocab, max_tokens)) return MARS_ERR_UNSUPPORTED;
    const Layout l = make_update_layout(hidden, vocab, max_tokens, kPlanSms);
    if (workspace_bytes < carve_update(l, nullptr, nullptr)) return MARS_ERR_INVALID_ARG;
    int dev = 0, sms = 0;
    RUN(device_info(&dev, &sms));
    RUN(launched(init_update_kernels()));
    mars_update* u = new (std::nothrow) mars_update();
    if (!u) return MARS_ERR_INVALID_ARG;
    u->device = dev; u->sms = sms; u->l = l;
    carve_update(l, (unsigned char*)workspace, u);
    // cudaMemset returns before the memory is set, and a non-blocking stream does not wait for it
    cudaError_t e = cudaMemset(u->err, 0, 512);
    if (e == cudaSuccess) e = cudaStreamSynchronize(cudaStreamLegacy);
    if (e != cudaSuccess) { delete u; return launched(e); }
    *out = u;
    return MARS_OK;
}

mars_status_t mars_update_free(mars_update_t* u) {
    if (!u) return MARS_ERR_BAD_HANDLE;
    delete u;
    return MARS_OK;
}

mars_status_t mars_update_poll_status(mars_update_t* u) {
    if (!u) return MARS_ERR_BAD_HANDLE;
    const DeviceGuard guard(u->device);
    if (!guard.ok) return MARS_ERR_CUDA;
    // the streams of the calls are not all known here: a captured call runs on whatever stream its graph is replayed on
    CUDA_TRY(cudaDeviceSynchronize());
    int32_t word = 0;
    CUDA_TRY(cudaMemcpy(&word, u->err, 4, cudaMemcpyDeviceToHost));
    if (word) {
        CUDA_TRY(cudaMemset(u->err, 0, 4));
        CUDA_TRY(cudaStreamSynchronize(cudaStreamLegacy));       // else it could clear a later call's report
    }
    if (word & kErrTimeout) return MARS_ERR_TIMEOUT;
    if (word & kErrBadToken) return MARS_ERR_BAD_TOKEN;
    return MARS_OK;
}

mars_status_t mars_logprob(mars_update_t* u, void* cuda_stream, int32_t n, const void* hidden, int64_t ld, const void* lm_head,
                           const int32_t* targets, float temperature, float* out_logprobs, float* out_lse) {
    RUN(check_logprob(u, n, hidden, ld, lm_head, targets, temperature));
    if (n == 0) return MARS_OK;
    if (!out_logprobs || !out_lse || !aligned4(out_logprobs) || !aligned4(out_lse)) return MARS_ERR_INVALID_ARG;
    const Layout& l = u->l;
    const size_t in_h = span(n, ld, l.H, 2), in_w = (size_t)l.V * l.H * 2, nb = (size_t)n * 4;
    for (const float* o : {out_logprobs, out_lse})
        if (overlap(o, nb, hidden, in_h) || overlap(o, nb, lm_head, in_w) || overlap(o, nb, targets, nb)) return MARS_ERR_INVALID_ARG;
    if (overlap(out_logprobs, nb, out_lse, nb)) return MARS_ERR_INVALID_ARG;
    const DeviceGuard guard(u->device);
    if (!guard.ok) return MARS_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    UpMaps maps{};
    RUN(map_k(&maps.a, lm_head, l.H, l.V, l.H));
    RUN(map_rows(&maps, u->rows, l.H, l.rows, l.H, n));

    LiveRows r{};
    r.hidden = (const __nv_bfloat16*)hidden; r.ld = ld; r.lm_head = (const __nv_bfloat16*)lm_head; r.targets = targets;
    r.n = n; r.H = l.H; r.vocab = l.V; r.inv_temp = 1.f / temperature;
    r.rows = u->rows; r.src = u->src; r.target = u->target; r.n_live = u->n_live; r.target_logit = u->target_logit;
    r.logp_out = out_logprobs; r.lse_out = out_lse; r.err = u->err;
    RUN(launched(launch_live_rows(r, st)));
    UpParams p{};
    p.m = l.V; p.n = n; p.k = l.H; p.n_live = u->n_live; p.splits = 1; p.n_block = update_n_block(l.H); p.err = u->err;
    p.e.target = u->target; p.e.inv_temp = 1.f / temperature; p.e.stats = u->stats;
    RUN(launched(launch_logit_stats(maps, p, u->sms, st)));
    return launched(launch_logprob_finish(u->stats, (l.V + 255) / 256 * 2, u->target_logit, u->src, u->n_live, n, 1.f / temperature,
                                          out_logprobs, out_lse, st));
}

mars_status_t mars_logprob_grad(mars_update_t* u, void* cuda_stream, int32_t n, const void* hidden, int64_t ld,
                                const void* lm_head, const int32_t* targets, float temperature, const float* lse,
                                const float* d_logprobs, void* d_hidden, int64_t ld_d, void* d_lm_head, int32_t d_type,
                                int32_t accumulate) {
    return mars_logprob_grad_lp(u, cuda_stream, n, hidden, ld, lm_head, targets, temperature, nullptr, lse, d_logprobs, d_hidden, ld_d,
                                d_lm_head, d_type, accumulate);
}

mars_status_t mars_logprob_grad_lp(mars_update_t* u, void* cuda_stream, int32_t n, const void* hidden, int64_t ld,
                                   const void* lm_head, const int32_t* targets, float temperature, const float* logprobs,
                                   const float* lse, const float* d_logprobs, void* d_hidden, int64_t ld_d, void* d_lm_head,
                                   int32_t d_type, int32_t accumulate) {
    RUN(check_logprob(u, n, hidden, ld, lm_head, targets, temperature));
    if (!d_lm_head || !aligned16(d_lm_head) || (d_type != MARS_BF16 && d_type != MARS_F32)) return MARS_ERR_INVALID_ARG;
    if (n > 0 && (!lse || !d_logprobs || !d_hidden || !aligned4(lse) || !aligned4(d_logprobs) || !aligned4(logprobs) ||
                   !aligned16(d_hidden) || ld_d < u->l.H || ld_d % 8)) return MARS_ERR_INVALID_ARG;
    const Layout& l = u->l;
    const size_t ow = (size_t)l.V * l.H * out_bytes(d_type), oh = span(n, ld_d, l.H, 2), nb = (size_t)n * 4;
    const struct { const void* p; size_t n; } ins[] = {{lm_head, (size_t)l.V * l.H * 2}, {targets, nb}, {lse, nb}, {d_logprobs, nb},
                                                       {logprobs, logprobs ? nb : 0}};
    for (const auto& i : ins)
        if (overlap(d_lm_head, ow, i.p, i.n) || overlap(d_hidden, oh, i.p, i.n)) return MARS_ERR_INVALID_ARG;
    if (overlap(d_lm_head, ow, hidden, span(n, ld, l.H, 2)) || rows_overlap(d_hidden, ld_d, l.H, 2, hidden, ld, l.H, 2, n))
        return MARS_ERR_INVALID_ARG;
    if (overlap(d_lm_head, ow, d_hidden, oh)) return MARS_ERR_INVALID_ARG;
    const DeviceGuard guard(u->device);
    if (!guard.ok) return MARS_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (n == 0) {
        if (!accumulate) CUDA_TRY(cudaMemsetAsync(d_lm_head, 0, ow, st));
        return MARS_OK;
    }
    // few rows: d as two bf16 rows each, the second ones behind the first; counts are then the padded ones
    const int lo = n <= kUpLoRows ? (int)align_up((size_t)n, 32) : 0;
    UpMaps logits{}, dhidden{}, dhead{};
    RUN(map_rows(&logits, u->rows, l.H, l.rows, l.H, lo ? lo : n));
    RUN(map_rows(&dhidden, u->dlogits, l.piece, l.rows, l.piece, lo ? 2 * lo : n));
    RUN(map_mn(&dhead.a, u->dlogits, l.piece, l.rows, l.piece));
    RUN(map_mn(&dhead.b[0], u->rows, l.H, l.rows, l.H));

    LiveRows r{};
    r.hidden = (const __nv_bfloat16*)hidden; r.ld = ld; r.lm_head = (const __nv_bfloat16*)lm_head; r.targets = targets;
    r.weight = d_logprobs; r.lse_in = lse; r.logp_in = logprobs;
    r.n = n; r.H = l.H; r.vocab = l.V; r.inv_temp = 1.f / temperature;
    r.rows = u->rows; r.lo_rows = lo; r.src = u->src; r.target = u->target; r.n_live = u->n_live;
    r.target_logit = u->target_logit; r.lse = u->lse; r.scaled = u->scaled; r.target_d = u->target_d;
    r.d_hidden = (__nv_bfloat16*)d_hidden; r.ld_d = ld_d; r.err = u->err;
    RUN(launched(launch_live_rows(r, st)));

    // as many parts of d_hidden as the rows of this call leave room for
    const int64_t rows_now = (int64_t)align_up((size_t)n, kUpTile), stride = rows_now * l.H;
    const int most_splits = (int)std::min<int64_t>(l.splits * l.rows / rows_now, 1 << 10), slots = u->sms / 2;
    const int beside = l.pieces == 1 ? both_hidden_pairs(n, l.V, l.H, slots) : 0;
    const int splits = std::min(most_splits, dhidden_splits(n, l.H, l.piece / 64, beside ? beside : slots));
    for (int i = 0; i < l.pieces; ++i) {
        const int v0 = i * l.piece;
        if (v0 >= l.V) break;
        const int width = std::min(l.piece, l.V - v0), padded = (int)align_up((size_t)width, kUpTile);
        const unsigned char* w_piece = (const unsigned char*)lm_head + (size_t)v0 * l.H * 2;
        RUN(map_k(&logits.a, w_piece, l.H, width, l.H));
        RUN(map_mn(&dhidden.a, w_piece, l.H, width, l.H));
        UpParams p{};
        p.m = padded; p.n = lo ? lo : n; p.k = l.H; p.n_live = lo ? nullptr : u->n_live; p.splits = 1; p.n_block = update_n_block(l.H); p.err = u->err;
        p.e.target = u->target; p.e.lse = u->lse; p.e.weight = u->scaled; p.e.target_d = u->target_d; p.e.n_live = u->n_live;
        p.e.inv_temp = 1.f / temperature;
        p.e.dlogits = u->dlogits; p.e.ld = l.piece; p.e.lo_rows = lo; p.e.v0 = v0; p.e.vocab = l.V;
        RUN(launched(launch_dlogits(logits, p, u->sms, st)));

        UpParams q{};
        q.m = l.H; q.n = lo ? 2 * lo : n; q.k = padded; q.n_live = lo ? nullptr : u->n_live; q.n_block = 1 << 20; q.err = u->err;
        q.e.out = u->parts; q.e.ld = l.H; q.e.split_stride = stride; q.e.out_f32 = 1; q.e.accumulate = i > 0;
        UpParams s{};
        s.m = width; s.n = l.H; s.k = lo ? 2 * lo : n; s.k_live = lo ? nullptr : u->n_live; s.splits = 1; s.n_block = 1 << 20; s.err = u->err;
        s.e.out = (unsigned char*)d_lm_head + (size_t)v0 * l.H * out_bytes(d_type);
        s.e.ld = l.H; s.e.out_f32 = d_type == MARS_F32; s.e.accumulate = accumulate != 0;
        s.e.bulk = !accumulate;
        if (s.e.bulk) RUN(map_out(&dhead.out, s.e.out, l.H, width, 1, d_type));
        q.splits = splits;
        if (beside) {
            RUN(launched(launch_both_gradients(dhidden, q, dhead, s, beside, u->sms, st)));
        } else {
            RUN(launched(launch_dhidden(dhidden, q, u->sms, st)));
            RUN(launched(launch_dhead(dhead, s, u->sms, st)));
        }
    }
    return launched(launch_dhidden_finish(u->parts, splits, stride, lo, u->src, u->n_live, n, l.H, (__nv_bfloat16*)d_hidden, ld_d, st));
}

mars_status_t mars_expert_matmul(mars_update_t* u, void* cuda_stream, int32_t E, int32_t rows, int32_t d_in, int32_t d_out,
                                 const void* x, int64_t ld_x, const int32_t* off, const void* w, void* y, int64_t ld_y,
                                 int32_t y_type) {
    RUN(check_experts(u, E, rows, d_in, d_out, x, ld_x, d_in, off));
    if (!w || !aligned16(w) || (y_type != MARS_BF16 && y_type != MARS_F32)) return MARS_ERR_INVALID_ARG;
    if (rows == 0) return MARS_OK;
    if (!y || !aligned16(y) || ld_y < d_out || ld_y % 8) return MARS_ERR_INVALID_ARG;
    const size_t oy = span(rows, ld_y, d_out, out_bytes(y_type));
    if (rows_overlap(y, ld_y, d_out, out_bytes(y_type), x, ld_x, d_in, 2, rows) || overlap(y, oy, w, (size_t)E * d_in * d_out * 2) ||
        overlap(y, oy, off, ((size_t)E + 1) * 4)) return MARS_ERR_INVALID_ARG;
    const DeviceGuard guard(u->device);
    if (!guard.ok) return MARS_ERR_CUDA;
    UpMaps maps{};
    RUN(map_stack(&maps.a, w, d_in, d_out, E, 128));
    RUN(map_rows(&maps, x, d_in, rows, ld_x, rows));
    UpParams p{};
    p.m = d_out; p.k = d_in; p.splits = 1; p.n_block = update_n_block(d_in); p.expert_off = off; p.experts = E; p.rows = rows; p.err = u->err;
    p.e.out = y; p.e.ld = ld_y; p.e.out_f32 = y_type == MARS_F32;
    return launched(launch_expert_fwd(maps, p, u->sms, (cudaStream_t)cuda_stream));
}

mars_status_t mars_expert_matmul_dx(mars_update_t* u, void* cuda_stream, int32_t E, int32_t rows, int32_t d_in, int32_t d_out,
                                    const void* dy, int64_t ld_dy, const int32_t* off, const void* w, void* dx, int64_t ld_dx,
                                    int32_t dx_type) {
    RUN(check_experts(u, E, rows, d_in, d_out, dy, ld_dy, d_out, off));
    if (!w || !aligned16(w) || (dx_type != MARS_BF16 && dx_type != MARS_F32)) return MARS_ERR_INVALID_ARG;
    if (rows == 0) return MARS_OK;
    if (!dx || !aligned16(dx) || ld_dx < d_in || ld_dx % 8) return MARS_ERR_INVALID_ARG;
    const size_t ox = span(rows, ld_dx, d_in, out_bytes(dx_type));
    if (rows_overlap(dx, ld_dx, d_in, out_bytes(dx_type), dy, ld_dy, d_out, 2, rows) || overlap(dx, ox, w, (size_t)E * d_in * d_out * 2) ||
        overlap(dx, ox, off, ((size_t)E + 1) * 4)) return MARS_ERR_INVALID_ARG;
    const DeviceGuard guard(u->device);
    if (!guard.ok) return MARS_ERR_CUDA;
    UpMaps maps{};
    RUN(map_stack(&maps.a, w, d_in, d_out, E, 64));
    RUN(map_rows(&maps, dy, d_out, rows, ld_dy, rows));
    UpParams p{};
    p.m = d_in; p.k = d_out; p.splits = 1; p.n_block = update_n_block(d_out); p.expert_off = off; p.experts = E; p.rows = rows; p.err = u->err;
    p.e.out = dx; p.e.ld = ld_dx; p.e.out_f32 = dx_type == MARS_F32;
    return launched(launch_expert_dx(maps, p, u->sms, (cudaStream_t)cuda_stream));
}

mars_status_t mars_expert_matmul_dw(mars_update_t* u, void* cuda_stream, int32_t E, int32_t rows, int32_t d_in, int32_t d_out,
                                    const void* dy, int64_t ld_dy, const void* x, int64_t ld_x, const int32_t* off, void* dw,
                                    int32_t dw_type, int32_t accumulate) {
    RUN(check_experts(u, E, rows, d_in, d_out, dy, ld_dy, d_out, off));
    if (rows > 0 && (!x || !aligned16(x) || ld_x < d_in || ld_x % 8)) return MARS_ERR_INVALID_ARG;
    if (!dw || !aligned16(dw) || (dw_type != MARS_BF16 && dw_type != MARS_F32)) return MARS_ERR_INVALID_ARG;
    const size_t ow = (size_t)E * d_in * d_out * out_bytes(dw_type);
    if (overlap(dw, ow, dy, span(rows, ld_dy, d_out, 2)) || overlap(dw, ow, x, span(rows, ld_x, d_in, 2)) ||
        overlap(dw, ow, off, ((size_t)E + 1) * 4)) return MARS_ERR_INVALID_ARG;
    const DeviceGuard guard(u->device);
    if (!guard.ok) return MARS_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (rows == 0) {
        if (!accumulate) CUDA_TRY(cudaMemsetAsync(dw, 0, ow, st));
        return MARS_OK;
    }
    UpMaps maps{};
    RUN(map_mn(&maps.a, dy, d_out, rows, ld_dy));
    RUN(map_mn(&maps.b[0], x, d_in, rows, ld_x));
    UpParams p{};
    p.m = d_out; p.n = d_in; p.splits = 1; p.n_block = 1 << 20; p.expert_off = off; p.experts = E; p.rows = rows; p.err = u->err;
    p.e.out = dw; p.e.ld = d_in; p.e.split_stride = (int64_t)d_in * d_out; p.e.out_f32 = dw_type == MARS_F32;
    p.e.accumulate = accumulate != 0; p.e.bulk = !accumulate;
    if (p.e.bulk) RUN(map_out(&maps.out, dw, d_in, d_out, E, dw_type));
    return launched(launch_expert_dw(maps, p, u->sms, st));
}

// ------------------------------------------------------------------------------------ gradient lists

static size_t grads_layout(int32_t n, size_t* partials, size_t* ticket) {
    size_t at = align_up((size_t)n * sizeof(GradEntry), 256);
    *partials = at;
    at = align_up(at + (size_t)grad_blocks(256) * sizeof(double), 256);      // room for any sm_100 part
    *ticket = at;
    return at + 256;
}

size_t mars_grads_bytes(int32_t n) {
    if (n < 1 || n > (1 << 20)) return 0;
    size_t a, b;
    return grads_layout(n, &a, &b);
}

mars_status_t mars_grads_create(const mars_grad_t* tensors, int32_t n, void* workspace, size_t workspace_bytes,
                                mars_grads_t** out) {
    if (!tensors || !workspace || !out || n < 1 || n > (1 << 20) || (uintptr_t)workspace % 256) return MARS_ERR_INVALID_ARG;
    size_t partials, ticket;
    if (workspace_bytes < grads_layout(n, &partials, &ticket)) return MARS_ERR_INVALID_ARG;
    try {
        struct Range { uintptr_t lo, hi; int tensor; bool out; };
        std::vector<GradEntry> table((size_t)n);
        std::vector<Range> ranges;
        ranges.reserve((size_t)n * 2);
        int64_t chunks = 0;
        for (int i = 0; i < n; ++i) {
            const mars_grad_t& t = tensors[i];
            if (t.numel < 0 || t.numel > ((int64_t)1 << 48) || (t.type != MARS_F32 && t.type != MARS_BF16 && t.type != MARS_F16))
                return MARS_ERR_INVALID_ARG;
            const size_t eb = t.type == MARS_F32 ? 4 : 2;
            if (t.numel > 0 && (!t.grad || !t.out || (uintptr_t)t.grad % eb || (uintptr_t)t.out % eb)) return MARS_ERR_INVALID_ARG;
            table[i] = GradEntry{t.grad, t.out, t.numel, chunks, t.type, 0};
            chunks += grad_chunks(t.grad, t.numel, t.type);
            if (t.numel > 0) {
                const size_t bytes = (size_t)t.numel * eb;
                if (t.grad != t.out) ranges.push_back(Range{(uintptr_t)t.grad, (uintptr_t)t.grad + bytes, i, false});
                ranges.push_back(Range{(uintptr_t)t.out, (uintptr_t)t.out + bytes, i, true});
            }
        }
        // an output must be alone in its memory (in place it stands for its gradient); gradients may be listed twice
        std::sort(ranges.begin(), ranges.end(), [](const Range& a, const Range& b) { return a.lo < b.lo; });
        uintptr_t hi_any = 0, hi_out = 0;
        for (const Range& r : ranges) {
            if (r.lo < hi_out || (r.out && r.lo < hi_any)) return MARS_ERR_INVALID_ARG;
            hi_any = std::max(hi_any, r.hi);
            if (r.out) hi_out = std::max(hi_out, r.hi);
        }
        int dev = 0, sms = 0;
        RUN(device_info(&dev, &sms));
        if (sms > 256) return MARS_ERR_UNSUPPORTED;
        unsigned char* base = (unsigned char*)workspace;
        CUDA_TRY(cudaMemcpy(base, table.data(), (size_t)n * sizeof(GradEntry), cudaMemcpyHostToDevice));
        CUDA_TRY(cudaMemset(base + ticket, 0, 256));
        CUDA_TRY(cudaStreamSynchronize(cudaStreamLegacy));       // a non-blocking stream does not wait for the two
        mars_grads* g = new (std::nothrow) mars_grads();
        if (!g) return MARS_ERR_INVALID_ARG;
        g->device = dev; g->sms = sms; g->n = n; g->chunks = chunks;
        g->table = (GradEntry*)base; g->partials = (double*)(base + partials);
        g->ticket = (int32_t*)(base + ticket); g->scale = (double*)(base + ticket + 64);
        *out = g;
        return MARS_OK;
    } catch (const std::bad_alloc&) {
        return MARS_ERR_INVALID_ARG;
    }
}

mars_status_t mars_grads_free(mars_grads_t* g) {
    if (!g) return MARS_ERR_BAD_HANDLE;
    delete g;
    return MARS_OK;
}

mars_status_t mars_grads_norm(mars_grads_t* g, void* cuda_stream, float* out_norm) {
    if (!g) return MARS_ERR_BAD_HANDLE;
    if (!out_norm || (uintptr_t)out_norm % 4) return MARS_ERR_INVALID_ARG;
    const DeviceGuard guard(g->device);
    if (!guard.ok) return MARS_ERR_CUDA;
    return launched(launch_grad_norm(g->table, g->n, g->chunks, g->partials, g->ticket, 0.f, out_norm, nullptr,
                                     grad_blocks(g->sms), (cudaStream_t)cuda_stream));
}

mars_status_t mars_grads_clip(mars_grads_t* g, void* cuda_stream, float max_norm, float* out_norm) {
    if (!g) return MARS_ERR_BAD_HANDLE;
    if (!out_norm || (uintptr_t)out_norm % 4 || !(max_norm >= 0.f)) return MARS_ERR_INVALID_ARG;
    const DeviceGuard guard(g->device);
    if (!guard.ok) return MARS_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    RUN(launched(launch_grad_norm(g->table, g->n, g->chunks, g->partials, g->ticket, max_norm, out_norm, g->scale,
                                  grad_blocks(g->sms), st)));
    return launched(launch_grad_scale(g->table, g->n, g->chunks, g->scale, grad_blocks(g->sms), st));
}

}  // extern "C"
