// Host side of the operators of a training pass: argument checks, workspace layout, launches.
#include <cmath>
#include <limits>
#include <new>

#include "api_common.h"
#include "train.h"

using namespace mars;

struct mars_train {
    int device, sms, max_width, max_experts, max_seqs;
    int32_t *tickets, *totals;       // [3]: router, policy loss (2); [2]
    int32_t *counts, *seq_live;      // zero between calls
    unsigned char* scratch;          // one call's partial sums
};

struct mars_rope_table {
    int device, sms, rotary, interleaved;
    float scale;
    const double* turns;
};

namespace {

constexpr int64_t kMaxLd = (int64_t)1 << 31;

size_t elem_bytes(int type) { return type == MARS_F32 ? 4 : 2; }
bool type_ok(int type) { return type == MARS_F32 || type == MARS_BF16 || type == MARS_F16; }
bool aligned_to(const void* p, size_t a) { return (uintptr_t)p % a == 0; }

size_t norm_scratch(int w) { return w ? 2 * align_up(norm_grad_part_bytes(w), 256) : 0; }
size_t router_scratch(int e) {
    const size_t blocks = (size_t)router_max_blocks(kTrainSms);
    return e ? align_up(blocks * e * 4, 256) + blocks * 8 : 0;
}
size_t policy_parts() { return align_up((size_t)policy_max_blocks(kTrainSms) * 4 * 8, 256); }
size_t policy_scratch(int s) { return s ? policy_parts() : 0; }

size_t carve_train(int w, int e, int s, unsigned char* base, mars_train* t) {
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at = align_up(at + bytes, 256); return base ? base + o : nullptr; };
    unsigned char* head = take(256);
    unsigned char *counts = take((size_t)e * 4), *live = take((size_t)s * 4);
    size_t most = norm_scratch(w);
    if (router_scratch(e) > most) most = router_scratch(e);
    if (policy_scratch(s) > most) most = policy_scratch(s);
    unsigned char* scratch = take(most);
    if (t) {
        t->tickets = (int32_t*)head; t->totals = (int32_t*)(head + 64);
        t->counts = (int32_t*)counts; t->seq_live = (int32_t*)live; t->scratch = scratch;
    }
    return at;
}
bool train_shape_ok(int32_t w, int32_t e, int32_t s) {
    return w >= 0 && w <= kNormMaxWidth && e >= 0 && e <= kRouterMaxExperts && s >= 0 && s <= (1 << 20) && (w || e || s);
}

// A matrix operand: rows of `cols` elements, `ld` elements apart.
struct Mat {
    const void* p;
    int64_t ld, cols;
    size_t elem;
};
bool mat_ok(const Mat& m, int64_t rows) {
    return rows == 0 || (m.p && aligned_to(m.p, m.elem) && m.ld >= m.cols && m.ld <= kMaxLd);
}
bool vector_ok(const Mat& m, size_t bytes = 16) { return aligned_to(m.p, bytes) && m.ld * (int64_t)m.elem % (int64_t)bytes == 0; }
// An output may take the place of an input, element for element, but share memory with it in no other way.
bool clash(const Mat& out, const Mat& in, int64_t rows, bool may_replace = true) {
    if (!out.p || !in.p || rows == 0) return false;
    if (may_replace && out.p == in.p && out.ld == in.ld && out.cols == in.cols && out.elem == in.elem) return false;
    return rows_overlap(out.p, out.ld, out.cols, out.elem, in.p, in.ld, in.cols, in.elem, rows);
}
bool clash(const Mat& m, int64_t rows, const void* p, size_t bytes) {
    return m.p && p && rows > 0 && overlap(m.p, span(rows, m.ld, m.cols, m.elem), p, bytes);
}
struct Flat {
    const void* p;
    size_t bytes;
};
bool overlap(const Flat& a, const Flat& b) { return a.p && b.p && mars::overlap(a.p, a.bytes, b.p, b.bytes); }
// No output among `out` shares memory with another or with one of `in`.
template <size_t N, size_t M>
bool flats_ok(const Flat (&out)[N], const Flat (&in)[M]) {
    for (size_t i = 0; i < N; ++i) {
        for (size_t j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return false;
        for (const Flat& f : in)
            if (overlap(out[i], f)) return false;
    }
    return true;
}

mars_status_t check_norm(const mars_train* t, const mars_norm_t* f, int32_t n_rows) {
    if (!t) return MARS_ERR_BAD_HANDLE;
    if (!f || n_rows < 0) return MARS_ERR_INVALID_ARG;
    if ((f->kind != MARS_NORM_RMS && f->kind != MARS_NORM_LAYER) || !type_ok(f->x_type) || !type_ok(f->y_type) || !type_ok(f->w_type))
        return MARS_ERR_INVALID_ARG;
    if (f->x_type != f->y_type && f->x_type != MARS_F32) return MARS_ERR_UNSUPPORTED;
    if (f->width < 1 || f->width > t->max_width || f->heads < 1 || (int64_t)f->heads * f->width > (1 << 30) ||
        (int64_t)n_rows * f->heads > INT32_MAX || !(f->eps > 0.f) || !std::isfinite(f->eps)) return MARS_ERR_INVALID_ARG;
    return MARS_OK;
}

}  // namespace

extern "C" {

size_t mars_train_workspace_bytes(int32_t max_width, int32_t max_experts, int32_t max_seqs) {
    if (!train_shape_ok(max_width, max_experts, max_seqs)) return 0;
    return carve_train(max_width, max_experts, max_seqs, nullptr, nullptr);
}

mars_status_t mars_train_create(int32_t max_width, int32_t max_experts, int32_t max_seqs, void* workspace, size_t workspace_bytes,
                                mars_train_t** out) {
    if (!workspace || !out || (uintptr_t)workspace % 256) return MARS_ERR_INVALID_ARG;
    if (!train_shape_ok(max_width, max_experts, max_seqs)) return MARS_ERR_UNSUPPORTED;
    if (workspace_bytes < carve_train(max_width, max_experts, max_seqs, nullptr, nullptr)) return MARS_ERR_INVALID_ARG;
    int dev = 0, sms = 0;
    RUN(device_info(&dev, &sms));
    if (max_width) RUN(launched(init_norm_kernels()));
    if (max_experts) RUN(launched(init_router_kernels()));
    if (max_seqs) RUN(launched(init_policy_kernels()));
    mars_train* t = new (std::nothrow) mars_train();
    if (!t) return MARS_ERR_INVALID_ARG;
    t->device = dev; t->sms = sms < kTrainSms ? sms : kTrainSms;
    t->max_width = max_width; t->max_experts = max_experts; t->max_seqs = max_seqs;
    carve_train(max_width, max_experts, max_seqs, (unsigned char*)workspace, t);
    // everything ahead of the scratch area starts at zero, on whatever stream the first call comes
    cudaError_t e = cudaMemset(workspace, 0, (size_t)(t->scratch - (unsigned char*)workspace));
    if (e == cudaSuccess) e = cudaStreamSynchronize(cudaStreamLegacy);
    if (e != cudaSuccess) { delete t; return launched(e); }
    *out = t;
    return MARS_OK;
}

mars_status_t mars_train_free(mars_train_t* t) {
    if (!t) return MARS_ERR_BAD_HANDLE;
    delete t;
    return MARS_OK;
}

// ------------------------------------------------------------------------------------------------- norms

mars_status_t mars_norm(mars_train_t* t, void* cuda_stream, const mars_norm_t* f, int32_t n_rows, const void* x, int64_t ld_x,
                        const void* add, int64_t ld_add, void* sum, int64_t ld_sum, const void* weight, const void* bias, void* y,
                        int64_t ld_y, float* mean, float* rstd) {
    RUN(check_norm(t, f, n_rows));
    const size_t xb = elem_bytes(f->x_type), yb = elem_bytes(f->y_type), wb = elem_bytes(f->w_type);
    const int64_t cols = (int64_t)f->heads * f->width, n = n_rows;
    const Mat mx{x, ld_x, cols, xb}, ma{add, ld_add, cols, yb}, ms{sum, ld_sum, cols, xb}, my{y, ld_y, cols, yb};
    if (!mat_ok(mx, n) || !mat_ok(my, n) || (add && !mat_ok(ma, n)) || (sum && (!add || !mat_ok(ms, n)))) return MARS_ERR_INVALID_ARG;
    if (!weight || !aligned_to(weight, wb) || !aligned_to(bias, wb) || !aligned4(mean) || !aligned4(rstd) ||
        (f->kind == MARS_NORM_RMS && (mean || bias))) return MARS_ERR_INVALID_ARG;
    if (n_rows == 0) return MARS_OK;
    const size_t wn = (size_t)f->width * wb, sn = (size_t)n * f->heads * 4;
    if (clash(my, mx, n) || clash(ms, mx, n) || clash(my, ma, n) || clash(ms, ma, n) || clash(my, ms, n, false)) return MARS_ERR_INVALID_ARG;
    // y in place of x or add and sum in place of the same would be one memory, caught above; statistics and weights stand alone
    for (const Mat* m : {&my, &ms})
        if (clash(*m, n, weight, wn) || clash(*m, n, bias, wn) || clash(*m, n, mean, sn) || clash(*m, n, rstd, sn)) return MARS_ERR_INVALID_ARG;
    for (float* s : {mean, rstd})
        if (clash(mx, n, s, sn) || clash(ma, n, s, sn)) return MARS_ERR_INVALID_ARG;
    const Flat out[2] = {{mean, sn}, {rstd, sn}}, in[2] = {{weight, wn}, {bias, wn}};
    if (!flats_ok(out, in)) return MARS_ERR_INVALID_ARG;
    const DeviceGuard guard(t->device);
    if (!guard.ok) return MARS_ERR_CUDA;
    NormArgs a{};
    a.rows = n_rows * f->heads; a.heads = f->heads; a.width = f->width; a.layer = f->kind == MARS_NORM_LAYER; a.eps = f->eps; a.w_type = f->w_type;
    a.has_add = add != nullptr; a.has_bias = bias != nullptr;
    a.x = x; a.add = add ? add : x; a.weight = weight; a.bias = bias ? bias : weight; a.sum = sum; a.y = y;
    a.ld_x = ld_x; a.ld_add = add ? ld_add : ld_x; a.ld_sum = ld_sum; a.ld_y = ld_y; a.mean = mean; a.rstd = rstd;
    // pieces of 16 bytes hold eight values of 16 bits; of fp32 a piece of eight is two of them
    const bool vector = f->width % 8 == 0 && vector_ok(mx) && vector_ok(my) && (!add || vector_ok(ma)) && (!sum || vector_ok(ms)) &&
                        aligned16(weight) && aligned16(bias);
    return launched(launch_norm(a, f->x_type, f->y_type, vector, t->sms, (cudaStream_t)cuda_stream));
}

mars_status_t mars_norm_grad(mars_train_t* t, void* cuda_stream, const mars_norm_t* f, int32_t n_rows, const void* dy, int64_t ld_dy,
                             const void* x, int64_t ld_x, const void* weight, const float* mean, const float* rstd, const void* d_sum,
                             int64_t ld_d_sum, void* dx, int64_t ld_dx, void* dw, void* db, int32_t dw_type, int32_t accumulate) {
    RUN(check_norm(t, f, n_rows));
    const size_t xb = elem_bytes(f->x_type), yb = elem_bytes(f->y_type), wb = elem_bytes(f->w_type);
    const int64_t cols = (int64_t)f->heads * f->width, n = n_rows;
    const bool layer = f->kind == MARS_NORM_LAYER;
    const Mat mdy{dy, ld_dy, cols, yb}, mx{x, ld_x, cols, xb}, ms{d_sum, ld_d_sum, cols, xb}, mdx{dx, ld_dx, cols, xb};
    if (!mat_ok(mdy, n) || !mat_ok(mx, n) || !mat_ok(mdx, n) || (d_sum && !mat_ok(ms, n))) return MARS_ERR_INVALID_ARG;
    if (!weight || !aligned_to(weight, wb) || (n > 0 && (!rstd || (layer && !mean))) || !aligned4(mean) || !aligned4(rstd) ||
        (!layer && (mean || db)) || !type_ok(dw_type) || !aligned_to(dw, elem_bytes(dw_type)) || !aligned_to(db, elem_bytes(dw_type)))
        return MARS_ERR_INVALID_ARG;
    const size_t wn = (size_t)f->width * wb, sn = (size_t)n * f->heads * 4, gn = (size_t)f->width * elem_bytes(dw_type);
    if (clash(mdx, mdy, n) || clash(mdx, mx, n) || clash(mdx, ms, n) || clash(mdx, n, weight, wn) || clash(mdx, n, mean, sn) ||
        clash(mdx, n, rstd, sn)) return MARS_ERR_INVALID_ARG;
    for (void* g : {dw, db})
        for (const Mat* m : {&mdx, &mdy, &mx, &ms})
            if (clash(*m, n, g, gn)) return MARS_ERR_INVALID_ARG;
    const Flat out[2] = {{dw, gn}, {db, gn}}, in[3] = {{weight, wn}, {mean, sn}, {rstd, sn}};
    if (!flats_ok(out, in)) return MARS_ERR_INVALID_ARG;
    const DeviceGuard guard(t->device);
    if (!guard.ok) return MARS_ERR_CUDA;
    NormGradArgs a{};
    a.rows = n_rows * f->heads; a.heads = f->heads; a.width = f->width; a.layer = layer; a.w_type = f->w_type;
    a.has_d_sum = d_sum != nullptr;
    a.dy = dy; a.x = x; a.weight = weight; a.d_sum = d_sum ? d_sum : x; a.dx = dx;
    a.ld_dy = ld_dy; a.ld_x = ld_x; a.ld_d_sum = d_sum ? ld_d_sum : ld_x; a.ld_dx = ld_dx; a.mean = mean; a.rstd = rstd;
    if (dw) a.part_w = (float*)t->scratch;
    if (db) a.part_b = (float*)(t->scratch + align_up(norm_grad_part_bytes(t->max_width), 256));
    const bool vector = f->width % 8 == 0 && vector_ok(mx) && vector_ok(mdy) && vector_ok(mdx) && (!d_sum || vector_ok(ms)) && aligned16(weight);
    return launched(launch_norm_grad(a, f->x_type, f->y_type, vector, t->sms, dw, db, dw_type, accumulate != 0, (cudaStream_t)cuda_stream));
}

// ---------------------------------------------------------------------------------------------- rotation

static bool rope_form_ok(const mars_rope_form_t* f) {
    if (!f || f->rotary < 2 || f->rotary > 512 || f->rotary % 2 || (f->layout != MARS_ROPE_HALF && f->layout != MARS_ROPE_INTERLEAVED))
        return false;
    if (!(f->theta > 0.) || !std::isfinite(f->theta) || !((float)f->scale > 0.f) || !std::isfinite((float)f->scale)) return false;
    if (f->scaling == MARS_ROPE_PLAIN) return true;
    if (!(f->factor > 0.) || !std::isfinite(f->factor)) return false;
    if (f->scaling == MARS_ROPE_LINEAR) return true;
    if (f->scaling == MARS_ROPE_BASE) return f->rotary > 2;
    return f->scaling == MARS_ROPE_PARTS && f->trained_positions > 0. && std::isfinite(f->trained_positions) && f->slow >= 0. &&
           f->fast > f->slow && std::isfinite(f->fast);
}

// The frequencies in 64 bits of mantissa, so that what is kept of them (angles for one position, turns for one position) is rounded once: in
// fp64 the exponent's rounding alone, times ln theta, is several steps.
static constexpr long double kTwoPi = 6.283185307179586476925286766559L;
static_assert(std::numeric_limits<long double>::digits >= 64, "frequencies need more bits than fp64 has");
static void long_frequencies(const mars_rope_form_t* f, long double* out) {
    const long double d = f->rotary, factor = f->factor;
    const long double theta = f->scaling == MARS_ROPE_BASE ? f->theta * std::pow(factor, d / (d - 2)) : f->theta;
    for (int i = 0; i < f->rotary / 2; ++i) {
        long double v = std::pow(theta, -2 * i / d);
        if (f->scaling == MARS_ROPE_LINEAR) v /= factor;
        if (f->scaling == MARS_ROPE_PARTS) {
            const long double turns = f->trained_positions * v / kTwoPi;
            const long double keep = std::fmin(1.L, std::fmax(0.L, (turns - f->slow) / ((long double)f->fast - f->slow)));
            v *= keep + (1 - keep) / factor;
        }
        out[i] = v;
    }
}

mars_status_t mars_rope_frequencies(const mars_rope_form_t* f, double* out) {
    if (!rope_form_ok(f) || !out) return MARS_ERR_INVALID_ARG;
    long double table[256];
    long_frequencies(f, table);
    for (int i = 0; i < f->rotary / 2; ++i) out[i] = (double)table[i];
    return MARS_OK;
}

size_t mars_rope_bytes(const mars_rope_form_t* f) { return rope_form_ok(f) ? align_up((size_t)f->rotary / 2 * 8, 256) : 0; }

mars_status_t mars_rope_create(const mars_rope_form_t* f, void* workspace, size_t workspace_bytes, mars_rope_t** out) {
    if (!rope_form_ok(f) || !workspace || !out || (uintptr_t)workspace % 256 || workspace_bytes < mars_rope_bytes(f)) return MARS_ERR_INVALID_ARG;
    long double frequency[256];
    double table[256];
    long_frequencies(f, frequency);
    for (int i = 0; i < f->rotary / 2; ++i) {
        table[i] = (double)(frequency[i] / kTwoPi);
        if (!std::isfinite(table[i])) return MARS_ERR_INVALID_ARG;
    }
    int dev = 0, sms = 0;
    RUN(device_info(&dev, &sms));
    RUN(launched(init_rope_kernels()));
    CUDA_TRY(cudaMemcpy(workspace, table, (size_t)f->rotary / 2 * 8, cudaMemcpyHostToDevice));
    CUDA_TRY(cudaStreamSynchronize(cudaStreamLegacy));           // a non-blocking stream does not wait for the copy
    mars_rope_t* r = new (std::nothrow) mars_rope_t();
    if (!r) return MARS_ERR_INVALID_ARG;
    r->device = dev; r->sms = sms; r->rotary = f->rotary; r->interleaved = f->layout == MARS_ROPE_INTERLEAVED;
    r->scale = (float)f->scale; r->turns = (const double*)workspace;
    *out = r;
    return MARS_OK;
}

mars_status_t mars_rope_free(mars_rope_t* r) {
    if (!r) return MARS_ERR_BAD_HANDLE;
    delete r;
    return MARS_OK;
}

mars_status_t mars_rope(mars_rope_t* r, void* cuda_stream, int32_t n, const int32_t* positions, int32_t head_dim, int32_t type,
                        const void* q, int64_t ld_q, int32_t q_heads, void* out_q, int64_t ld_out_q, const void* k, int64_t ld_k,
                        int32_t k_heads, void* out_k, int64_t ld_out_k, int32_t inverse) {
    if (!r) return MARS_ERR_BAD_HANDLE;
    if (n < 0 || head_dim < r->rotary || head_dim > 512 || !type_ok(type) || q_heads < 1 || k_heads < 0 || q_heads > (1 << 16) || k_heads > (1 << 16))
        return MARS_ERR_INVALID_ARG;
    const size_t eb = elem_bytes(type);
    const Mat iq{q, ld_q, (int64_t)q_heads * head_dim, eb}, oq{out_q, ld_out_q, (int64_t)q_heads * head_dim, eb};
    const Mat ik{k_heads ? k : nullptr, ld_k, (int64_t)k_heads * head_dim, eb}, ok{k_heads ? out_k : nullptr, ld_out_k, (int64_t)k_heads * head_dim, eb};
    if (!mat_ok(iq, n) || !mat_ok(oq, n) || (k_heads && (!mat_ok(ik, n) || !mat_ok(ok, n)))) return MARS_ERR_INVALID_ARG;
    if (n > 0 && (!positions || !aligned4(positions))) return MARS_ERR_INVALID_ARG;
    if (n == 0) return MARS_OK;
    const size_t pn = (size_t)n * 4;
    if (clash(oq, iq, n) || clash(ok, ik, n) || clash(oq, ik, n, false) || clash(ok, iq, n, false) || clash(oq, ok, n, false) ||
        clash(oq, n, positions, pn) || clash(ok, n, positions, pn)) return MARS_ERR_INVALID_ARG;
    const DeviceGuard guard(r->device);
    if (!guard.ok) return MARS_ERR_CUDA;
    RopeArgs a{};
    a.tokens = n; a.head_dim = head_dim; a.rotary = r->rotary; a.interleaved = r->interleaved; a.scale = r->scale; a.sign = inverse ? -1.f : 1.f;
    a.positions = positions; a.turns = r->turns;
    a.in[0] = q; a.in[1] = k_heads ? k : q; a.out[0] = out_q; a.out[1] = k_heads ? out_k : out_q;
    a.ld_in[0] = ld_q; a.ld_in[1] = k_heads ? ld_k : ld_q; a.ld_out[0] = ld_out_q; a.ld_out[1] = k_heads ? ld_out_k : ld_out_q;
    a.heads[0] = q_heads; a.heads[1] = k_heads;
    const bool vector = head_dim % 8 == 0 && r->rotary % (r->interleaved ? 8 : 16) == 0 && vector_ok(iq) && vector_ok(oq) &&
                        (!k_heads || (vector_ok(ik) && vector_ok(ok)));
    return launched(launch_rope(a, type, vector, r->sms, (cudaStream_t)cuda_stream));
}

// ------------------------------------------------------------------------------------------------ router

static mars_status_t check_router(const mars_train* t, int32_t rows, int32_t experts, int32_t top_k, const Mat& logits, int32_t type) {
    if (!t) return MARS_ERR_BAD_HANDLE;
    if (rows < 0 || experts < 1 || experts > t->max_experts || top_k < 1 || top_k > experts || top_k > kRouterMaxK || !type_ok(type) ||
        (int64_t)rows * top_k > INT32_MAX || !mat_ok(logits, rows)) return MARS_ERR_INVALID_ARG;
    return MARS_OK;
}
// neighbouring fours of a row in one load
static bool fours(const Mat& m, int experts) { return experts % 4 == 0 && vector_ok(m, 4 * m.elem); }

mars_status_t mars_router(mars_train_t* t, void* cuda_stream, int32_t rows, int32_t experts, int32_t top_k, const void* logits,
                          int64_t ld, int32_t type, const uint8_t* live, int32_t renormalise, int32_t* idx, float* weights, float* lse,
                          int32_t* counts, int32_t* offsets, float* prob_sums, float* losses) {
    const Mat m{logits, ld, experts, type_ok(type) ? elem_bytes(type) : 4};
    RUN(check_router(t, rows, experts, top_k, m, type));
    if (rows > 0 && (!idx || !weights)) return MARS_ERR_INVALID_ARG;
    for (const void* p : {(const void*)idx, (const void*)weights, (const void*)lse, (const void*)counts, (const void*)offsets,
                          (const void*)prob_sums, (const void*)losses})
        if (!aligned4(p)) return MARS_ERR_INVALID_ARG;
    const size_t n = (size_t)rows, en = (size_t)experts * 4;
    const Flat out[7] = {{idx, n * top_k * 4}, {weights, n * top_k * 4}, {lse, n * 4}, {counts, en}, {offsets, en + 4}, {prob_sums, en}, {losses, 8}};
    const Flat in[2] = {{live, n}, {rows ? logits : nullptr, span(rows, ld, experts, m.elem)}};
    if (!flats_ok(out, in)) return MARS_ERR_INVALID_ARG;
    const DeviceGuard guard(t->device);
    if (!guard.ok) return MARS_ERR_CUDA;
    RouterArgs a{};
    a.rows = rows; a.experts = experts; a.top_k = top_k; a.renormalise = renormalise != 0; a.logits = logits; a.ld = ld;
    a.has_live = live != nullptr; a.live = live ? live : (const uint8_t*)logits;
    a.idx = idx; a.weights = weights; a.lse = lse; a.counts = counts; a.offsets = offsets; a.prob_sums = prob_sums; a.losses = losses;
    const size_t blocks = (size_t)router_max_blocks(kTrainSms);
    a.work_counts = t->counts; a.parts = (float*)t->scratch;
    a.z_parts = (double*)(t->scratch + align_up(blocks * t->max_experts * 4, 256)); a.ticket = t->tickets;
    return launched(launch_router(a, type, fours(m, experts), t->sms, (cudaStream_t)cuda_stream));
}

mars_status_t mars_router_grad(mars_train_t* t, void* cuda_stream, int32_t rows, int32_t experts, int32_t top_k, const void* logits,
                               int64_t ld, int32_t type, const int32_t* idx, const float* lse, const int32_t* counts,
                               const float* d_weights, int32_t renormalise, float balance_coef, float z_coef, void* d_logits,
                               int64_t ld_d) {
    const Mat m{logits, ld, experts, type_ok(type) ? elem_bytes(type) : 4}, d{d_logits, ld_d, experts, m.elem};
    RUN(check_router(t, rows, experts, top_k, m, type));
    if (!mat_ok(d, rows) || !std::isfinite(balance_coef) || !std::isfinite(z_coef)) return MARS_ERR_INVALID_ARG;
    if (rows == 0) return MARS_OK;
    if (!idx || !lse || !counts || !aligned4(idx) || !aligned4(lse) || !aligned4(counts) || !aligned4(d_weights)) return MARS_ERR_INVALID_ARG;
    const size_t n = (size_t)rows;
    if (clash(d, m, rows) || clash(d, rows, idx, n * top_k * 4) || clash(d, rows, lse, n * 4) || clash(d, rows, counts, (size_t)experts * 4) ||
        clash(d, rows, d_weights, n * top_k * 4)) return MARS_ERR_INVALID_ARG;
    const DeviceGuard guard(t->device);
    if (!guard.ok) return MARS_ERR_CUDA;
    RouterGradArgs a{};
    a.rows = rows; a.experts = experts; a.top_k = top_k; a.renormalise = renormalise != 0; a.logits = logits; a.ld = ld; a.idx = idx;
    a.counts = counts; a.lse = lse; a.has_d_weights = d_weights != nullptr; a.d_weights = d_weights ? d_weights : (const float*)idx; a.balance = balance_coef; a.z = z_coef; a.d_logits = d_logits; a.ld_d = ld_d;
    return launched(launch_router_grad(a, type, fours(m, experts) && fours(d, experts), t->sms, (cudaStream_t)cuda_stream));
}

// ------------------------------------------------------------------------------------------- policy loss

mars_status_t mars_policy_loss(mars_train_t* t, void* cuda_stream, const mars_policy_t* f, int32_t n_tokens, int32_t n_seqs,
                               const int32_t* seq_off, const int32_t* targets, const float* logprobs, const float* old_logprobs,
                               const float* ref_logprobs, const float* advantages, float* stats, float* d_logprobs) {
    if (!t) return MARS_ERR_BAD_HANDLE;
    if (!f || n_tokens < 0 || n_tokens > (1 << 30) || n_seqs < 1 || n_seqs > t->max_seqs) return MARS_ERR_INVALID_ARG;
    if (f->reduce < MARS_MEAN_TOKENS || f->reduce > MARS_SUM || !(f->clip_low >= 0.) || f->clip_low > 1. || !(f->clip_high >= 0.) ||
        !std::isfinite((float)f->clip_high) || !std::isfinite((float)f->kl_coef) || !std::isfinite((float)f->scale)) return MARS_ERR_INVALID_ARG;
    if (f->kl_coef != 0. && !ref_logprobs) return MARS_ERR_INVALID_ARG;
    if (!seq_off || !stats || !aligned4(seq_off) || !aligned4(stats)) return MARS_ERR_INVALID_ARG;
    const bool per_token = f->advantages_per_token != 0;
    if ((n_tokens > 0 && (!targets || !logprobs || !old_logprobs)) || (!advantages && !(per_token && n_tokens == 0))) return MARS_ERR_INVALID_ARG;
    for (const void* p : {(const void*)targets, (const void*)logprobs, (const void*)old_logprobs, (const void*)ref_logprobs,
                          (const void*)advantages, (const void*)d_logprobs})
        if (!aligned4(p)) return MARS_ERR_INVALID_ARG;
    const size_t nb = (size_t)n_tokens * 4, ab = per_token ? nb : (size_t)n_seqs * 4;
    const Flat out[2] = {{stats, kPolicyStats * 4}, {d_logprobs, nb}};
    // the gradient may take the place of the log-probs
    const Flat in[6] = {{seq_off, ((size_t)n_seqs + 1) * 4}, {targets, nb}, {logprobs == d_logprobs ? nullptr : logprobs, nb},
                        {old_logprobs, nb}, {ref_logprobs, nb}, {advantages, ab}};
    if (!flats_ok(out, in) || overlap(out[0], Flat{logprobs, nb})) return MARS_ERR_INVALID_ARG;
    const DeviceGuard guard(t->device);
    if (!guard.ok) return MARS_ERR_CUDA;
    PolicyArgs a{};
    a.tokens = n_tokens; a.seqs = n_seqs; a.reduce = f->reduce; a.per_token = per_token; a.lp = logprobs; a.old_lp = old_logprobs;
    a.has_ref = ref_logprobs != nullptr; a.ref = ref_logprobs ? ref_logprobs : logprobs; a.adv = advantages; a.targets = targets; a.seq_off = seq_off;
    a.log_low = f->clip_low < 1. ? std::log1p(-f->clip_low) : -HUGE_VAL; a.log_high = std::log1p(f->clip_high);
    a.low = (float)(1. - f->clip_low); a.high = (float)(1. + f->clip_high); a.kl = (float)f->kl_coef; a.scale = f->scale;
    a.stats = stats; a.d_lp = d_logprobs; a.seq_live = t->seq_live; a.totals = t->totals; a.parts = (double*)t->scratch;
    a.ticket = t->tickets + 1;
    a.vector = aligned16(targets) && aligned16(logprobs) && aligned16(old_logprobs) && aligned16(ref_logprobs) && aligned16(d_logprobs) &&
               (!per_token || aligned16(advantages));
    return launched(launch_policy_loss(a, t->sms, (cudaStream_t)cuda_stream));
}

}  // extern "C"
