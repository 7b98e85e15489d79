// C entry points of linear layers and layer normalisation: argument checks and dispatch.
#include <string.h>

#include <algorithm>

#include "boss_args.cuh"
#include "layer_norm.cuh"
#include "linear.cuh"

namespace aa {

namespace {

constexpr int64_t kMaxWidth = 1ll << 30, kMaxRows = (1ll << 31) - 1;

MatArg mat(const aa_rows* m) { return m ? MatArg{m->data, m->row_stride} : MatArg{nullptr, 0}; }

bool check_live(const int32_t* offsets, int64_t n_seg) { return offsets ? n_seg >= 0 : n_seg == 0; }

LiveRows live_arg(const int32_t* offsets, int64_t n_seg, const int32_t* count_dev, int64_t rows) { return LiveRows{offsets, n_seg, count_dev, rows}; }

// In bytes, so that matrices of different types compare.
Extent bytes_of(const aa_rows* m) {
    const int64_t es = m->dtype == AA_BF16 ? 2 : 4;
    return Extent{m->data, m->rows, m->row_stride * es, 1, 0, m->cols * es};
}
Extent bytes_of(const float* v, int64_t n) { return Extent{v, v ? 1 : 0, 0, 1, 0, n * 4}; }
bool clear_of(const aa_rows* out, const aa_rows* other) { return !out || !other || apart(bytes_of(out), bytes_of(other), 1); }
bool clear_of(const aa_rows* out, const float* v, int64_t n) { return !out || !v || apart(bytes_of(out), bytes_of(v, n), 1); }
bool clear_of(const float* a, const float* b, int64_t n) { return !a || !b || a + n <= b || b + n <= a; }
// The same matrix, or nothing in common.
bool same_or_clear(const aa_rows* out, const aa_rows* in) {
    if (!out || !in) return true;
    return in->data == out->data ? in->row_stride == out->row_stride || in->rows <= 1 : clear_of(out, in);
}

bool floats_ok(const float* p) { return (uintptr_t)p % 4 == 0; }
bool act_ok(int32_t a) { return a >= AA_ACT_NONE && a <= AA_ACT_SILU; }

// Operands that TMA cannot fetch are copied into scratch memory - fp32 numbers as three planes of bf16 terms, bf16 rows with an alignment that it can - rather than
// taken apart by every tile that needs them.  Gradients of 8,000 x 1,024 -> 1,024 unaligned bf16 take 61 us with copies, 239 without, 200 x 512 -> 512 20
// and 34, 25,000 x 8 -> 512 61 and 133; fp32 188 and 338, 29 and 40, 91 and 124.  Weights in fp32 that few rows use are not worth it: 64 x 512 ->
// 32,000 takes 260 us with copies, 186 without, 5 x 2,000 -> 3,000 66 and 51; at 500 rows both take 370.
constexpr int64_t kFewRowsOfCopies = 512, kWeightsOfCopies = 1 << 21;

bool by_tma(const aa_rows* m) { return (uintptr_t)m->data % 16 == 0 && m->row_stride % 8 == 0; }

// G, x and w as far as they are copied, then the column sums' parts or (later in the call) the products' parts.
struct LinearScratch {
    size_t g, x, w, parts, total;      // bytes
    bool copies;
};
// The parts of a cut tile are 256 KB in fp32 on each of a B200's 74 pairs of SMs; three rounds of them (58 MB) leave little to balance.
constexpr int64_t kProductParts = 3ll * 74 * 256 * 256;         // floats
// What a product [m x n] over k can use of them, whatever its tiles are (256 x 256 at most, 64 columns at least): up to 16 parts of a tile and of its rows' sums (make_plan), of
// four slices or more.
int64_t part_floats(int64_t m, int64_t n, int64_t k) {
    const int64_t splits = std::min<int64_t>(16, (k + 63) / 64 / 4), tm = (m + 255) / 256, tn = (n + 255) / 256;
    return splits < 2 ? 0 : std::min(kProductParts, std::min(tm * tn, kProductParts) * splits * (256 * 256 + 256 * 4));
}
int64_t padded(int64_t cols) { return (cols + 7) / 8 * 8; }
LinearScratch linear_scratch(const aa_rows* x, const aa_rows* w, int act) {
    const auto up = [](size_t b) { return (b + 255) / 256 * 256; };
    LinearScratch s = {};
    const bool wide = x->dtype == AA_F32;
    const int64_t rows = x->rows, inner = x->cols, cols = w->rows;
    s.copies = !wide || rows >= kFewRowsOfCopies || inner * cols <= kWeightsOfCopies;
    const size_t each = s.copies && wide ? 6 : (wide ? 4 : 2);
    if (act != AA_ACT_NONE || (s.copies && (wide || cols % 8 || !by_tma(x) || !by_tma(w)))) s.g = up((size_t)rows * (size_t)padded(cols) * each);
    if (s.copies && (wide || !by_tma(x))) s.x = up((size_t)rows * (size_t)padded(inner) * each);
    if (s.copies && (wide || !by_tma(w))) s.w = up((size_t)cols * (size_t)padded(inner) * each);
    s.parts = up(std::max({kSlopeParts * cols, part_floats(rows, inner, cols), part_floats(cols, inner, rows)}) * sizeof(float));
    s.total = s.g + s.x + s.w + s.parts;
    return s;
}

aa_status check_linear(const aa_rows* x, const aa_rows* w) {
    if (check_rows(x) != AA_OK || check_rows(w) != AA_OK || x->dtype != w->dtype || x->cols != w->cols || w->rows < 1) return AA_ERR_INVALID_ARG;
    return x->cols > kMaxWidth || w->rows > kMaxWidth || x->rows > kMaxRows ? AA_ERR_UNSUPPORTED : AA_OK;
}

}  // namespace
}  // namespace aa

namespace aa {

// Up to 16 rows of a forward call straight from memory; bf16 operands that TMA can fetch by TMA; the others by the kernel that takes its operands apart on the way.
aa_status launch_product(aa_ctx_impl* c, const ProductParams& p, int dtype) {
    if (product_few_fits(p)) return launch_product_few(c, p, dtype);
    if (dtype == AA_BF16 && product_tc_fits(p)) return launch_product_tc(c, p);
    return launch_product_split(c, p, dtype);
}

}  // namespace aa

using namespace aa;

extern "C" {

aa_status aa_linear(aa_ctx* ctx, const aa_rows* x, const aa_rows* w, const float* bias, int32_t activation, const aa_rows* residual, const int32_t* offsets,
                    int64_t n_seg, const int32_t* count_dev, const aa_rows* pre, const aa_rows* out) {
    if (!ctx || !act_ok(activation) || !check_live(offsets, n_seg) || !floats_ok(bias)) return AA_ERR_INVALID_ARG;
    const aa_status st = check_linear(x, w);
    if (st != AA_OK) return st;
    const auto like_out = [&](const aa_rows* m) { return check_rows(m) == AA_OK && m->dtype == x->dtype && m->rows == x->rows && m->cols == w->rows; };
    if (!like_out(out) || (residual && !like_out(residual)) || (pre && !like_out(pre))) return AA_ERR_INVALID_ARG;
    for (const aa_rows* m : {pre, out})
        if (!clear_of(m, x) || !clear_of(m, w) || !clear_of(m, bias, w->rows)) return AA_ERR_INVALID_ARG;
    if (!same_or_clear(out, residual) || !clear_of(pre, residual) || !clear_of(pre, out)) return AA_ERR_INVALID_ARG;
    if (x->rows == 0) return AA_OK;
    aa_ctx_impl* c = reinterpret_cast<aa_ctx_impl*>(ctx);
    ProductParams p = {};
    p.a = mat(x);
    p.b = mat(w);
    p.m = x->rows;
    p.n = w->rows;
    p.k = x->cols;
    p.live = live_arg(offsets, n_seg, count_dev, x->rows);
    p.bias = bias;
    p.act = activation;
    p.residual = mat(residual);
    p.pre = mat(pre);
    p.out = mat(out);
    p.ctl = c->ctl;
    return launch_product(c, p, x->dtype);
}

aa_status aa_linear_grad_scratch_bytes(const aa_rows* x, const aa_rows* w, int32_t activation, size_t* bytes) {
    if (!bytes || !act_ok(activation)) return AA_ERR_INVALID_ARG;
    const aa_status st = check_linear(x, w);
    if (st != AA_OK) return st;
    *bytes = linear_scratch(x, w, activation).total;
    return AA_OK;
}

aa_status aa_linear_grad(aa_ctx* ctx, const aa_rows* x, const aa_rows* w, int32_t activation, const aa_rows* pre, const aa_rows* dout, const aa_rows* residual,
                         const int32_t* offsets, int64_t n_seg, const int32_t* count_dev, const aa_rows* dx, const aa_rows* dw, float* dbias, void* scratch,
                         size_t scratch_bytes) {
    if (!ctx || !act_ok(activation) || !check_live(offsets, n_seg) || !floats_ok(dbias) || (activation == AA_ACT_NONE) != !pre || (residual && !dx)) return AA_ERR_INVALID_ARG;
    const aa_status st = check_linear(x, w);
    if (st != AA_OK) return st;
    const auto like_out = [&](const aa_rows* m) { return check_rows(m) == AA_OK && m->dtype == x->dtype && m->rows == x->rows && m->cols == w->rows; };
    if (!like_out(dout) || (pre && !like_out(pre))) return AA_ERR_INVALID_ARG;
    for (const aa_rows* m : {residual, dx})
        if (m && (check_rows(m) != AA_OK || !same_shape(*m, *x))) return AA_ERR_INVALID_ARG;
    if (dw && (check_rows(dw) != AA_OK || !same_shape(*dw, *w))) return AA_ERR_INVALID_ARG;
    for (const aa_rows* in : {x, w, pre, dout})
        if (!clear_of(dx, in) || !clear_of(dw, in) || !clear_of(in, dbias, w->rows)) return AA_ERR_INVALID_ARG;
    if (!same_or_clear(dx, residual) || !clear_of(dw, residual) || !clear_of(dw, dx) || !clear_of(dx, dbias, w->rows) || !clear_of(dw, dbias, w->rows) ||
        !clear_of(residual, dbias, w->rows))
        return AA_ERR_INVALID_ARG;
    const LinearScratch need = linear_scratch(x, w, activation);
    if (!scratch || (uintptr_t)scratch % 256) return AA_ERR_INVALID_ARG;
    if (scratch_bytes < need.total) return AA_ERR_WORKSPACE;
    aa_ctx_impl* c = reinterpret_cast<aa_ctx_impl*>(ctx);
    const LiveRows live = live_arg(offsets, n_seg, count_dev, x->rows);
    if (x->rows == 0) {
        aa_status zero = AA_OK;
        if (dw) zero = cuda_ok(cudaMemset2DAsync(dw->data, (size_t)dw->row_stride * (dw->dtype == AA_BF16 ? 2 : 4), 0, (size_t)dw->cols * (dw->dtype == AA_BF16 ? 2 : 4), (size_t)dw->rows, c->stream));
        if (zero == AA_OK && dbias) zero = cuda_ok(cudaMemsetAsync(dbias, 0, (size_t)w->rows * sizeof(float), c->stream));
        return zero;
    }
    const bool act = activation != AA_ACT_NONE, wide = x->dtype == AA_F32, planes = wide && need.copies;
    char* at = static_cast<char*>(scratch);
    float* parts = reinterpret_cast<float*>(at + need.g + need.x + need.w);
    ProductParams grad_x = {}, grad_w = {};
    grad_x.ctl = grad_w.ctl = c->ctl;
    grad_x.live = grad_w.live = live;
    grad_x.parts = grad_w.parts = parts;
    grad_x.part_floats = grad_w.part_floats = (int64_t)(need.parts / sizeof(float));
    // G is a matrix of its own where there is an activation, or where dout is copied.  In bf16 it is rounded: 25,000 x 512 -> 2,048 with GELU is off by 2.3e-3 of its results then, by
    // 1.7e-3 if G kept 32 bits (the results' own rounding), for which both products, 97 of the call's 172 us, would be done twice.
    const bool copy_g = need.g > 0 && (act || planes || !by_tma(dout));
    const MatArg g = copy_g ? MatArg{at, padded(w->rows)} : mat(dout);
    const MatArg xs = need.x ? MatArg{at + need.g, padded(x->cols)} : mat(x), ws = need.w ? MatArg{at + need.g + need.x, padded(x->cols)} : mat(w);
    grad_x.a = grad_w.a = g;
    grad_x.b = ws;
    grad_w.b = xs;
    if (planes) {
        grad_x.plane_a = grad_w.plane_a = x->rows * g.stride;
        grad_x.plane_b = w->rows * ws.stride;
        grad_w.plane_b = x->rows * xs.stride;
    }
    if (dw) {
        grad_w.a_across = grad_w.b_across = grad_w.live_k = true;
        grad_w.m = w->rows;
        grad_w.n = x->cols;
        grad_w.k = x->rows;
        grad_w.out = mat(dw);
        // the sums come with the product where its kernel has them and there is no other pass over dout
        if (!copy_g && dbias && !wide && product_tc_fits(grad_w)) grad_w.a_sums = dbias;
    }
    aa_status done = AA_OK;
    // the pass over dout, then the copies of x and w
    SlopeParams jobs[kSlopeJobs];
    int n_jobs = 0;
    const auto pass = [&](const aa_rows* from, const MatArg& to, const LiveRows& rows) -> SlopeParams& {
        SlopeParams& s = jobs[n_jobs++];
        s = {};
        s.dout = mat(from);
        s.g = to;
        if (to.data && need.copies) s.plane = from->rows * to.stride;
        s.rows = from->rows;
        s.cols = from->cols;
        s.live = rows;
        s.act = AA_ACT_NONE;
        s.ctl = c->ctl;
        return s;
    };
    const bool want_g = copy_g && (dx || dw);
    if (want_g || (dbias && !grad_w.a_sums)) {
        SlopeParams& s = pass(dout, want_g ? g : MatArg{nullptr, 0}, live);
        s.pre = mat(pre);
        s.act = activation;
        s.parts = parts;
        s.dbias = grad_w.a_sums ? nullptr : dbias;
        // a pass that copies nothing is of another kind
        if (s.plane == 0) {
            if ((done = launch_slopes(c, jobs, 1, x->dtype)) != AA_OK) return done;
            n_jobs = 0;
        }
    }
    if (dw && need.x) pass(x, xs, live);
    if (dx && need.w) pass(w, ws, live_arg(nullptr, 0, nullptr, w->rows));
    if (n_jobs > 0 && (done = launch_slopes(c, jobs, n_jobs, x->dtype)) != AA_OK) return done;
    if (dx) {
        grad_x.b_across = true;
        grad_x.m = x->rows;
        grad_x.n = x->cols;
        grad_x.k = w->rows;
        grad_x.residual = mat(residual);
        grad_x.out = mat(dx);
        if ((done = planes ? launch_product_planes(c, grad_x) : launch_product(c, grad_x, x->dtype)) != AA_OK) return done;
    }
    if (!dw) return AA_OK;
    return planes ? launch_product_planes(c, grad_w) : launch_product(c, grad_w, x->dtype);
}

aa_status aa_layer_norm(aa_ctx* ctx, const aa_rows* x, const float* gamma, const float* beta, float eps, const int32_t* offsets, int64_t n_seg,
                        const int32_t* count_dev, const aa_rows* out) {
    if (!ctx || !check_live(offsets, n_seg) || check_rows(x) != AA_OK || check_rows(out) != AA_OK || !same_shape(*x, *out)) return AA_ERR_INVALID_ARG;
    if (!(eps >= 0.0f) || !floats_ok(gamma) || !floats_ok(beta) || !same_or_clear(out, x) || !clear_of(out, gamma, x->cols) || !clear_of(out, beta, x->cols)) return AA_ERR_INVALID_ARG;
    if (x->cols > kMaxWidth) return AA_ERR_UNSUPPORTED;
    if (x->rows == 0) return AA_OK;
    aa_ctx_impl* c = reinterpret_cast<aa_ctx_impl*>(ctx);
    NormParams p = {};
    p.x = mat(x);
    p.out = mat(out);
    p.cols = x->cols;
    p.live = live_arg(offsets, n_seg, count_dev, x->rows);
    p.gamma = gamma;
    p.beta = beta;
    p.eps = eps;
    p.ctl = c->ctl;
    return launch_layer_norm(c, p, x->dtype, false, nullptr, nullptr);
}

aa_status aa_layer_norm_grad_scratch_bytes(const aa_rows* x, size_t* bytes) {
    if (!bytes || check_rows(x) != AA_OK) return AA_ERR_INVALID_ARG;
    if (x->cols > kMaxWidth) return AA_ERR_UNSUPPORTED;
    const size_t stats = x->cols > kNormInRegisters ? ((size_t)x->rows * sizeof(NormStats) + 255) / 256 * 256 : 0;
    *bytes = stats + norm_scratch_floats(x->rows, x->cols) * sizeof(float);
    return AA_OK;
}

aa_status aa_layer_norm_grad(aa_ctx* ctx, const aa_rows* x, const float* gamma, float eps, const aa_rows* dout, const aa_rows* residual, const int32_t* offsets,
                             int64_t n_seg, const int32_t* count_dev, const aa_rows* dx, float* dgamma, float* dbeta, void* scratch, size_t scratch_bytes) {
    if (!ctx || !check_live(offsets, n_seg) || check_rows(x) != AA_OK || !(eps >= 0.0f)) return AA_ERR_INVALID_ARG;
    for (const aa_rows* m : {dout, dx})
        if (check_rows(m) != AA_OK || !same_shape(*m, *x)) return AA_ERR_INVALID_ARG;
    if (residual && (check_rows(residual) != AA_OK || !same_shape(*residual, *x))) return AA_ERR_INVALID_ARG;
    const int64_t n = x->cols;
    if (!floats_ok(gamma) || !floats_ok(dgamma) || !floats_ok(dbeta) || !same_or_clear(dx, x) || !same_or_clear(dx, dout) || !same_or_clear(dx, residual) || !clear_of(dx, gamma, n) ||
        !clear_of(dgamma, dbeta, n) || !clear_of(gamma, dgamma, n) || !clear_of(gamma, dbeta, n))
        return AA_ERR_INVALID_ARG;
    for (const aa_rows* m : {x, dout, residual, dx})
        if (!clear_of(m, dgamma, n) || !clear_of(m, dbeta, n)) return AA_ERR_INVALID_ARG;
    size_t need = 0;
    const aa_status st = aa_layer_norm_grad_scratch_bytes(x, &need);
    if (st != AA_OK) return st;
    if (need > 0 && (!scratch || (uintptr_t)scratch % 256)) return AA_ERR_INVALID_ARG;
    if (scratch_bytes < need) return AA_ERR_WORKSPACE;
    aa_ctx_impl* c = reinterpret_cast<aa_ctx_impl*>(ctx);
    if (x->rows == 0) {
        aa_status zero = dgamma ? cuda_ok(cudaMemsetAsync(dgamma, 0, (size_t)n * sizeof(float), c->stream)) : AA_OK;
        if (zero == AA_OK && dbeta) zero = cuda_ok(cudaMemsetAsync(dbeta, 0, (size_t)n * sizeof(float), c->stream));
        return zero;
    }
    NormParams p = {};
    p.x = mat(x);
    p.dout = mat(dout);
    p.residual = mat(residual);
    p.out = mat(dx);
    p.cols = n;
    p.live = live_arg(offsets, n_seg, count_dev, x->rows);
    p.gamma = gamma;
    p.eps = eps;
    p.ctl = c->ctl;
    const size_t stats = n > kNormInRegisters ? ((size_t)x->rows * sizeof(NormStats) + 255) / 256 * 256 : 0;
    p.stats = static_cast<NormStats*>(scratch);
    if (dgamma || dbeta) p.parts = reinterpret_cast<float*>(static_cast<char*>(scratch) + stats);
    return launch_layer_norm(c, p, x->dtype, true, dgamma, dbeta);
}

}  // extern "C"
