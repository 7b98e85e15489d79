// C entry points of the operators that train the Boss on the generated batch: argument checks and dispatch.
#include <math.h>
#include <string.h>

#include "rel_attention.cuh"

namespace aa {

namespace {

bool elem_size(int32_t dtype, int64_t& es) {
    es = dtype == AA_BF16 ? 2 : 4;
    return dtype == AA_F32 || dtype == AA_BF16;
}

aa_status check_rows(const aa_rows* m) {
    int64_t es;
    if (!m || !elem_size(m->dtype, es) || m->rows < 0 || m->cols <= 0 || m->cols > 0x7FFFFFF0ll || m->row_stride < m->cols) return AA_ERR_INVALID_ARG;
    if (m->rows > 0 && !m->data) return AA_ERR_INVALID_ARG;
    return (uintptr_t)m->data % (uintptr_t)es ? AA_ERR_INVALID_ARG : AA_OK;
}

// Elements of an operand: data + r * row_step + h * head_step + [0, width), r < rows, h < heads.
struct Extent {
    const void* data;
    int64_t rows, row_step, heads, head_step, width;
};

// No element in common.  Operands whose address ranges interleave are told apart exactly if they have the same steps (views of one packed array);
// interleaving ranges of different steps count as an overlap.
bool apart(Extent a, Extent b, int64_t es) {
    if (a.rows <= 0 || b.rows <= 0) return true;
    const auto span = [](const Extent& x) { return (x.rows - 1) * x.row_step + (x.heads - 1) * x.head_step + x.width; };
    const int64_t d = ((int64_t)(uintptr_t)b.data - (int64_t)(uintptr_t)a.data) / es;
    if (d >= span(a) || -d >= span(b)) return true;
    // an axis of length one has no step
    if (a.rows == 1) a.row_step = b.row_step;
    if (b.rows == 1) b.row_step = a.row_step;
    if (a.heads == 1) a.head_step = b.head_step;
    if (b.heads == 1) b.head_step = a.head_step;
    if (a.row_step != b.row_step || a.head_step != b.head_step) return false;
    // element (r1, h1, e1) of a is (r2, h2, e2) of b:  e1 - e2 = d - (r1 - r2) row_step - (h1 - h2) head_step
    const int64_t lo = 1 - b.width, hi = a.width - 1, step = a.row_step;
    for (int64_t h = 1 - b.heads; h < a.heads; ++h) {
        const int64_t left = d - h * a.head_step;
        if (step == 0) {
            if (left >= lo && left <= hi) return false;
            continue;
        }
        int64_t r = (left - hi) / step;                     // the smallest r with left - r step <= hi
        if (r * step < left - hi) ++r;
        if (r < 1 - b.rows) r = 1 - b.rows;
        if (r < a.rows && left - r * step >= lo) return false;
    }
    return true;
}

// `out` written while `in` is read: the same matrix, or nothing in common.
bool same_or_apart(const void* in, int64_t in_stride, const void* out, int64_t out_stride, int64_t rows, int64_t cols, int64_t es) {
    if (in == out) return in_stride == out_stride || rows <= 1;
    return apart(Extent{in, rows, in_stride, 1, 0, cols}, Extent{out, rows, out_stride, 1, 0, cols}, es);
}

bool same_shape(const aa_rows& a, const aa_rows& b) { return a.dtype == b.dtype && a.rows == b.rows && a.cols == b.cols; }

}  // namespace

bool rel_bucket_bounds(const aa_rel_bias* b, int* per_dir, int* lower) {
    if (b->buckets <= 0 || (b->bidirectional && b->buckets % 2)) return false;
    const int n = b->bidirectional ? b->buckets / 2 : b->buckets, e = n / 2;
    if (n < 2 || n > kMaxPerDir || b->max_distance <= e || b->max_distance > kMaxReach) return false;
    *per_dir = n;
    for (int k = 0; k < n; ++k)
        lower[k] = k < e ? k : (int)ceil((double)e * pow((double)b->max_distance / e, (double)(k - e) / (n - e)) * (1.0 - 1e-9));
    return true;
}

namespace {

aa_status check_tokens(const aa_tokens& t, int64_t es, int64_t rows, int heads, int dim, bool written) {
    if (rows > 0 && !t.data) return AA_ERR_INVALID_ARG;
    if ((uintptr_t)t.data % (uintptr_t)es || t.token_stride < 0 || t.head_stride < 0) return AA_ERR_INVALID_ARG;
    if (written && rows > 0) {
        // two elements never share an address: tokens outside of heads, or heads outside of tokens
        const bool by_token = (heads == 1 || t.head_stride >= dim) && (rows == 1 || t.token_stride >= (heads - 1) * t.head_stride + dim);
        const bool by_head = (rows == 1 || t.token_stride >= dim) && (heads == 1 || t.head_stride >= (rows - 1) * t.token_stride + dim);
        if (!by_token && !by_head) return AA_ERR_INVALID_ARG;
    }
    return AA_OK;
}

TokArg tok(const aa_tokens& t) { return TokArg{t.data, t.token_stride, t.head_stride}; }

Extent query_extent(const aa_tokens& t, const RelParams& p) { return Extent{t.data, p.q_rows, t.token_stride, p.heads, t.head_stride, p.dim}; }
Extent key_extent(const aa_tokens& t, const RelParams& p) { return Extent{t.data, p.k_rows, t.token_stride, p.kv_heads, t.head_stride, p.dim}; }

}  // namespace

aa_status make_rel_params(const aa_attn* a, const aa_rel_bias* b, const aa_dropout_rule* d, RelParams& p) {
    int64_t es;
    if (!a || !elem_size(a->dtype, es)) return AA_ERR_INVALID_ARG;
    if (a->heads <= 0 || a->kv_heads <= 0 || a->heads % a->kv_heads || a->head_dim <= 0 || !(a->scale == a->scale)) return AA_ERR_INVALID_ARG;
    if (a->n_seq < 0 || a->q_rows < 0 || a->k_rows < 0 || a->max_q < 0 || a->max_k < 0) return AA_ERR_INVALID_ARG;
    if (a->n_seq > 0 && (!a->q_offsets || !a->k_offsets)) return AA_ERR_INVALID_ARG;
    if (a->head_dim > 256 || a->heads > 65535 || a->n_seq > 0x7FFFFFFFll || a->max_q > 0x3FFFFFFFll || a->max_k > 0x3FFFFFFFll) return AA_ERR_UNSUPPORTED;
    if (check_tokens(a->q, es, a->q_rows, a->heads, a->head_dim, false) != AA_OK || check_tokens(a->k, es, a->k_rows, a->kv_heads, a->head_dim, false) != AA_OK ||
        check_tokens(a->v, es, a->k_rows, a->kv_heads, a->head_dim, false) != AA_OK)
        return AA_ERR_INVALID_ARG;
    memset(&p, 0, sizeof p);
    p.q = tok(a->q);
    p.k = tok(a->k);
    p.v = tok(a->v);
    p.heads = a->heads;
    p.kv_heads = a->kv_heads;
    p.group = a->heads / a->kv_heads;
    p.dim = a->head_dim;
    p.causal = a->causal != 0;
    p.scale = a->scale;
    p.scale2 = a->scale * kAttnLog2e;
    p.n_seq = a->n_seq;
    p.q_rows = a->q_rows;
    p.k_rows = a->k_rows;
    // a bound above the stored tokens says nothing more than they do
    p.max_q = a->max_q < a->q_rows ? a->max_q : a->q_rows;
    p.max_k = a->max_k < a->k_rows ? a->max_k : a->k_rows;
    p.q_off = a->q_offsets;
    p.k_off = a->k_offsets;
    p.count_dev = a->count_dev;
    if (b) {
        if (!b->table) return AA_ERR_INVALID_ARG;
        if (!rel_bucket_bounds(b, &p.per_dir, p.lower)) return AA_ERR_INVALID_ARG;
        p.table = b->table;
        p.buckets = b->buckets;
        p.bidir = b->bidirectional != 0;
        p.reach = p.lower[p.per_dir - 1];
    }
    return make_drop_rule(d, p.drop) ? AA_OK : AA_ERR_INVALID_ARG;
}

bool rel_bf16_fits(const RelParams& p) {
    const auto ok = [&](const TokArg& a) { return !a.data || ((uintptr_t)a.data % 16 == 0 && a.tok % 8 == 0 && a.head % 8 == 0 && a.tok < (1 << 30)); };
    return p.dim % 8 == 0 && p.dim <= 128 && ok(p.q) && ok(p.k) && ok(p.v) && ok(p.out) && ok(p.dout) && ok(p.dq) && ok(p.dk) && ok(p.dv);
}

// A few new tokens: split over the context.  Sentences: a CTA each.  What is longer: tiles on the tcgen05 tensor cores.
aa_status launch_rel_attention_bf16(aa_ctx_impl* c, const RelParams& p) {
    if (rel_decode_fits(p)) return launch_rel_decode(c, p);
    int covered = -1;
    const aa_status st = launch_rel_sentences(c, p, &covered);
    if (st != AA_OK || (p.max_q <= covered && p.max_k <= covered)) return st;
    return launch_rel_attention_tc(c, p, covered);
}

aa_status launch_rel_attention_grad_bf16(aa_ctx_impl* c, const RelParams& p, int* n_parts) {
    *n_parts = 0;
    int covered = -1;
    const aa_status st = launch_rel_sentences_grad(c, p, &covered, n_parts);
    if (st != AA_OK || (p.max_q <= covered && p.max_k <= covered)) return st;
    return launch_rel_attention_grad_tc(c, p, covered, n_parts);
}

int rel_grad_parts(int heads) { return (1184 + heads - 1) / heads; }

namespace {

size_t stats_bytes(const aa_attn* a) { return ((size_t)a->heads * (size_t)a->q_rows * sizeof(float4) + 255) / 256 * 256; }

}  // namespace
}  // namespace aa

using namespace aa;

extern "C" {

aa_status aa_dropout(aa_ctx* ctx, const aa_rows* x, const aa_dropout_rule* rule, const int32_t* offsets, int64_t n_seg, const int32_t* count_dev,
                     const aa_rows* residual, const aa_rows* out) {
    if (!ctx || !rule || check_rows(x) != AA_OK || check_rows(out) != AA_OK || !same_shape(*x, *out)) return AA_ERR_INVALID_ARG;
    if (residual && (check_rows(residual) != AA_OK || !same_shape(*x, *residual))) return AA_ERR_INVALID_ARG;
    if (offsets ? n_seg < 0 : n_seg != 0) return AA_ERR_INVALID_ARG;
    if (x->cols > kMaxDropoutCols) return AA_ERR_UNSUPPORTED;
    DropParams p = {};
    if (!make_drop_rule(rule, p.rule)) return AA_ERR_INVALID_ARG;
    if (x->rows == 0 || (offsets && n_seg == 0)) return AA_OK;
    const int64_t es = x->dtype == AA_BF16 ? 2 : 4;
    if (!same_or_apart(x->data, x->row_stride, out->data, out->row_stride, x->rows, x->cols, es)) return AA_ERR_INVALID_ARG;
    if (residual && !same_or_apart(residual->data, residual->row_stride, out->data, out->row_stride, x->rows, x->cols, es)) return AA_ERR_INVALID_ARG;
    p.x = {x->data, x->row_stride};
    p.out = {out->data, out->row_stride};
    if (residual) p.res = {residual->data, residual->row_stride};
    p.rows = x->rows;
    p.cols = x->cols;
    p.offsets = offsets;
    p.n_inst = offsets ? n_seg : x->rows;
    p.count_dev = count_dev;
    p.ctl = reinterpret_cast<aa_ctx_impl*>(ctx)->ctl;
    return launch_dropout(reinterpret_cast<aa_ctx_impl*>(ctx), p, x->dtype);
}

aa_status aa_instance_loss_grad(aa_ctx* ctx, const aa_logits* lg, const int32_t* labels, const int32_t* offsets, int64_t n_seg,
                                const int32_t* count_dev, const float* weight, float scale, int32_t reduce_mode, float* out_loss, const aa_rows* grad) {
    if (!ctx || !lg || check_rows(grad) != AA_OK) return AA_ERR_INVALID_ARG;
    const aa_rows as_rows = {const_cast<void*>(lg->data), lg->dtype, 0, lg->rows, lg->cols, lg->row_stride};
    if (check_rows(&as_rows) != AA_OK || !same_shape(as_rows, *grad) || (lg->rows > 0 && !labels)) return AA_ERR_INVALID_ARG;
    if (offsets ? n_seg < 0 : n_seg != 0) return AA_ERR_INVALID_ARG;
    if (reduce_mode != AA_REDUCE_SUM && reduce_mode != AA_REDUCE_MEAN) return AA_ERR_INVALID_ARG;
    const int64_t es = lg->dtype == AA_BF16 ? 2 : 4;
    if (lg->rows > 0 && !same_or_apart(lg->data, lg->row_stride, grad->data, grad->row_stride, lg->rows, lg->cols, es)) return AA_ERR_INVALID_ARG;
    aa_ctx_impl* c = reinterpret_cast<aa_ctx_impl*>(ctx);
    if (offsets && out_loss && lg->rows > c->max_rows) return AA_ERR_WORKSPACE;
    return launch_instance_loss_grad(c, *lg, labels, offsets, n_seg, count_dev, weight, scale, reduce_mode == AA_REDUCE_MEAN, out_loss, *grad);
}

int32_t aa_rel_bucket(const aa_rel_bias* bias, int64_t delta) {
    int per_dir, lower[kMaxPerDir];
    if (!bias || !rel_bucket_bounds(bias, &per_dir, lower)) return -1;
    const int64_t n = bias->bidirectional ? (delta < 0 ? -delta : delta) : (delta < 0 ? -delta : 0);
    int k = 0;
    while (k + 1 < per_dir && lower[k + 1] <= n) ++k;
    return k + (bias->bidirectional && delta > 0 ? per_dir : 0);
}

aa_status aa_rel_attention(aa_ctx* ctx, const aa_attn* attn, const aa_rel_bias* bias, const aa_dropout_rule* dropout, const aa_tokens* out) {
    if (!ctx || !out) return AA_ERR_INVALID_ARG;
    RelParams p;
    aa_status st = make_rel_params(attn, bias, dropout, p);
    if (st != AA_OK) return st;
    const int64_t es = attn->dtype == AA_BF16 ? 2 : 4;
    if ((st = check_tokens(*out, es, p.q_rows, p.heads, p.dim, true)) != AA_OK) return st;
    // the output may take the queries' place: whoever writes a row has read it, and nobody else reads it
    const Extent o = query_extent(*out, p);
    const bool in_place = out->data == attn->q.data && (p.q_rows <= 1 || out->token_stride == attn->q.token_stride) && (p.heads == 1 || out->head_stride == attn->q.head_stride);
    if ((!in_place && !apart(o, query_extent(attn->q, p), es)) || !apart(o, key_extent(attn->k, p), es) || !apart(o, key_extent(attn->v, p), es)) return AA_ERR_INVALID_ARG;
    if (p.n_seq == 0) return AA_OK;
    aa_ctx_impl* c = reinterpret_cast<aa_ctx_impl*>(ctx);
    p.out = tok(*out);
    p.ctl = c->ctl;
    // a bound of zero leaves only the sequences to be looked over, which the fp32 kernel does
    return attn->dtype == AA_BF16 && p.max_q > 0 && rel_bf16_fits(p) ? launch_rel_attention_bf16(c, p) : launch_rel_attention_plain(c, p, attn->dtype);
}

aa_status aa_rel_attention_scratch_bytes(const aa_attn* attn, const aa_rel_bias* bias, size_t* bytes) {
    if (!bytes) return AA_ERR_INVALID_ARG;
    RelParams p;
    const aa_status st = make_rel_params(attn, bias, nullptr, p);
    if (st != AA_OK) return st;
    // up to three launches (short, middle and long sequences) leave partial sums of the table's gradient
    *bytes = stats_bytes(attn) + 3 * (size_t)rel_grad_parts(p.heads) * (size_t)p.heads * (size_t)p.buckets * sizeof(float);
    return AA_OK;
}

aa_status aa_rel_attention_grad(aa_ctx* ctx, const aa_attn* attn, const aa_rel_bias* bias, const aa_dropout_rule* dropout, const aa_tokens* dout,
                                const aa_tokens* dq, const aa_tokens* dk, const aa_tokens* dv, float* dtable, void* scratch, size_t scratch_bytes) {
    if (!ctx || !dout || !dq || !dk || !dv || (dtable && !bias)) return AA_ERR_INVALID_ARG;
    RelParams p;
    aa_status st = make_rel_params(attn, bias, dropout, p);
    if (st != AA_OK) return st;
    const int64_t es = attn->dtype == AA_BF16 ? 2 : 4;
    if ((st = check_tokens(*dout, es, p.q_rows, p.heads, p.dim, false)) != AA_OK || (st = check_tokens(*dq, es, p.q_rows, p.heads, p.dim, true)) != AA_OK ||
        (st = check_tokens(*dk, es, p.k_rows, p.kv_heads, p.dim, true)) != AA_OK || (st = check_tokens(*dv, es, p.k_rows, p.kv_heads, p.dim, true)) != AA_OK)
        return st;
    // gradients are written while operands are still to be read (those of long sequences by a later kernel): nothing in common
    const Extent in[4] = {query_extent(attn->q, p), key_extent(attn->k, p), key_extent(attn->v, p), query_extent(*dout, p)};
    const Extent to[3] = {query_extent(*dq, p), key_extent(*dk, p), key_extent(*dv, p)};
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < 4; ++j)
            if (!apart(to[i], in[j], es)) return AA_ERR_INVALID_ARG;
        for (int j = 0; j < i; ++j)
            if (!apart(to[i], to[j], es)) return AA_ERR_INVALID_ARG;
    }
    size_t need = 0;
    if ((st = aa_rel_attention_scratch_bytes(attn, bias, &need)) != AA_OK) return st;
    if (need > 0 && (!scratch || (uintptr_t)scratch % 256)) return AA_ERR_INVALID_ARG;
    if (scratch_bytes < need) return AA_ERR_WORKSPACE;
    aa_ctx_impl* c = reinterpret_cast<aa_ctx_impl*>(ctx);
    if (p.n_seq == 0)
        return dtable ? cuda_ok(cudaMemsetAsync(dtable, 0, sizeof(float) * (size_t)p.buckets * (size_t)p.heads, c->stream)) : AA_OK;
    p.dout = tok(*dout);
    p.dq = tok(*dq);
    p.dk = tok(*dk);
    p.dv = tok(*dv);
    p.dtable = dtable;
    p.ctl = c->ctl;
    p.stats = static_cast<float4*>(scratch);
    p.parts = reinterpret_cast<float*>(static_cast<char*>(scratch) + stats_bytes(attn));
    p.n_parts = rel_grad_parts(p.heads);
    st = attn->dtype == AA_BF16 && (p.max_q > 0 || p.max_k > 0) && rel_bf16_fits(p) ? launch_rel_attention_grad_bf16(c, p, &p.n_parts) : launch_rel_attention_grad_plain(c, p, attn->dtype);
    if (st != AA_OK || !dtable) return st;
    return launch_rel_table_grad(c, p);
}

}  // extern "C"
