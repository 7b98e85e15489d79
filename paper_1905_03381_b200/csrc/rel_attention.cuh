// Attention over ragged sequences with a learned relative position bias: parameters, the bias by distance, the draws of its dropout
// and the tile bookkeeping that the kernels share.
//
// Scores are kept in base 2:  t_ij = scale log2(e) q_i.k_j + log2(e) table[bucket(delta)][h],  p_ij = 2^(t_ij - m_i) / l_i.
// A finite bias is clamped to +-3e38 after the change of base, so that the type's lowest value stays a finite mask.
#pragma once

#include "boss_common.cuh"

namespace aa {

constexpr int kMaxPerDir = 128;          // buckets per direction
constexpr int kMaxReach = 2048;          // largest max_distance
constexpr float kAttnLog2e = 1.4426950408889634f;

struct TokArg {
    const void* data;
    int64_t tok, head;                   // strides in elements
};

struct RelParams {
    TokArg q, k, v, out, dout, dq, dk, dv;
    int heads, kv_heads, group, dim, causal;
    float scale2;                        // scale * log2(e)
    float scale;
    int64_t n_seq, q_rows, k_rows, max_q, max_k;
    const int32_t* q_off;
    const int32_t* k_off;
    const int32_t* count_dev;
    // bias: distances below `reach` have an entry each in the kernels' distance table, the rest are the last bucket's
    const float* table;                  // nullable
    int buckets, per_dir, bidir, reach;
    int lower[kMaxPerDir];               // first distance of every bucket of a direction
    DropRule drop;
    Control* ctl;
    // backward
    float4* stats;                       // [heads][q_rows]: m, 1 / l, D
    float* parts;                        // [n_parts][heads][buckets] partial sums of the table's gradient
    int n_parts;
    float* dtable;                       // nullable
};

// First distances of the buckets of one direction; false: malformed.
bool rel_bucket_bounds(const aa_rel_bias* b, int* per_dir, int* lower);
// Shapes and offsets of one problem; AA_OK or the argument error.
aa_status make_rel_params(const aa_attn* a, const aa_rel_bias* b, const aa_dropout_rule* d, RelParams& p);
int rel_grad_parts(int heads);                                       // CTAs per head that share the table's gradient

aa_status launch_rel_attention_plain(aa_ctx_impl* c, const RelParams& p, int dtype);
aa_status launch_rel_attention_grad_plain(aa_ctx_impl* c, const RelParams& p, int dtype);
// bf16 kernels on the tensor cores: aligned tokens, head width a multiple of 8 up to 128.
bool rel_bf16_fits(const RelParams& p);
aa_status launch_rel_attention_bf16(aa_ctx_impl* c, const RelParams& p);
// ... of them the sequences of more than `lo` tokens on either side, on the tcgen05 tensor cores
aa_status launch_rel_attention_tc(aa_ctx_impl* c, const RelParams& p, int lo);
// ... a few new tokens over long contexts
bool rel_decode_fits(const RelParams& p);
aa_status launch_rel_decode(aa_ctx_impl* c, const RelParams& p);
// ... of them the sequences of at most *covered tokens on both sides (set by the call; -1: none)
aa_status launch_rel_sentences(aa_ctx_impl* c, const RelParams& p, int* covered);
aa_status launch_rel_sentences_grad(aa_ctx_impl* c, const RelParams& p, int* covered, int* n_parts);
aa_status launch_rel_attention_grad_tc(aa_ctx_impl* c, const RelParams& p, int lo, int* n_parts);
aa_status launch_rel_attention_grad_bf16(aa_ctx_impl* c, const RelParams& p, int* n_parts);
aa_status launch_rel_table_grad(aa_ctx_impl* c, const RelParams& p);  // parts -> dtable

#ifdef __CUDACC__

struct Seq {
    int64_t q0, k0;                      // first tokens
    int lq, lk;
};

// Sequence s; false: not counted, or its offsets are bad (latched).
__device__ __forceinline__ bool load_seq(const RelParams& p, int64_t s, Seq& q) {
    if (s >= counted(p.count_dev, p.n_seq)) return false;
    const int a = p.q_off[s], b = p.q_off[s + 1], c = p.k_off[s], d = p.k_off[s + 1];
    if (a < 0 || b < a || b > p.q_rows || b - a > p.max_q || c < 0 || d < c || d > p.k_rows || d - c > p.max_k) {
        latch(p.ctl, AA_ERR_BAD_INDEX);
        return false;
    }
    q.q0 = a;
    q.lq = b - a;
    q.k0 = c;
    q.lk = d - c;
    return true;
}

// Base-2 bias by distance for head h: bias[delta + reach + MARGIN]; the ends beyond the reach repeat the last buckets' values for MARGIN
// distances, so that a tile that touches the reach needs no clamping.  A warp per bucket: the bounds are read at one address.
template <int MARGIN>
__device__ __forceinline__ void fill_bias(const RelParams& p, int h, float* bias, int warps, int self) {      // `warps` warps call, this one as the self-th
    if (!p.table) return;
    const int lane = threadIdx.x & 31;
    float* zero = bias + p.reach + MARGIN;
    for (int b0 = 0; b0 < p.buckets; b0 += 32) {
        float v = 0.0f;                                                 // a lane per bucket: one trip to memory for 32 of them
        if (b0 + lane < p.buckets) {
            const float x = p.table[(int64_t)(b0 + lane) * p.heads + h];
            v = isinf(x) || isnan(x) ? x : fminf(fmaxf(x * kAttnLog2e, -3.0e38f), 3.0e38f);
        }
        const int b1 = min(p.buckets - b0, 32);
        for (int i = self; i < b1; i += warps) {
            const float x = __shfl_sync(0xFFFFFFFFu, v, i);
            const bool up = b0 + i >= p.per_dir;
            const int k = up ? b0 + i - p.per_dir : b0 + i;
            const int end = k == p.per_dir - 1 ? p.reach + MARGIN + 1 : p.lower[k + 1];
            for (int n = max(p.lower[k], up ? 1 : 0) + lane; n < end; n += 32) zero[up ? n : -n] = x;
            if (!p.bidir && k == 0)                                     // one direction: later keys count as distance 0
                for (int n = 1 + lane; n <= p.reach + MARGIN; n += 32) zero[n] = x;
        }
    }
}
template <int MARGIN>
__device__ __forceinline__ void fill_bias(const RelParams& p, int h, float* bias) {
    fill_bias<MARGIN>(p, h, bias, (int)(blockDim.x >> 5), (int)(threadIdx.x >> 5));
}
__host__ __device__ constexpr int bias_floats(int reach, int margin) { return 2 * (reach + margin) + 1; }
__device__ __forceinline__ float bias_at(const RelParams& p, const float* bias, int delta) {      // a table without margins
    return p.table ? bias[min(max(delta, -p.reach), p.reach) + p.reach] : 0.0f;
}

// Number of the first draw block of query row i, head h.
__device__ __forceinline__ uint64_t draw_row(const Seq& s, int h, int i) {
    return ((uint64_t)h * (uint64_t)s.lq + (uint64_t)i) * (uint64_t)((s.lk + 31) >> 5) * 4ull;
}

// Keys [0, n) that some query of rows [i0, i1) sees.
__device__ __forceinline__ int keys_seen(const RelParams& p, const Seq& s, int i1) {
    return p.causal ? max(0, min(s.lk, i1 + s.lk - s.lq)) : s.lk;
}
// First query row that sees key j.
__device__ __forceinline__ int first_query(const RelParams& p, const Seq& s, int j) {
    return p.causal ? max(0, j - (s.lk - s.lq)) : 0;
}

// Partial sums of the table's gradient by distance, then by bucket.  Distances inside the table's reach have a bin of their own,
// [delta + reach] for -reach < delta < reach (and delta <= 0 when one-directional); the rest are summed per side.
struct FarSums {
    float neg, pos;
};
__device__ __forceinline__ void bin_diagonal(const RelParams& p, float* bins, FarSums& far, int delta, float sum) {
    if (delta <= -p.reach) far.neg += sum;
    else if (delta >= p.reach || (!p.bidir && delta > 0)) far.pos += sum;
    else bins[delta + p.reach] += sum;
}

// Bins -> one CTA's partial sums by bucket.  `copies` arrays `pitch` floats apart, each 2 reach bins, then n_far sums of the far past and
// n_far of the far future (visible to the CTA).  A warp per bucket, lanes over its distances, joined in a fixed order.
__device__ __forceinline__ void write_table_part(const RelParams& p, int64_t index, int h, const float* bins, int pitch, int copies, int n_far) {
    float* part = p.parts + (index * p.heads + h) * p.buckets;
    const int lane = threadIdx.x & 31;
    for (int b = threadIdx.x >> 5; b < p.buckets; b += blockDim.x >> 5) {
        const bool up = b >= p.per_dir;
        const int k = up ? b - p.per_dir : b;
        const bool last = k == p.per_dir - 1;
        const int hi = last ? p.reach : p.lower[k + 1];                 // distances [lower[k], hi); up: delta > 0
        double sum = 0.0;
        for (int c = 0; c < copies; ++c) {
            const float* one = bins + c * pitch;
            const float* far_neg = one + 2 * p.reach;
            for (int n = max(p.lower[k], up ? 1 : 0) + lane; n < hi; n += 32) sum += (double)one[p.reach + (up ? n : -n)];
            if (last)
                for (int i = lane; i < n_far; i += 32) sum += (double)far_neg[i + (up ? n_far : 0)];
            if (!p.bidir && k == 0)                                     // delta > 0 counts as 0
                for (int i = lane; i < n_far; i += 32) sum += (double)far_neg[i + n_far];
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        if (lane == 0) part[b] = (float)sum;
    }
}

#endif  // __CUDACC__

}  // namespace aa
