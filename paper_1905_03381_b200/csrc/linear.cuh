// Linear layers of the Boss: what the kernels of the forward call and of the two products of the backward call share.
//
// Every product is C[m][n] = sum_k A(m, k) B(n, k) on matrices stored by rows:
//   out = x w^T   : A = x, B = w, both with the contraction along their rows;
//   dx  = G w     : A = G, contraction along its rows; B(n, k) = w[k][n], contraction across w's rows;
//   dw  = G^T x   : A(m, k) = G[k][m], B(n, k) = x[k][n], contraction across the rows of both, which are the tokens.
#pragma once

#include "boss_common.cuh"

namespace aa {

// The rows of a batch that are evaluated (see the header: R).
struct LiveRows {
    const int32_t* offsets;
    int64_t n_seg;
    const int32_t* count_dev;
    int64_t rows;
};

struct MatArg {              // rows of one matrix
    const void* data;
    int64_t stride;          // elements
};

struct ProductParams {
    MatArg a, b;
    bool a_across, b_across; // the contraction runs across the stored rows of A, of B
    int64_t m, n, k;
    LiveRows live;           // bounds m, or k if both operands are stored by token
    bool live_k;
    const float* bias;       // [n], nullable
    int act;                 // aa_activation
    MatArg residual, pre, out;   // nullable but out
    float* parts;            // scratch for tiles cut along the contraction, nullable (then bias, act and pre are empty)
    int64_t part_floats;
    Control* ctl;
};

aa_status launch_product(aa_ctx_impl* c, const ProductParams& p, int dtype);
// bf16 operands that TMA can fetch (16-byte aligned bases and rows).
bool product_tc_fits(const ProductParams& p);
aa_status launch_product_tc(aa_ctx_impl* c, const ProductParams& p);
// g = dout * act'(pre), rounded to the matrices' type; column sums of the unrounded g (or of dout alone where act is AA_ACT_NONE and g null) into dbias.
struct SlopeParams {
    MatArg dout, pre, g;
    int64_t rows, cols;
    LiveRows live;
    int act;
    float* parts;            // [kSlopeParts][cols] (dbias not null)
    float* dbias;            // nullable
    Control* ctl;
};
constexpr int kSlopeParts = 148;
aa_status launch_slope(aa_ctx_impl* c, const SlopeParams& p, int dtype);

#ifdef __CUDACC__

// R.  `tell`: this thread latches a bad offset.
__device__ __forceinline__ int64_t live_rows(const LiveRows& l, Control* ctl, bool tell) {
    if (!l.offsets) return counted(l.count_dev, l.rows);
    const int64_t m = counted(l.count_dev, l.n_seg);
    if (m == 0) return 0;
    const int64_t r = l.offsets[m];
    if (r >= 0 && r <= l.rows) return r;
    if (tell) latch(ctl, AA_ERR_BAD_INDEX);
    return 0;
}

__device__ __forceinline__ float activate(float z, int act) {
    if (act == AA_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if (act == AA_ACT_GELU) return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
    if (act == AA_ACT_SILU) return z / (1.0f + expf(-z));
    return z;
}

// act'(z); relu'(0) = 0.
__device__ __forceinline__ float activation_slope(float z, int act) {
    if (act == AA_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if (act == AA_ACT_GELU) return 0.5f * (1.0f + erff(z * 0.70710678118654752f)) + z * expf(-0.5f * z * z) * 0.39894228040143268f;
    if (act == AA_ACT_SILU) {
        const float s = 1.0f / (1.0f + expf(-z));
        return s * (1.0f + z * (1.0f - s));
    }
    return 1.0f;
}

#endif  // __CUDACC__

}  // namespace aa
