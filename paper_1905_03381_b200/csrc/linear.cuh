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
    int64_t plane_a, plane_b;    // above 0: A and B are three planes of bf16 terms of fp32 numbers, so many elements apart
    float* a_sums;           // [m] sums of A over the contraction, nullable (a_across)
    Control* ctl;
};

aa_status launch_product(aa_ctx_impl* c, const ProductParams& p, int dtype);
// bf16 operands that TMA can fetch (16-byte aligned bases and rows).
bool product_tc_fits(const ProductParams& p);
aa_status launch_product_tc(aa_ctx_impl* c, const ProductParams& p);
// At most 16 rows, forward.
bool product_few_fits(const ProductParams& p);
aa_status launch_product_few(aa_ctx_impl* c, const ProductParams& p, int dtype);
// fp32 operands taken apart beforehand (plane_a, plane_b).
aa_status launch_product_planes(aa_ctx_impl* c, const ProductParams& p);
aa_status launch_product_split(aa_ctx_impl* c, const ProductParams& p, int dtype);
// g = dout * act'(pre), rounded to the matrices' type (null: not written); column sums of the unrounded g into dbias.
struct SlopeParams {
    MatArg dout, pre, g;
    int64_t plane;           // above 0: g is bf16 terms (three of fp32, one of bf16) in planes so many elements apart, rows padded to a multiple of 8 elements
    int64_t rows, cols;
    LiveRows live;
    int act;
    float* parts;            // [kSlopeParts][cols] (dbias not null)
    float* dbias;            // nullable
    Control* ctl;
};
constexpr int kSlopeParts = 148;
// n passes, one or up to kSlopeJobs copies (plane above 0), of which the first may have an activation and dbias.
constexpr int kSlopeJobs = 3;
aa_status launch_slopes(aa_ctx_impl* c, const SlopeParams* p, int n, int dtype);

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

__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Normal distribution at z and its density's exponential e = exp(-z^2 / 2), which the gradient needs too.  FINE (fp32 matrices): by the functions of the library, good to
// a few parts in 2^24.  Otherwise (results that are rounded to bf16) the tail is Hastings' rational approximation (Abramowitz and Stegun, 7.1.26):
// erfc(x) = (a1 t + ... + a5 t^5) exp(-x^2), t = 1 / (1 + 0.3275911 x), within 1.5e-7 (5e-4 of the tail down to z = -4, 4e-3 at -6); it shares e
// (8,000 x 256 -> 2,048 fp32 with GELU takes 92 us by it, 111 by the functions).
template <bool FINE>
__device__ __forceinline__ float normal_cdf(float z, float& e) {
    const float x = fabsf(z) * 0.70710678118654752f;
    float q;
    if (FINE) {
        e = expf(-0.5f * z * z);
        q = 0.5f * erfcf(x);
    } else {
        const float t = rcp_approx(fmaf(0.3275911f, x, 1.0f));
        e = ex2_approx(z * z * -0.72134752044448170f);
        q = fmaf(t, 1.061405429f, -1.453152027f);
        q = fmaf(t, q, 1.421413741f);
        q = fmaf(t, q, -0.284496736f);
        q = fmaf(t, q, 0.254829592f);
        q = 0.5f * t * q * e;
    }
    return z > 0.0f ? 1.0f - q : q;
}
template <bool FINE>
__device__ __forceinline__ float logistic(float z) {
    return rcp_approx(1.0f + (FINE ? expf(-z) : ex2_approx(z * -1.4426950408889634f)));
}

template <int ACT, bool FINE>
__device__ __forceinline__ float activate(float z) {
    if (ACT == AA_ACT_RELU) return z < 0.0f ? 0.0f : z;
    float e;
    if (ACT == AA_ACT_GELU) return z * normal_cdf<FINE>(z, e);
    if (ACT == AA_ACT_SILU) return z * logistic<FINE>(z);
    return z;
}
// The same where the activation is known at run time: one branch for N values.
template <bool FINE, int N>
__device__ __forceinline__ void activate_all(float (&z)[N], int act) {
    if (act == AA_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = activate<AA_ACT_RELU, FINE>(z[i]);
    } else if (act == AA_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = activate<AA_ACT_GELU, FINE>(z[i]);
    } else if (act == AA_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = activate<AA_ACT_SILU, FINE>(z[i]);
    }
}

// act'(z); relu'(0) = 0.
template <int ACT, bool FINE>
__device__ __forceinline__ float activation_slope(float z) {
    if (ACT == AA_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if (ACT == AA_ACT_GELU) {
        float e;
        const float cdf = normal_cdf<FINE>(z, e);
        return fmaf(z * 0.39894228040143268f, e, cdf);
    }
    if (ACT == AA_ACT_SILU) {
        const float s = logistic<FINE>(z);
        return s * fmaf(z, 1.0f - s, 1.0f);
    }
    return 1.0f;
}

#endif  // __CUDACC__

}  // namespace aa
