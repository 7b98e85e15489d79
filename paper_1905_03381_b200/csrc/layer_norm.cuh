// Arguments of the layer normalisation kernels.
#pragma once

#include "linear.cuh"

namespace aa {

constexpr int kNormParts = 592;              // CTAs that leave column sums, at most
constexpr int kSweepParts = 64;
constexpr int64_t kNormInRegisters = 8192;   // columns of the longest row that stays in registers

// Of a row too long for registers: its mean (mean + d, more exactly) and 1 / sqrt(var + eps).
struct alignas(16) NormStats {
    float mean, d, r, unused;
#ifdef __CUDACC__
    __device__ __forceinline__ float h(float x) const { return (x - mean - d) * r; }
#endif
};

struct NormParams {
    MatArg x, dout, residual, out;           // dout: gradients only; residual nullable
    int64_t cols;
    LiveRows live;
    const float* gamma;                      // nullable
    const float* beta;
    float eps;
    float* parts;                            // column sums, [parts][2][cols]; null: neither dgamma nor dbeta is wanted
    NormStats* stats;                          // [rows] (rows longer than kNormInRegisters)
    Control* ctl;
};

size_t norm_scratch_floats(int64_t rows, int64_t cols);   // of parts
aa_status launch_layer_norm(aa_ctx_impl* c, const NormParams& p, int dtype, bool grad, float* dgamma, float* dbeta);

}  // namespace aa
