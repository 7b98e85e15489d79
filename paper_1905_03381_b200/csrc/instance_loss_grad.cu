// Gradient of the weighted instance losses with respect to the logits:  G_rc = g_r (softmax(x_r)_c - [c = y_r]).
//
// Two sweeps over a row: the running maximum and sum of the one-pass log-sum-exp, then the gradient.  LPR lanes (short rows) or a CTA
// (long rows) own a row, so the second sweep finds it in L1 or L2.
#include "boss_common.cuh"
#include "loss_common.cuh"

namespace aa {

namespace {

struct GradParams {
    LossParams loss;         // logits, rows, cols, labels; out = row losses (nullable); count_dev unused
    const int32_t* offsets;
    int64_t n_inst;
    const int32_t* count_dev;
    const float* weight;
    float scale;
    int mean;
    void* grad;
    int64_t grad_stride;
};

// The factor g_r of row r, or false where no counted instance holds the row.
__device__ __forceinline__ bool row_factor(const GradParams& p, int64_t n_inst, int64_t r, float& g) {
    int64_t inst = r;
    if (p.offsets) {
        if (n_inst == 0) return false;
        inst = find_segment(p.offsets, n_inst, r);
        // empty segments share their start with the next one; the search ends at the last of them
        if (r < __ldg(p.offsets + inst) || r >= __ldg(p.offsets + inst + 1)) return false;
    } else if (r >= n_inst) {
        return false;
    }
    g = p.scale;
    if (p.mean) g = g / (float)n_inst;
    if (p.weight) g *= __ldg(p.weight + inst);
    return true;
}

// Running maximum and sum of a row in the logits' own scale: exponents are 2^((x - m) log2 e), so that logits near the type's limits do not
// overflow in a change of base (one subtraction more per element than the loss kernels' fused form; these kernels have the room).
struct NatState {
    float m, s;
};
__device__ __forceinline__ float exp_from(float x, float m) { return ex2_approx((x - m) * kLog2e); }
template <int N>
__device__ __forceinline__ void absorb_nat(NatState& st, const float (&x)[N]) {
    float top = x[0];
#pragma unroll
    for (int e = 1; e < N; ++e) top = fmaxf(top, x[e]);
    if (top > st.m) {
        st.s *= exp_from(st.m, top);       // st.m = -inf gives 0 * 0
        st.m = top;
    }
    const float ref = st.m == -INFINITY ? 0.0f : st.m;      // only -inf so far: every term is 0
    float a = 0.0f, b = 0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) (e & 1 ? b : a) += exp_from(x[e], ref);
    st.s += a + b;
}
__device__ __forceinline__ NatState merge(const NatState& a, const NatState& b) {
    const float m = fmaxf(a.m, b.m), ref = m == -INFINITY ? 0.0f : m;
    return NatState{m, a.s * exp_from(a.m, ref) + b.s * exp_from(b.m, ref)};
}
template <int WIDTH>
__device__ __forceinline__ NatState group_merge_nat(NatState st) {
#pragma unroll
    for (int o = WIDTH / 2; o > 0; o >>= 1)
        st = merge(st, NatState{__shfl_xor_sync(0xFFFFFFFFu, st.m, o), __shfl_xor_sync(0xFFFFFFFFu, st.s, o)});
    return st;
}
__device__ __forceinline__ float row_loss(const NatState& st, float label_logit) { return (st.m - label_logit) + lg2_approx(st.s) * kLn2; }

// First sweep: elements rank, rank + nthreads, ... in 16-byte vectors between the row's 16-byte boundaries.
template <typename T>
__device__ __forceinline__ void scan_row_nat(NatState& st, const T* row, int64_t cols, int rank, int nthreads) {
    constexpr int VE = Vec<T>::kElems;
    int64_t head = ((16 - ((uintptr_t)row & 15)) & 15) / sizeof(T);
    if (head > cols) head = cols;
    const int64_t nvec = (cols - head) / VE;
    int64_t v = rank;
    for (; v + 3 * (int64_t)nthreads < nvec; v += 4 * (int64_t)nthreads) {
        float x[4 * VE];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float y[VE];
            Vec<T>::unpack(*reinterpret_cast<const uint4*>(row + head + (v + k * (int64_t)nthreads) * VE), y);
#pragma unroll
            for (int e = 0; e < VE; ++e) x[k * VE + e] = y[e];
        }
        absorb_nat(st, x);
    }
    for (; v < nvec; v += nthreads) {
        float x[VE];
        Vec<T>::unpack(*reinterpret_cast<const uint4*>(row + head + v * VE), x);
        absorb_nat(st, x);
    }
    for (int64_t c = rank; c < head; c += nthreads) {
        const float x[1] = {load1(row + c)};
        absorb_nat(st, x);
    }
    for (int64_t c = head + nvec * VE + rank; c < cols; c += nthreads) {
        const float x[1] = {load1(row + c)};
        absorb_nat(st, x);
    }
}

// Second sweep, a = g / sum: elements rank, rank + nthreads, ... in 16-byte vectors where both rows are aligned alike.
template <typename T>
__device__ __forceinline__ void write_row(const T* row, T* out, int64_t cols, float m, float a, float g, int y, int rank, int nthreads) {
    constexpr int VE = Vec<T>::kElems;
    const auto at = [&](float x, int64_t c) { return fmaf(a, exp_from(x, m), c == y ? -g : 0.0f); };
    int64_t head = cols, nvec = 0;
    if ((((uintptr_t)row ^ (uintptr_t)out) & 15) == 0) {
        head = ((16 - ((uintptr_t)row & 15)) & 15) / sizeof(T);
        if (head > cols) head = cols;
        nvec = (cols - head) / VE;
    }
    for (int64_t v = rank; v < nvec; v += nthreads) {
        const int64_t c = head + v * VE;
        float x[VE];
        Vec<T>::unpack(*reinterpret_cast<const uint4*>(row + c), x);
#pragma unroll
        for (int e = 0; e < VE; ++e) x[e] = at(x[e], c + e);
        if constexpr (VE == 8) store8(out + c, x);
        else *reinterpret_cast<float4*>(out + c) = make_float4(x[0], x[1], x[2], x[3]);
    }
    for (int64_t c = rank; c < head; c += nthreads) store1(out + c, at(load1(row + c), c));
    for (int64_t c = head + nvec * VE + rank; c < cols; c += nthreads) store1(out + c, at(load1(row + c), c));
}

template <typename T>
__device__ __forceinline__ void zero_row(T* out, int64_t cols, int rank, int nthreads) {
    for (int64_t c = rank; c < cols; c += nthreads) store1(out + c, 0.0f);
}

template <typename T, int LPR>
__global__ void __launch_bounds__(256) row_grad_group_kernel(GradParams p) {
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t n_inst = counted(p.count_dev, p.n_inst);
    if (p.offsets && blockIdx.x == 0) check_offsets(p.loss.ctl, p.offsets, n_inst, p.loss.rows);
    const int gl = threadIdx.x % LPR;
    const int64_t groups_per_grid = (int64_t)gridDim.x * (blockDim.x / LPR);
    const int64_t group0 = (int64_t)blockIdx.x * (blockDim.x / LPR) + threadIdx.x / LPR;
    const int64_t rounds = (p.loss.rows + groups_per_grid - 1) / groups_per_grid;   // whole warps iterate together (shuffles)
    for (int64_t it = 0; it < rounds; ++it) {
        const int64_t r = group0 + it * groups_per_grid;
        float g = 0.0f;
        const bool live = r < p.loss.rows && row_factor(p, n_inst, r, g);
        const int y = live ? checked_label(p.loss, r) : -1;
        const T* row = static_cast<const T*>(p.loss.logits) + (live ? r : 0) * p.loss.row_stride;
        NatState st = {-INFINITY, 0.0f};
        float label_logit = 0.0f;
        if (y >= 0) {
            label_logit = load1(row + y);
            scan_row_nat<T>(st, row, p.loss.cols, gl, LPR);
        }
        st = group_merge_nat<LPR>(st);          // also: every lane has read the row before any lane writes over it
        __syncwarp();
        if (live) {
            T* out = static_cast<T*>(p.grad) + r * p.grad_stride;
            if (y >= 0) write_row<T>(row, out, p.loss.cols, st.m, g / st.s, g, y, gl, LPR);
            else zero_row<T>(out, p.loss.cols, gl, LPR);
            if (p.loss.out && gl == 0) p.loss.out[r] = y >= 0 ? row_loss(st, label_logit) : 0.0f;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256) row_grad_cta_kernel(GradParams p) {
    __shared__ NatState warp_state[8];
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t n_inst = counted(p.count_dev, p.n_inst);
    if (p.offsets && blockIdx.x == 0) check_offsets(p.loss.ctl, p.offsets, n_inst, p.loss.rows);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int64_t r = blockIdx.x; r < p.loss.rows; r += gridDim.x) {
        float g = 0.0f;
        if (!row_factor(p, n_inst, r, g)) continue;     // uniform over the CTA
        const int y = checked_label(p.loss, r);
        const T* row = static_cast<const T*>(p.loss.logits) + r * p.loss.row_stride;
        T* out = static_cast<T*>(p.grad) + r * p.grad_stride;
        if (y < 0) {
            zero_row<T>(out, p.loss.cols, threadIdx.x, 256);
            if (p.loss.out && threadIdx.x == 0) p.loss.out[r] = 0.0f;
            continue;
        }
        const float label_logit = load1(row + y);
        NatState st = {-INFINITY, 0.0f};
        scan_row_nat<T>(st, row, p.loss.cols, threadIdx.x, 256);
        st = group_merge_nat<32>(st);
        __syncthreads();                                 // the previous row's states have been read
        if (lane == 0) warp_state[warp] = st;
        __syncthreads();
        st = group_merge_nat<32>(lane < 8 ? warp_state[lane] : NatState{-INFINITY, 0.0f});
        write_row<T>(row, out, p.loss.cols, st.m, g / st.s, g, y, threadIdx.x, 256);
        if (p.loss.out && threadIdx.x == 0) p.loss.out[r] = row_loss(st, label_logit);
    }
}

template <typename T>
aa_status launch_rows(aa_ctx_impl* c, GradParams& p) {
    const int64_t row_bytes = p.loss.cols * (int64_t)sizeof(T);
    void* args[] = {&p};
    const void* kernel;
    int64_t want;
    if (row_bytes > 8 * 1024) {
        kernel = (const void*)row_grad_cta_kernel<T>;
        want = p.loss.rows;
    } else {
        const int64_t work = (row_bytes + 15) / 16;
        int lpr = 2;
        while (lpr < 32 && lpr * 4 <= work) lpr <<= 1;
        switch (lpr) {
            case 2: kernel = (const void*)row_grad_group_kernel<T, 2>; break;
            case 4: kernel = (const void*)row_grad_group_kernel<T, 4>; break;
            case 8: kernel = (const void*)row_grad_group_kernel<T, 8>; break;
            case 16: kernel = (const void*)row_grad_group_kernel<T, 16>; break;
            default: kernel = (const void*)row_grad_group_kernel<T, 32>; break;
        }
        want = (p.loss.rows + 256 / lpr - 1) / (256 / lpr);
    }
    const int cap = resident_ctas(c, kernel, 256, 0);
    if (cap <= 0) return AA_ERR_CUDA;
    const unsigned grid = (unsigned)(want < cap ? want : cap);
    if (launch_overlapped(c, kernel, dim3(grid), dim3(256), args, 0, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

}  // namespace

aa_status launch_instance_loss_grad(aa_ctx_impl* c, const aa_logits& lg, const int32_t* labels, const int32_t* offsets, int64_t n_seg,
                                    const int32_t* count_dev, const float* weight, float scale, int mean, float* out_loss, const aa_rows& grad) {
    GradParams p = {};
    p.loss.logits = lg.data;
    p.loss.rows = p.loss.n_stored = lg.rows;
    p.loss.cols = lg.cols;
    p.loss.row_stride = lg.row_stride;
    p.loss.labels = labels;
    p.loss.ctl = c->ctl;
    p.loss.out = out_loss && offsets ? c->row_scratch : out_loss;
    p.offsets = offsets;
    p.n_inst = offsets ? n_seg : lg.rows;
    p.count_dev = count_dev;
    p.weight = weight;
    p.scale = scale;
    p.mean = mean;
    p.grad = grad.data;
    p.grad_stride = grad.row_stride;
    if (lg.rows > 0) {
        const aa_status st = lg.dtype == AA_BF16 ? launch_rows<uint16_t>(c, p) : launch_rows<float>(c, p);
        if (st != AA_OK) return st;
    }
    if (offsets && out_loss && n_seg > 0) return launch_segment_sum(c, c->row_scratch, offsets, n_seg, count_dev, lg.rows, out_loss);
    return AA_OK;
}

}  // namespace aa
