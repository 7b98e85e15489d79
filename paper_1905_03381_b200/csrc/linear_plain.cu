// Products of linear layers in fp32 arithmetic on the ordinary lanes: any type, stride and alignment.
#include "linear.cuh"

namespace aa {

namespace {

constexpr int kT = 64, kK = 16;

template <typename T>
__global__ void __launch_bounds__(256) product_plain_kernel(ProductParams p) {
    __shared__ float As[kK][kT + 4], Bs[kK][kT + 4];
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0);
    const int64_t m_end = p.live_k ? p.m : min(p.m, live), k_end = p.live_k ? min(p.k, live) : p.k;
    const int64_t m0 = (int64_t)blockIdx.x * kT, n0 = (int64_t)blockIdx.y * kT;
    if (m0 >= m_end) return;
    const T *a = static_cast<const T*>(p.a.data), *b = static_cast<const T*>(p.b.data);
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4] = {};
    for (int64_t k0 = 0; k0 < k_end; k0 += kK) {
        for (int i = threadIdx.x; i < kT * kK; i += 256) {
            {
                const int r = p.a_across ? i % kT : i / kK, k = p.a_across ? i / kT : i % kK;
                const int64_t m = m0 + r, kk = k0 + k;
                As[k][r] = m < m_end && kk < k_end ? load1(a + (p.a_across ? kk * p.a.stride + m : m * p.a.stride + kk)) : 0.0f;
            }
            {
                const int r = p.b_across ? i % kT : i / kK, k = p.b_across ? i / kT : i % kK;
                const int64_t n = n0 + r, kk = k0 + k;
                Bs[k][r] = n < p.n && kk < k_end ? load1(b + (p.b_across ? kk * p.b.stride + n : n * p.b.stride + kk)) : 0.0f;
            }
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kK; ++k) {
            const float4 u = *reinterpret_cast<const float4*>(&As[k][ty * 4]), v = *reinterpret_cast<const float4*>(&Bs[k][tx * 4]);
            const float x[4] = {u.x, u.y, u.z, u.w}, y[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(x[i], y[j], acc[i][j]);
        }
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i) {
        const int64_t m = m0 + ty * 4 + i;
        if (m >= m_end) break;
        for (int j = 0; j < 4; ++j) {
            const int64_t n = n0 + tx * 4 + j;
            if (n >= p.n) break;
            float z = acc[i][j] + (p.bias ? p.bias[n] : 0.0f);
            if (p.pre.data) store1(static_cast<T*>(const_cast<void*>(p.pre.data)) + m * p.pre.stride + n, z);
            z = activate(z, p.act);
            if (p.residual.data) z += load1(static_cast<const T*>(p.residual.data) + m * p.residual.stride + n);
            store1(static_cast<T*>(const_cast<void*>(p.out.data)) + m * p.out.stride + n, z);
        }
    }
}

// Rows are shared out in kSlopeParts runs whose column sums stay apart until the join.
template <typename T>
__global__ void __launch_bounds__(256) slope_kernel(SlopeParams p) {
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0);
    const int64_t col = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (col >= p.cols) return;
    const int64_t run = (p.rows + kSlopeParts - 1) / kSlopeParts, r0 = run * blockIdx.y, r1 = min(live, r0 + run);
    const T *d = static_cast<const T*>(p.dout.data), *z = static_cast<const T*>(p.pre.data);
    T* g = static_cast<T*>(const_cast<void*>(p.g.data));
    float sum = 0.0f;
    for (int64_t r = r0; r < r1; ++r) {
        float x = load1(d + r * p.dout.stride + col);
        if (p.act != AA_ACT_NONE) x *= activation_slope(load1(z + r * p.pre.stride + col), p.act);
        if (g) store1(g + r * p.g.stride + col, x);
        sum += x;
    }
    if (p.dbias) p.parts[(int64_t)blockIdx.y * p.cols + col] = sum;
}

__global__ void __launch_bounds__(256) slope_join_kernel(const float* parts, float* dbias, int64_t cols) {
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t col = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (col >= cols) return;
    float sum = 0.0f;
    for (int i = 0; i < kSlopeParts; ++i) sum += parts[(int64_t)i * cols + col];
    dbias[col] = sum;
}

}  // namespace

aa_status launch_product(aa_ctx_impl* c, const ProductParams& in, int dtype) {
    ProductParams p = in;
    if (dtype == AA_BF16 && product_tc_fits(p)) return launch_product_tc(c, p);
    const int64_t mt = (p.m + kT - 1) / kT, nt = (p.n + kT - 1) / kT;
    if (mt > 0x7FFFFFFFll || nt > 65535) return AA_ERR_UNSUPPORTED;
    const void* kernel = dtype == AA_BF16 ? (const void*)product_plain_kernel<uint16_t> : (const void*)product_plain_kernel<float>;
    void* args[] = {&p};
    if (launch_overlapped(c, kernel, dim3((unsigned)mt, (unsigned)nt), dim3(256), args, 0, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

aa_status launch_slope(aa_ctx_impl* c, const SlopeParams& in, int dtype) {
    SlopeParams p = in;
    const unsigned ct = (unsigned)((p.cols + 255) / 256);
    const void* kernel = dtype == AA_BF16 ? (const void*)slope_kernel<uint16_t> : (const void*)slope_kernel<float>;
    void* args[] = {&p};
    if (launch_overlapped(c, kernel, dim3(ct, kSlopeParts), dim3(256), args, 0, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    if (!p.dbias) return AA_OK;
    void* join[] = {&p.parts, &p.dbias, &p.cols};
    if (launch_overlapped(c, (const void*)slope_join_kernel, dim3(ct), dim3(256), join, 0, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

}  // namespace aa
