// Products of linear layers in fp32 arithmetic on the ordinary lanes: any type, stride and alignment.
#include <type_traits>

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
            float y[1] = {z};
            activate_all(y, p.act);
            z = y[0];
            if (p.residual.data) z += load1(static_cast<const T*>(p.residual.data) + m * p.residual.stride + n);
            store1(static_cast<T*>(const_cast<void*>(p.out.data)) + m * p.out.stride + n, z);
        }
    }
}

// Bound by memory: two values read and one written an element (one read where only the sums are wanted).  A CTA takes 32 x V columns of a run of rows, a
// warp every eighth row, a lane V neighbouring columns (VEC: as one word); rows are shared out in kSlopeParts runs whose column sums stay apart until the join.
// TERMS 0: g in the matrices' type.  1 or 3: bf16 terms of g in planes, rows up to a multiple of 64 behind the counted ones zero (the products that read them take 64 at a time).
template <typename T, bool VEC, int ACT, int TERMS>
__global__ void __launch_bounds__(256) slope_kernel(SlopeParams p) {
    constexpr int V = 16 / (int)sizeof(T);
    __shared__ float sums[8][32 * V];
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t col = ((int64_t)blockIdx.x * 32 + lane) * V;
    const int n = (int)max((int64_t)0, min((int64_t)V, p.cols - col));          // columns of this lane
    const int64_t run = (p.rows + kSlopeParts - 1) / kSlopeParts, r0 = run * blockIdx.y, r1 = min(r0 + run, TERMS ? min(p.rows, (live + 63) / 64 * 64) : live);
    const T *d = static_cast<const T*>(p.dout.data), *z = static_cast<const T*>(p.pre.data);
    T* g = static_cast<T*>(const_cast<void*>(p.g.data));
    float sum[V] = {};
    // ROWS rows' loads, all before the first store: nothing tells the compiler that g is apart from dout and pre
    using Word = typename std::conditional<VEC, uint4, T>::type;
    constexpr int N = VEC ? 1 : V, ROWS = VEC ? 4 : 2;
    const auto fetch = [&](const T* at, Word (&w)[N]) {
        if constexpr (VEC) {
            w[0] = *reinterpret_cast<const uint4*>(at);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) w[e] = at[min(e, n - 1)];
        }
    };
    const auto values = [&](const Word (&w)[N], float (&x)[V]) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            if constexpr (VEC && sizeof(T) == 4) x[e] = __uint_as_float((&w[0].x)[e]);
            else if constexpr (VEC) x[e] = e % 2 ? bf16_hi((&w[0].x)[e / 2]) : bf16_lo((&w[0].x)[e / 2]);
            else if constexpr (sizeof(T) == 4) x[e] = e < n ? (float)w[e] : 0.0f;
            else x[e] = e < n ? __uint_as_float((uint32_t)w[e] << 16) : 0.0f;
        }
    };
    const auto put = [&](int64_t r, const float (&x)[V]) {
        if constexpr (TERMS > 0) {
            // padded rows: the columns behind the last are written too, and not read
            uint16_t* to = static_cast<uint16_t*>(const_cast<void*>(p.g.data)) + r * p.g.stride + col;
            float y[V];
#pragma unroll
            for (int e = 0; e < V; ++e) y[e] = x[e];
#pragma unroll
            for (int t = 0; t < TERMS; ++t) {
                uint32_t w[V / 2];
#pragma unroll
                for (int e = 0; e < V; e += 2) {
                    w[e / 2] = pack_bf16(y[e], y[e + 1]);
                    y[e] -= bf16_lo(w[e / 2]);
                    y[e + 1] -= bf16_hi(w[e / 2]);
                }
                if constexpr (V == 8) *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
                else *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
                to += p.plane;
            }
        } else if (ACT != AA_ACT_NONE && g) {
            if constexpr (VEC) {
                store_elems<T, V>(g + r * p.g.stride + col, x);
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (e < n) store1(g + r * p.g.stride + col + e, x[e]);
            }
        }
    };
    if (n > 0) {
        const int64_t last = min(r1, live) - 1;
        for (int64_t r = r0 + warp; r <= last; r += 8 * ROWS) {
            Word dw[ROWS][N], zw[ROWS][N];
#pragma unroll
            for (int i = 0; i < ROWS; ++i) {
                const int64_t at = min(r + 8 * i, last);
                fetch(d + at * p.dout.stride + col, dw[i]);
                if (ACT != AA_ACT_NONE) fetch(z + at * p.pre.stride + col, zw[i]);
            }
#pragma unroll
            for (int i = 0; i < ROWS; ++i) {
                if (r + 8 * i > last) break;
                float x[V];
                values(dw[i], x);
                if (ACT != AA_ACT_NONE) {
                    float y[V];
                    values(zw[i], y);
#pragma unroll
                    for (int e = 0; e < V; ++e) x[e] *= activation_slope<ACT>(y[e]);
                }
                put(r + 8 * i, x);
#pragma unroll
                for (int e = 0; e < V; ++e) sum[e] += x[e];
            }
        }
        if (TERMS > 0) {
            const float zero[V] = {};
            for (int64_t r = max(r0, live) + warp; r < r1; r += 8) put(r, zero);
        }
    }
    if (!p.dbias) return;
#pragma unroll
    for (int e = 0; e < V; ++e) sums[warp][lane * V + e] = sum[e];
    __syncthreads();
    for (int i = threadIdx.x; i < 32 * V; i += 256) {
        const int64_t c = (int64_t)blockIdx.x * 32 * V + i;
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < 8; ++w) s += sums[w][i];
        if (c < p.cols) p.parts[(int64_t)blockIdx.y * p.cols + c] = s;
    }
}

// 32 columns a CTA; each of 8 warps adds up every eighth part.
__global__ void __launch_bounds__(256) slope_join_kernel(const float* parts, float* dbias, int64_t cols) {
    __shared__ float sums[8][32];
    grid_dependency_wait();
    grid_dependency_release();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t col = (int64_t)blockIdx.x * 32 + lane;
    float sum = 0.0f;
    if (col < cols)
#pragma unroll 4
        for (int i = warp; i < kSlopeParts; i += 8) sum += parts[(int64_t)i * cols + col];
    sums[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && col < cols) {
#pragma unroll
        for (int w = 1; w < 8; ++w) sum += sums[w][lane];
        dbias[col] = sum;
    }
}

template <typename T, bool VEC, int TERMS>
const void* slope_of(int act) {
    if (act == AA_ACT_RELU) return (const void*)slope_kernel<T, VEC, AA_ACT_RELU, TERMS>;
    if (act == AA_ACT_GELU) return (const void*)slope_kernel<T, VEC, AA_ACT_GELU, TERMS>;
    if (act == AA_ACT_SILU) return (const void*)slope_kernel<T, VEC, AA_ACT_SILU, TERMS>;
    return (const void*)slope_kernel<T, VEC, AA_ACT_NONE, TERMS>;
}

template <typename T, bool VEC>
const void* slope_of(int act, bool planes) { return planes ? slope_of<T, VEC, sizeof(T) == 4 ? 3 : 1>(act) : slope_of<T, VEC, 0>(act); }

}  // namespace

aa_status launch_product(aa_ctx_impl* c, const ProductParams& in, int dtype) {
    ProductParams p = in;
    if (product_few_fits(p)) return launch_product_few(c, p, dtype);
    if (dtype == AA_BF16 && product_tc_fits(p)) return launch_product_tc(c, p);
    return launch_product_split(c, p, dtype);
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
    const int es = dtype == AA_BF16 ? 2 : 4, wide = 16 / es;
    const auto aligned = [&](const MatArg& a) { return !a.data || ((uintptr_t)a.data % 16 == 0 && (a.stride * es) % 16 == 0); };
    const bool vec = p.cols % wide == 0 && aligned(p.dout) && aligned(p.pre) && (p.plane > 0 || aligned(p.g));
    const bool planes = p.plane > 0;
    const void* kernel = dtype == AA_BF16 ? (vec ? slope_of<uint16_t, true>(p.act, planes) : slope_of<uint16_t, false>(p.act, planes))
                                          : (vec ? slope_of<float, true>(p.act, planes) : slope_of<float, false>(p.act, planes));
    void* args[] = {&p};
    if (launch_overlapped(c, kernel, dim3((unsigned)((p.cols + 32 * wide - 1) / (32 * wide)), kSlopeParts), dim3(256), args, 0, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    if (!p.dbias) return AA_OK;
    void* join[] = {&p.parts, &p.dbias, &p.cols};
    if (launch_overlapped(c, (const void*)slope_join_kernel, dim3((unsigned)((p.cols + 31) / 32)), dim3(256), join, 0, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

}  // namespace aa
