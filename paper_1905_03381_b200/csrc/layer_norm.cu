// Layer normalisation of rows and its gradients.
//
//   c = x - mean(x),  r = 1 / sqrt(mean(c^2) + eps),  h = c r,  out = h gamma + beta
//   g = dout gamma,   dx = r (g - mean(g) - h mean(g h)) + residual,   dgamma = sum_rows dout h,  dbeta = sum_rows dout
//
// Bound by memory: 2 values a column pass forward, 3 or 4 backward, against about 10 and 20 instructions.  A row stays in the registers of a group of
// threads (16 columns each) between its sums and its result, so that memory is touched once; mean and variance are two rounds over registers, so that
// nothing cancels.  Backward the rounds carry (sum x, sum g) and (sum c^2, sum g c): mean(g h) = r mean(g c), and no statistics are kept from the
// forward pass (two floats a row would save one round of shuffles and no memory).  A group walks over rows of its own and adds up dout h and dout of its
// columns in registers; the sums of a CTA's groups are joined in shared memory, those of the CTAs by a second kernel, both in a fixed order.
// Rows too long for registers are swept three times, and their columns are summed by a kernel of their own.
#include "boss_args.cuh"
#include "linear.cuh"
#include "layer_norm.cuh"

namespace aa {

namespace {

constexpr int kEach = 16;                // columns a thread

// Sums of two values over a group of G lanes of a warp, or over the CTA (G > 32; `buf` is not used again before another barrier).
template <int G>
__device__ __forceinline__ float2 group_sum(float2 s, float2* buf) {
#pragma unroll
    for (int o = (G < 32 ? G : 32) / 2; o > 0; o >>= 1) {
        s.x += __shfl_xor_sync(0xFFFFFFFFu, s.x, o);
        s.y += __shfl_xor_sync(0xFFFFFFFFu, s.y, o);
    }
    if constexpr (G > 32) {
        if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = s;
        __syncthreads();
        s = buf[0];
#pragma unroll
        for (int w = 1; w < G / 32; ++w) {
            s.x += buf[w].x;
            s.y += buf[w].y;
        }
    }
    return s;
}

template <int G>
constexpr int kThreadsOf = G > 32 ? G : 256;      // a group is part of a warp, or the CTA

template <typename T, int V, int G>
__global__ void __launch_bounds__(kThreadsOf<G>) norm_kernel(NormParams p) {
    constexpr int TH = kThreadsOf<G>, N = kEach / V;
    __shared__ float2 buf[2][32];
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, blockIdx.x == 0 && threadIdx.x == 0);
    const int l = threadIdx.x % G, groups = TH / G;
    const int cols = (int)p.cols;
    const float inv = 1.0f / (float)cols;
    // the lanes of a warp keep step: rows past the end are looked at as the last one and not written
    for (int64_t r0 = (int64_t)blockIdx.x * groups; r0 < live; r0 += (int64_t)gridDim.x * groups) {
        const int64_t row = r0 + threadIdx.x / G;
        const bool on = row < live;
        const T* x = static_cast<const T*>(p.x.data) + (on ? row : live - 1) * p.x.stride;
        float v[kEach];
        float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = (i * G + l) * V;
#pragma unroll
            for (int e = 0; e < V; ++e) v[i * V + e] = 0.0f;
            if (c < cols) load_elems<T, V>(x + c, v + i * V);
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) s.x += v[i];
        const float mean = group_sum<G>(s, buf[0]).x * inv;
        s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if ((i * G + l) * V < cols)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    v[i * V + e] -= mean;
                    s.x = fmaf(v[i * V + e], v[i * V + e], s.x);
                }
        const float r = 1.0f / sqrtf(group_sum<G>(s, buf[1]).x * inv + p.eps);
        T* out = static_cast<T*>(const_cast<void*>(p.out.data)) + row * p.out.stride;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = (i * G + l) * V;
            if (c >= cols || !on) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) v[i * V + e] = fmaf(v[i * V + e] * r, p.gamma ? p.gamma[c + e] : 1.0f, p.beta ? p.beta[c + e] : 0.0f);
            store_elems<T, V>(out + c, v + i * V);
        }
    }
}

template <typename T, int V, int G>
__global__ void __launch_bounds__(kThreadsOf<G>) norm_grad_kernel(NormParams p) {
    constexpr int TH = kThreadsOf<G>, N = kEach / V;
    __shared__ float2 buf[2][32];
    extern __shared__ float sums[];          // [2][cols], where a CTA has several groups
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, blockIdx.x == 0 && threadIdx.x == 0);
    const int l = threadIdx.x % G, groups = TH / G;
    const int cols = (int)p.cols;
    const float inv = 1.0f / (float)cols;
    float gm[kEach], dg[kEach], db[kEach];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int c = (i * G + l) * V + e;
            gm[i * V + e] = c < cols ? (p.gamma ? p.gamma[c] : 1.0f) : 0.0f;
            dg[i * V + e] = db[i * V + e] = 0.0f;
        }
    for (int64_t r0 = (int64_t)blockIdx.x * groups; r0 < live; r0 += (int64_t)gridDim.x * groups) {
        const int64_t row = r0 + threadIdx.x / G, at = row < live ? row : live - 1;
        const bool on = row < live;
        const T *x = static_cast<const T*>(p.x.data) + at * p.x.stride, *d = static_cast<const T*>(p.dout.data) + at * p.dout.stride;
        const T* res = p.residual.data ? static_cast<const T*>(p.residual.data) + at * p.residual.stride : nullptr;
        float v[kEach], u[kEach];
        float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = (i * G + l) * V;
#pragma unroll
            for (int e = 0; e < V; ++e) v[i * V + e] = u[i * V + e] = 0.0f;
            if (c < cols) {
                load_elems<T, V>(x + c, v + i * V);
                load_elems<T, V>(d + c, u + i * V);
            }
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            s.x += v[i];
            s.y = fmaf(u[i], gm[i], s.y);
        }
        s = group_sum<G>(s, buf[0]);
        const float mean = s.x * inv, mg = s.y * inv;
        s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if ((i * G + l) * V < cols)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    float& c = v[i * V + e];
                    c -= mean;
                    s.x = fmaf(c, c, s.x);
                    s.y = fmaf(c, u[i * V + e] * gm[i * V + e], s.y);
                }
        s = group_sum<G>(s, buf[1]);
        const float r = 1.0f / sqrtf(s.x * inv + p.eps), k = s.y * inv * r;
        T* out = static_cast<T*>(const_cast<void*>(p.out.data)) + row * p.out.stride;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = (i * G + l) * V;
            if (c >= cols || !on) continue;
            float y[V], add[V];
            if (res) load_elems<T, V>(res + c, add);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int j = i * V + e;
                const float h = v[j] * r;
                dg[j] = fmaf(u[j], h, dg[j]);
                db[j] += u[j];
                y[e] = r * (fmaf(u[j], gm[j], -mg) - h * k);
                if (res) y[e] += add[e];
            }
            store_elems<T, V>(out + c, y);
        }
    }
    if (!p.parts) return;
    float* to = p.parts + (int64_t)blockIdx.x * 2 * cols;
    if constexpr (G > 32) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int c = (i * G + l) * V + e;
                if (c < cols) {
                    to[c] = dg[i * V + e];
                    to[cols + c] = db[i * V + e];
                }
            }
    } else {
        for (int w = 0; w < groups; ++w) {       // one group after the other
            if (threadIdx.x / G == w) {
#pragma unroll
                for (int i = 0; i < N; ++i)
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const int c = (i * G + l) * V + e;
                        if (c < cols) {
                            sums[c] = w ? sums[c] + dg[i * V + e] : dg[i * V + e];
                            sums[cols + c] = w ? sums[cols + c] + db[i * V + e] : db[i * V + e];
                        }
                    }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < 2 * cols; c += TH) to[c] = sums[c];
    }
}

// ---------------------------------------------------------------------- rows too long for registers

constexpr int kSweep = 512;

template <typename T>
__global__ void __launch_bounds__(kSweep) norm_sweep_kernel(NormParams p) {
    __shared__ float2 buf[2][32];
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, blockIdx.x == 0 && threadIdx.x == 0);
    const float inv = 1.0f / (float)p.cols;
    for (int64_t row = blockIdx.x; row < live; row += gridDim.x) {
        const T* x = static_cast<const T*>(p.x.data) + row * p.x.stride;
        float2 s = make_float2(0.0f, 0.0f);
        for (int64_t c = threadIdx.x; c < p.cols; c += kSweep) s.x += load1(x + c);
        const float mean = group_sum<kSweep>(s, buf[0]).x * inv;
        s = make_float2(0.0f, 0.0f);
        for (int64_t c = threadIdx.x; c < p.cols; c += kSweep) {
            const float d = load1(x + c) - mean;
            s.x = fmaf(d, d, s.x);
        }
        const float r = 1.0f / sqrtf(group_sum<kSweep>(s, buf[1]).x * inv + p.eps);
        T* out = static_cast<T*>(const_cast<void*>(p.out.data)) + row * p.out.stride;
        for (int64_t c = threadIdx.x; c < p.cols; c += kSweep)
            store1(out + c, fmaf((load1(x + c) - mean) * r, p.gamma ? p.gamma[c] : 1.0f, p.beta ? p.beta[c] : 0.0f));
    }
}

// Sums of dout h and dout over runs of rows, before the rows' own kernel may overwrite x or dout.  stats: mean and r of each row.
template <typename T>
__global__ void __launch_bounds__(256) norm_columns_kernel(NormParams p) {
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, false);
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= p.cols) return;
    const int64_t run = (p.live.rows + kSweepParts - 1) / kSweepParts, r0 = run * blockIdx.y, r1 = min(live, r0 + run);
    float a = 0.0f, b = 0.0f;
    for (int64_t row = r0; row < r1; ++row) {
        const float2 st = p.stats[row];
        const float d = load1(static_cast<const T*>(p.dout.data) + row * p.dout.stride + c);
        a = fmaf(d, (load1(static_cast<const T*>(p.x.data) + row * p.x.stride + c) - st.x) * st.y, a);
        b += d;
    }
    float* to = p.parts + (int64_t)blockIdx.y * 2 * p.cols;
    to[c] = a;
    to[p.cols + c] = b;
}

template <typename T>
__global__ void __launch_bounds__(kSweep) norm_stats_kernel(NormParams p) {
    __shared__ float2 buf[2][32];
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, blockIdx.x == 0 && threadIdx.x == 0);
    const float inv = 1.0f / (float)p.cols;
    for (int64_t row = blockIdx.x; row < live; row += gridDim.x) {
        const T* x = static_cast<const T*>(p.x.data) + row * p.x.stride;
        float2 s = make_float2(0.0f, 0.0f);
        for (int64_t c = threadIdx.x; c < p.cols; c += kSweep) s.x += load1(x + c);
        const float mean = group_sum<kSweep>(s, buf[0]).x * inv;
        s = make_float2(0.0f, 0.0f);
        for (int64_t c = threadIdx.x; c < p.cols; c += kSweep) {
            const float d = load1(x + c) - mean;
            s.x = fmaf(d, d, s.x);
        }
        const float r = 1.0f / sqrtf(group_sum<kSweep>(s, buf[1]).x * inv + p.eps);
        if (threadIdx.x == 0) p.stats[row] = make_float2(mean, r);
    }
}

template <typename T>
__global__ void __launch_bounds__(kSweep) norm_grad_sweep_kernel(NormParams p) {
    __shared__ float2 buf[2][32];
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, false);
    const float inv = 1.0f / (float)p.cols;
    for (int64_t row = blockIdx.x; row < live; row += gridDim.x) {
        const T *x = static_cast<const T*>(p.x.data) + row * p.x.stride, *d = static_cast<const T*>(p.dout.data) + row * p.dout.stride;
        const float2 st = p.stats[row];
        float2 s = make_float2(0.0f, 0.0f);
        for (int64_t c = threadIdx.x; c < p.cols; c += kSweep) {
            const float g = load1(d + c) * (p.gamma ? p.gamma[c] : 1.0f);
            s.x += g;
            s.y = fmaf(g, load1(x + c) - st.x, s.y);
        }
        s = group_sum<kSweep>(s, buf[0]);
        const float mg = s.x * inv, k = s.y * inv * st.y;
        T* out = static_cast<T*>(const_cast<void*>(p.out.data)) + row * p.out.stride;
        for (int64_t c = threadIdx.x; c < p.cols; c += kSweep) {
            float y = st.y * (load1(d + c) * (p.gamma ? p.gamma[c] : 1.0f) - mg - (load1(x + c) - st.x) * st.y * k);
            if (p.residual.data) y += load1(static_cast<const T*>(p.residual.data) + row * p.residual.stride + c);
            store1(out + c, y);
        }
        __syncthreads();                     // buf[0] is read by all before the next row writes it
    }
}

// Columns of [parts][2 cols] -> dgamma, dbeta.  32 columns a CTA; each of 8 warps adds up every eighth part.
__global__ void __launch_bounds__(256) norm_join_kernel(const float* parts, int n_parts, int64_t cols, float* dgamma, float* dbeta) {
    __shared__ float part[8][33];
    grid_dependency_wait();
    grid_dependency_release();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (c < 2 * cols)
        for (int i = w; i < n_parts; i += 8) s += parts[(int64_t)i * 2 * cols + c];
    part[w][lane] = s;
    __syncthreads();
    if (w == 0 && c < 2 * cols) {
#pragma unroll
        for (int i = 1; i < 8; ++i) s += part[i][lane];
        if (c < cols) {
            if (dgamma) dgamma[c] = s;
        } else if (dbeta) {
            dbeta[c - cols] = s;
        }
    }
}

template <typename T, int V, int G>
aa_status launch_rows(aa_ctx_impl* c, NormParams p, bool grad, int* n_parts) {
    constexpr int TH = kThreadsOf<G>, groups = TH / G;
    const void* kernel = grad ? (const void*)norm_grad_kernel<T, V, G> : (const void*)norm_kernel<T, V, G>;
    const size_t smem = grad && p.parts && G <= 32 ? 2 * sizeof(float) * (size_t)p.cols : 0;
    int ctas = resident_ctas(c, kernel, TH, smem);
    if (ctas < 1) return AA_ERR_CUDA;
    const int64_t wanted = (p.live.rows + groups - 1) / groups;
    if (grad && ctas > kNormParts) ctas = kNormParts;
    if (ctas > wanted) ctas = (int)wanted;
    void* args[] = {&p};
    if (launch_overlapped(c, kernel, dim3(ctas), dim3(TH), args, smem, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    *n_parts = ctas;
    return AA_OK;
}

template <typename T, int V>
aa_status launch_width(aa_ctx_impl* c, const NormParams& p, bool grad, int* n) {
    const int64_t g = (p.cols + kEach - 1) / kEach;
    if (g <= 8) return launch_rows<T, V, 8>(c, p, grad, n);
    if (g <= 16) return launch_rows<T, V, 16>(c, p, grad, n);
    if (g <= 32) return launch_rows<T, V, 32>(c, p, grad, n);
    if (g <= 128) return launch_rows<T, V, 128>(c, p, grad, n);
    if (g <= 256) return launch_rows<T, V, 256>(c, p, grad, n);
    return launch_rows<T, V, 512>(c, p, grad, n);
}

template <typename T>
aa_status launch_sweeps(aa_ctx_impl* c, NormParams p, bool grad, int* n_parts) {
    const int grid = (int)(p.live.rows < 2 * c->sm_count ? p.live.rows : 2 * c->sm_count);
    void* args[] = {&p};
    const void* first = grad ? (const void*)norm_stats_kernel<T> : (const void*)norm_sweep_kernel<T>;
    if (launch_overlapped(c, first, dim3(grid), dim3(kSweep), args, 0, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    if (!grad) return AA_OK;
    if (p.parts) {
        if (launch_overlapped(c, (const void*)norm_columns_kernel<T>, dim3((unsigned)((p.cols + 255) / 256), kSweepParts), dim3(256), args, 0, false) != cudaSuccess)
            return AA_ERR_CUDA;
        ++c->launches;
    }
    if (launch_overlapped(c, (const void*)norm_grad_sweep_kernel<T>, dim3(grid), dim3(kSweep), args, 0, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    *n_parts = kSweepParts;
    return AA_OK;
}

}  // namespace

size_t norm_scratch_floats(int64_t rows, int64_t cols) {
    const int64_t parts = cols > kNormInRegisters ? kSweepParts : kNormParts;
    return (size_t)(parts < rows || cols > kNormInRegisters ? parts : rows) * 2 * (size_t)cols;
}

aa_status launch_layer_norm(aa_ctx_impl* c, const NormParams& p, int dtype, bool grad, float* dgamma, float* dbeta) {
    const int es = dtype == AA_BF16 ? 2 : 4, wide = 16 / es;
    const auto aligned = [&](const MatArg& a) { return !a.data || ((uintptr_t)a.data % 16 == 0 && (a.stride * es) % 16 == 0); };
    const bool vec = p.cols % wide == 0 && aligned(p.x) && aligned(p.out) && aligned(p.dout) && aligned(p.residual);
    int n_parts = 0;
    aa_status st;
    if (p.cols > kNormInRegisters) st = dtype == AA_BF16 ? launch_sweeps<uint16_t>(c, p, grad, &n_parts) : launch_sweeps<float>(c, p, grad, &n_parts);
    else if (dtype == AA_BF16) st = vec ? launch_width<uint16_t, 8>(c, p, grad, &n_parts) : launch_width<uint16_t, 1>(c, p, grad, &n_parts);
    else st = vec ? launch_width<float, 4>(c, p, grad, &n_parts) : launch_width<float, 1>(c, p, grad, &n_parts);
    if (st != AA_OK || !grad || !p.parts) return st;
    float* parts = p.parts;
    int64_t cols = p.cols;
    void* args[] = {&parts, &n_parts, &cols, &dgamma, &dbeta};
    if (launch_overlapped(c, (const void*)norm_join_kernel, dim3((unsigned)((2 * cols + 31) / 32)), dim3(256), args, 0, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

}  // namespace aa
