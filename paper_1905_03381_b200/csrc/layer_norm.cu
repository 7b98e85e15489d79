// Layer normalisation of rows and its gradients.
//
//   c = x - mean(x),  r = 1 / sqrt(mean(c^2) + eps),  h = c r,  out = h gamma + beta
//   g = dout gamma,   dx = r (g - mean(g) - h mean(g h)) + residual,   dgamma = sum_rows dout h,  dbeta = sum_rows dout
//
// Bound by memory: 2 values a column pass forward, 3 or 4 backward, against about 10 and 20 instructions.  A row stays in the registers of a group of
// threads (8 or 16 columns each) between its sums and its result, so that memory is touched once; mean and variance are two rounds over registers, so that
// nothing cancels.  Backward the rounds carry (sum x, sum g) and (sum c^2, sum g c): mean(g h) = r mean(g c), and no statistics are kept from the
// forward pass (two floats a row would save one round of shuffles and no memory).  A group walks over rows of its own and adds up dout h and dout of its
// columns; the sums of a CTA's groups are joined in shared memory, those of the CTAs by a second kernel, both in a fixed order.
// Rows too long for registers are swept three times, and their columns are summed by a kernel of their own.
#include <type_traits>

#include "layer_norm.cuh"

namespace aa {

namespace {

template <int G>
constexpr int kThreadsOf = G > 256 ? G : 256;     // CTAs of several groups, or of one

// Sums of two values over a group of G threads.  Groups of more than a warp meet at a barrier of their own; `buf` (theirs) is not used again before the
// next one.
template <int G>
__device__ __forceinline__ float2 group_sum(float2 s, float2* buf) {
#pragma unroll
    for (int o = (G < 32 ? G : 32) / 2; o > 0; o >>= 1) {
        s.x += __shfl_xor_sync(0xFFFFFFFFu, s.x, o);
        s.y += __shfl_xor_sync(0xFFFFFFFFu, s.y, o);
    }
    if constexpr (G > 32) {
        const int group = threadIdx.x / G;
        float2* mine = buf + group * (G / 32);
        if ((threadIdx.x & 31) == 0) mine[threadIdx.x % G >> 5] = s;
        if constexpr (kThreadsOf<G> == G) __syncthreads();
        else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(G) : "memory");
        s = mine[0];
#pragma unroll
        for (int w = 1; w < G / 32; ++w) {
            s.x += mine[w].x;
            s.y += mine[w].y;
        }
    }
    return s;
}

// What a thread fetches of a row, as it lies in memory.
template <typename T, int V, int E>
struct Raw {
    using Word = typename std::conditional<V == 1, T, uint4>::type;
    static constexpr int N = E / V;
    Word w[N];
    __device__ __forceinline__ void fetch(const T* row, int first, int step, int cols) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (first + i * step < cols) w[i] = *reinterpret_cast<const Word*>(row + first + i * step);
    }
    __device__ __forceinline__ void values(int i, float* out) const {
        if constexpr (V == 1) {
            if constexpr (sizeof(T) == 4) out[0] = w[i];
            else out[0] = __uint_as_float((uint32_t)w[i] << 16);
        } else {
            float t[V];
            Vec<T>::unpack(w[i], t);
#pragma unroll
            for (int e = 0; e < V; ++e) out[e] = t[e];
        }
    }
};

// gamma and beta of the thread's columns stay in registers over its rows.
template <typename T, int V, int E, int G>
__global__ void __launch_bounds__(kThreadsOf<G>, 512 / kThreadsOf<G>) norm_kernel(NormParams p) {
    constexpr int TH = kThreadsOf<G>, N = E / V;
    __shared__ float2 buf[2][32];
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, blockIdx.x == 0 && threadIdx.x == 0);
    const int l = threadIdx.x % G, groups = TH / G;
    const int cols = (int)p.cols, first = l * V, step = G * V;
    const float inv = 1.0f / (float)cols;
    float gm[E], bt[E];
#pragma unroll
    for (int j = 0; j < E; ++j) {
        const int c = first + j / V * step + j % V;
        gm[j] = c < cols && p.gamma ? p.gamma[c] : 1.0f;
        bt[j] = c < cols && p.beta ? p.beta[c] : 0.0f;
    }
    Raw<T, V, E> x;
    // the lanes of a warp keep step: rows past the end are looked at as the last one and not written
    const auto fetch = [&](int64_t r0) { x.fetch(static_cast<const T*>(p.x.data) + min(r0 + threadIdx.x / G, live - 1) * p.x.stride, first, step, cols); };
    const int64_t jump = (int64_t)gridDim.x * groups;
    int64_t r0 = (int64_t)blockIdx.x * groups;
    if (r0 < live) fetch(r0);
    for (; r0 < live; r0 += jump) {
        const int64_t row = r0 + threadIdx.x / G;
        float v[E];
        float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x.values(i, v + i * V);
#pragma unroll
            for (int e = 0; e < V; ++e) v[i * V + e] = first + i * step < cols ? v[i * V + e] : 0.0f;
        }
        if (r0 + jump < live) fetch(r0 + jump);
#pragma unroll
        for (int j = 0; j < E; j += 4) s.x += (v[j] + v[j + 1]) + (v[j + 2] + v[j + 3]);
        const float mean = __fdiv_rn(group_sum<G>(s, buf[0]).x, (float)cols);     // exact for constant rows
        s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            v[j] = first + j / V * step < cols ? v[j] - mean : 0.0f;
            s.x = fmaf(v[j], v[j], s.x);
        }
        const float r = 1.0f / sqrtf(group_sum<G>(s, buf[1]).x * inv + p.eps);
        T* out = static_cast<T*>(const_cast<void*>(p.out.data)) + row * p.out.stride;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = first + i * step;
            if (c >= cols || row >= live) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) v[i * V + e] = fmaf(v[i * V + e] * r, gm[i * V + e], bt[i * V + e]);
            store_elems<T, V>(out + c, v + i * V);
        }
    }
}

// AHEAD: the next row's loads are under way while a row is worked on; otherwise more CTAs share the SM (loads of single elements, which a thread has many of,
// wait for one another).  gamma and the thread's column sums lie in shared memory, [quad][thread], a private float4 each.
template <typename T, int V, int E, int G, bool AHEAD>
__global__ void __launch_bounds__(kThreadsOf<G>, (AHEAD || E == 16 ? 512 : 1024) / kThreadsOf<G>) norm_grad_kernel(NormParams p) {
    constexpr int TH = kThreadsOf<G>, N = E / V, Q = E / 4;
    __shared__ float2 buf[2][32];
    extern __shared__ float4 quads[];        // gamma[Q][TH], dgamma[Q][TH], dbeta[Q][TH]
    float4 *gm4 = quads + threadIdx.x, *dg4 = gm4 + Q * TH, *db4 = dg4 + Q * TH;
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, blockIdx.x == 0 && threadIdx.x == 0);
    const int l = threadIdx.x % G, groups = TH / G;
    const int cols = (int)p.cols, first = l * V, step = G * V;
    const float inv = 1.0f / (float)cols;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        float g[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int j = q * 4 + e, c = first + j / V * step + j % V;
            g[e] = c < cols ? (p.gamma ? p.gamma[c] : 1.0f) : 0.0f;
        }
        gm4[q * TH] = make_float4(g[0], g[1], g[2], g[3]);
        dg4[q * TH] = db4[q * TH] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    Raw<T, V, E> x, d, res;
    // the lanes of a warp keep step: rows past the end are looked at as the last one and not written
    const auto fetch = [&](int64_t r0) {
        const int64_t row = min(r0 + threadIdx.x / G, live - 1);
        x.fetch(static_cast<const T*>(p.x.data) + row * p.x.stride, first, step, cols);
        d.fetch(static_cast<const T*>(p.dout.data) + row * p.dout.stride, first, step, cols);
        if (p.residual.data) res.fetch(static_cast<const T*>(p.residual.data) + row * p.residual.stride, first, step, cols);
    };
    const int64_t jump = (int64_t)gridDim.x * groups;
    int64_t r0 = (int64_t)blockIdx.x * groups;
    if (AHEAD && r0 < live) fetch(r0);
    for (; r0 < live; r0 += jump) {
        const int64_t row = r0 + threadIdx.x / G;
        const bool on = row < live;
        if (!AHEAD) fetch(r0);
        float v[E], u[E];
        float2 s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const bool has = first + i * step < cols;
            x.values(i, v + i * V);
            d.values(i, u + i * V);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                v[i * V + e] = has ? v[i * V + e] : 0.0f;
                u[i * V + e] = has ? u[i * V + e] : 0.0f;
            }
        }
        const Raw<T, V, E> add = res;
        if (AHEAD && r0 + jump < live) fetch(r0 + jump);
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const float4 g = gm4[q * TH];
            s.x += (v[4 * q] + v[4 * q + 1]) + (v[4 * q + 2] + v[4 * q + 3]);
            s.y = fmaf(u[4 * q], g.x, s.y);
            s.y = fmaf(u[4 * q + 1], g.y, s.y);
            s.y = fmaf(u[4 * q + 2], g.z, s.y);
            s.y = fmaf(u[4 * q + 3], g.w, s.y);
        }
        s = group_sum<G>(s, buf[0]);
        const float mean = __fdiv_rn(s.x, (float)cols), mg = s.y * inv;
        s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const float4 g4 = gm4[q * TH];
            const float g[4] = {g4.x, g4.y, g4.z, g4.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = 4 * q + e;
                v[j] = first + j / V * step < cols ? v[j] - mean : 0.0f;
                s.x = fmaf(v[j], v[j], s.x);
                s.y = fmaf(v[j], u[j] * g[e], s.y);
            }
        }
        s = group_sum<G>(s, buf[1]);
        const float r = 1.0f / sqrtf(s.x * inv + p.eps), k = s.y * inv * r;
        T* out = static_cast<T*>(const_cast<void*>(p.out.data)) + row * p.out.stride;
        float y[E];
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const float4 g4 = gm4[q * TH];
            const float g[4] = {g4.x, g4.y, g4.z, g4.w};
            float h[4], w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int j = 4 * q + e;
                h[e] = v[j] * r;
                w[e] = on ? u[j] : 0.0f;
                y[j] = r * (fmaf(u[j], g[e], -mg) - h[e] * k);
            }
            float4 a = dg4[q * TH], b = db4[q * TH];
            a.x = fmaf(w[0], h[0], a.x), a.y = fmaf(w[1], h[1], a.y), a.z = fmaf(w[2], h[2], a.z), a.w = fmaf(w[3], h[3], a.w);
            b.x += w[0], b.y += w[1], b.z += w[2], b.w += w[3];
            dg4[q * TH] = a;
            db4[q * TH] = b;
        }
        if (!on) continue;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = first + i * step;
            if (c >= cols) continue;
            if (p.residual.data) {
                float z[V];
                add.values(i, z);
#pragma unroll
                for (int e = 0; e < V; ++e) y[i * V + e] += z[e];
            }
            store_elems<T, V>(out + c, y + i * V);
        }
    }
    if (!p.parts) return;
    __syncthreads();
    float* to = p.parts + (int64_t)blockIdx.x * 2 * cols;
    const float *dg = reinterpret_cast<const float*>(quads + Q * TH), *db = dg + 4 * Q * TH;
    for (int c = threadIdx.x; c < cols; c += TH) {
        const int j = c / step * V + c % V, owner = c % step / V;      // element j of the group's thread `owner`
        float a = 0.0f, b = 0.0f;
        for (int w = 0; w < groups; ++w) {                             // one group after the other
            const int at = ((j >> 2) * TH + w * G + owner) * 4 + (j & 3);
            a += dg[at];
            b += db[at];
        }
        to[c] = a;
        to[cols + c] = b;
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
        const float mean = __fdiv_rn(group_sum<kSweep>(s, buf[0]).x, (float)p.cols);
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
        const float mean = __fdiv_rn(group_sum<kSweep>(s, buf[0]).x, (float)p.cols);
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
#pragma unroll 8
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

template <typename T, int V, int E, int G>
aa_status launch_rows(aa_ctx_impl* c, NormParams p, bool grad, int* n_parts) {
    constexpr int TH = kThreadsOf<G>, groups = TH / G;
    const void* kernel = grad ? (const void*)norm_grad_kernel<T, V, E, G, (V > 1)> : (const void*)norm_kernel<T, V, E, G>;
    const size_t smem = grad ? 3 * sizeof(float) * E * TH : 0;
    if (smem && allow_smem(c, kernel, smem) != AA_OK) return AA_ERR_CUDA;
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

// The smallest group whose threads have 8 columns each at most (narrow rows of packed bf16: 16, which are two words).
template <typename T, int V>
aa_status launch_width(aa_ctx_impl* c, const NormParams& p, bool grad, int* n) {
    if constexpr (V == 8) {
        if (p.cols <= 128) return launch_rows<T, V, 16, 8>(c, p, grad, n);
        if (p.cols <= 256) return launch_rows<T, V, 16, 16>(c, p, grad, n);
        if (p.cols <= 512) return launch_rows<T, V, 16, 32>(c, p, grad, n);
    } else {
        if (p.cols <= 128) return launch_rows<T, V, 8, 16>(c, p, grad, n);
        if (p.cols <= 256) return launch_rows<T, V, 8, 32>(c, p, grad, n);
        if (p.cols <= 512) return launch_rows<T, V, 8, 64>(c, p, grad, n);
    }
    if (p.cols <= 1024) return launch_rows<T, V, 8, 128>(c, p, grad, n);
    if (p.cols <= 2048) return launch_rows<T, V, 8, 256>(c, p, grad, n);
    if (p.cols <= 4096) return launch_rows<T, V, 8, 512>(c, p, grad, n);
    if constexpr (V != 8)
        if (p.cols <= 6144) return launch_rows<T, V, 12, 512>(c, p, grad, n);
    return launch_rows<T, V, 16, 512>(c, p, grad, n);
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
