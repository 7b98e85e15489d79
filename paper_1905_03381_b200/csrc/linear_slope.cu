// Gradients through the activations of linear layers, column sums of gradients, and copies of operands for the products: one pass over memory.
#include <type_traits>

#include "linear.cuh"

namespace aa {

namespace {

// Bound by memory: two values read and one written an element (one read where only the sums are wanted); with GELU, whose slope takes 28 instructions an element,
// about as much by instructions (25,000 x 2,048 bf16: 57 us, 5.4 TB/s, 71 % of the issue slots).  A CTA takes 32 x V columns of a run of rows, a
// warp every eighth row, a lane V neighbouring columns (VEC: as one word); rows are shared out in kSlopeParts runs whose column sums stay apart until the join.
// TERMS 0: g in the matrices' type.  1 or 3: bf16 terms of g in planes, rows up to a multiple of 64 behind the counted ones zero (the products that read them take 64 at a time).
template <typename T, bool VEC, int ACT, int TERMS>
__device__ __forceinline__ void slope(const SlopeParams& p, float (*sums)[32 * (16 / (int)sizeof(T))]) {
    constexpr int V = 16 / (int)sizeof(T);
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
                    for (int e = 0; e < V; ++e) x[e] *= activation_slope<ACT, sizeof(T) == 4>(y[e]);
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

// The copies of a call are one launch (blockIdx.z): 4,099 x 515 x 1,001 fp32 takes 24 us as three and 18 as one.
struct Slopes {
    SlopeParams of[kSlopeJobs];
};
template <typename T, bool VEC, int ACT, int TERMS>
__global__ void __launch_bounds__(256) slope_kernel(const __grid_constant__ Slopes jobs) {
    __shared__ float sums[8][32 * (16 / (int)sizeof(T))];
    grid_dependency_wait();
    grid_dependency_release();
    if (TERMS == 0 || blockIdx.z == 0) slope<T, VEC, ACT, TERMS>(jobs.of[0], sums);
    else slope<T, VEC, AA_ACT_NONE, TERMS>(jobs.of[blockIdx.z], sums);
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
#pragma unroll
        for (int i = 0; i < kSlopeParts; i += 8)             // all loads at once
            if (i + warp < kSlopeParts) sum += parts[(int64_t)(i + warp) * cols + col];
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

aa_status launch_slopes(aa_ctx_impl* c, const SlopeParams* in, int n, int dtype) {
    const int es = dtype == AA_BF16 ? 2 : 4, wide = 16 / es;
    const auto aligned = [&](const MatArg& a) { return !a.data || ((uintptr_t)a.data % 16 == 0 && (a.stride * es) % 16 == 0); };
    const auto vectors = [&](const SlopeParams& p) { return p.cols % wide == 0 && aligned(p.dout) && aligned(p.pre) && (p.plane > 0 || aligned(p.g)); };
    // neighbours whose rows are read in the same way go together
    for (int i = 0, j; i < n; i = j) {
        Slopes jobs = {};
        const bool vec = vectors(in[i]), planes = in[i].plane > 0;
        int64_t cols = 0;
        for (j = i; j < n && vectors(in[j]) == vec; ++j) {
            jobs.of[j - i] = in[j];
            cols = cols < in[j].cols ? in[j].cols : cols;
        }
        const void* kernel = dtype == AA_BF16 ? (vec ? slope_of<uint16_t, true>(in[i].act, planes) : slope_of<uint16_t, false>(in[i].act, planes))
                                              : (vec ? slope_of<float, true>(in[i].act, planes) : slope_of<float, false>(in[i].act, planes));
        void* args[] = {&jobs};
        if (launch_overlapped(c, kernel, dim3((unsigned)((cols + 32 * wide - 1) / (32 * wide)), kSlopeParts, (unsigned)(j - i)), dim3(256), args, 0, false) != cudaSuccess) return AA_ERR_CUDA;
        ++c->launches;
    }
    if (!in[0].dbias) return AA_OK;
    SlopeParams p = in[0];
    void* join[] = {&p.parts, &p.dbias, &p.cols};
    if (launch_overlapped(c, (const void*)slope_join_kernel, dim3((unsigned)((p.cols + 31) / 32)), dim3(256), join, 0, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

}  // namespace aa
