// Attention with a relative position bias, forward and backward, in fp32 arithmetic on the ordinary lanes: every dtype, stride and head
// width up to 256.  (The bf16 kernels on the tensor cores take the aligned bf16 problems.)
//
// A CTA of 256 threads holds a B x B score tile, each thread an M x M part of it (rows ty*M + a, columns tx + 16 b), and loops over the
// other axis with the running maximum and sum of a softmax.  Operand tiles sit in shared memory as fp32, zero past the sequence's end.
// Bound by the loads that feed the multiply-adds (eight 16-byte reads for 64 of them at best), by a width of 40 padded to 64, and by unequal CTAs (the
// busiest SM is active 1.4 to 1.5 times as long as the mean one): 24 sentences of up to 301 tokens, 5 heads of 40, forward and every gradient with
// dropout 0.39 ms for 1.9 GFLOP.  Operands split into two or three narrower terms would bring these products onto the tensor cores within the same
// bounds; that is not built.
#include "rel_attention.cuh"

namespace aa {

namespace {

constexpr int kThreads = 256;

template <int DT>
struct Geo {
    static constexpr int B = DT == 256 ? 32 : 64;   // tile side
    static constexpr int M = B / 16;
    static constexpr int LD = DT + 4;               // row pitch of an operand tile: float4 reads of 8 rows cover the 32 banks
    static constexpr int LP = B + 4;                // ... of a probability tile
    static constexpr int W = DT / 16;               // head elements per thread of an output row
    static size_t smem(int tiles, int reach_floats) { return sizeof(float) * (size_t)(tiles * B * LD + B * LP + reach_floats); }
};

template <typename T, int DT>
__device__ __forceinline__ void load_tile(const RelParams& p, const TokArg& a, int head, int64_t row0, int n, float* dst) {
    using G = Geo<DT>;
    const T* base = static_cast<const T*>(a.data) + row0 * a.tok + (int64_t)head * a.head;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll 4
    for (int r = warp; r < G::B; r += kThreads / 32)                  // a warp per row
#pragma unroll
        for (int e0 = 0; e0 < DT; e0 += 32) {
            const int e = e0 + lane;
            dst[r * G::LD + e] = r < n && e < p.dim ? load1(base + (int64_t)r * a.tok + e) : 0.0f;
        }
}

// acc[a][b] = x[ty*M + a] . y[tx + 16 b]
template <int DT>
__device__ __forceinline__ void dot_tile(const float* x, const float* y, int ty, int tx, float (&acc)[Geo<DT>::M][Geo<DT>::M]) {
    using G = Geo<DT>;
#pragma unroll
    for (int a = 0; a < G::M; ++a)
#pragma unroll
        for (int b = 0; b < G::M; ++b) acc[a][b] = 0.0f;
#pragma unroll 4
    for (int e = 0; e < DT; e += 4) {
        float4 u[G::M], w[G::M];
#pragma unroll
        for (int a = 0; a < G::M; ++a) u[a] = *reinterpret_cast<const float4*>(x + (ty * G::M + a) * G::LD + e);
#pragma unroll
        for (int b = 0; b < G::M; ++b) w[b] = *reinterpret_cast<const float4*>(y + (tx + 16 * b) * G::LD + e);
#pragma unroll
        for (int a = 0; a < G::M; ++a)
#pragma unroll
            for (int b = 0; b < G::M; ++b) {
                acc[a][b] = fmaf(u[a].x, w[b].x, acc[a][b]);
                acc[a][b] = fmaf(u[a].y, w[b].y, acc[a][b]);
                acc[a][b] = fmaf(u[a].z, w[b].z, acc[a][b]);
                acc[a][b] = fmaf(u[a].w, w[b].w, acc[a][b]);
            }
    }
}

// acc[a][w] += sum_j P[ty*M + a][j] X[j][tx + 16 w]
template <int DT>
__device__ __forceinline__ void rows_times(const float* P, const float* X, int ty, int tx, float (&acc)[Geo<DT>::M][Geo<DT>::W]) {
    using G = Geo<DT>;
#pragma unroll 2
    for (int j = 0; j < G::B; ++j) {
        float u[G::M];
#pragma unroll
        for (int a = 0; a < G::M; ++a) u[a] = P[(ty * G::M + a) * G::LP + j];
#pragma unroll
        for (int w = 0; w < G::W; ++w) {
            const float x = X[j * G::LD + tx + 16 * w];
#pragma unroll
            for (int a = 0; a < G::M; ++a) acc[a][w] = fmaf(u[a], x, acc[a][w]);
        }
    }
}
// acc[a][w] += sum_i P[i][ty*M + a] X[i][tx + 16 w]
template <int DT>
__device__ __forceinline__ void cols_times(const float* P, const float* X, int ty, int tx, float (&acc)[Geo<DT>::M][Geo<DT>::W]) {
    using G = Geo<DT>;
#pragma unroll 2
    for (int i = 0; i < G::B; ++i) {
        float u[G::M];
#pragma unroll
        for (int a = 0; a < G::M; ++a) u[a] = P[i * G::LP + ty * G::M + a];
#pragma unroll
        for (int w = 0; w < G::W; ++w) {
            const float x = X[i * G::LD + tx + 16 * w];
#pragma unroll
            for (int a = 0; a < G::M; ++a) acc[a][w] = fmaf(u[a], x, acc[a][w]);
        }
    }
}

// Products -> base-2 scores with bias and masks; masked ones are -inf whatever the products hold.
template <int DT>
__device__ __forceinline__ void finish_scores(const RelParams& p, const Seq& s, const float* bias, int i0, int j0, int ty, int tx,
                                              float (&acc)[Geo<DT>::M][Geo<DT>::M]) {
    using G = Geo<DT>;
#pragma unroll
    for (int a = 0; a < G::M; ++a) {
        const int i = i0 + ty * G::M + a;
#pragma unroll
        for (int b = 0; b < G::M; ++b) {
            const int j = j0 + tx + 16 * b, delta = j - (i + s.lk - s.lq);
            const bool seen = i < s.lq && j < s.lk && !(p.causal && delta > 0);
            acc[a][b] = seen ? fmaf(acc[a][b], p.scale2, bias_at(p, bias, delta)) : -INFINITY;
        }
    }
}

// keep[a][b] = 0 or the scale of a kept probability.
template <int DT>
__device__ __forceinline__ void draw_tile(const RelParams& p, const Seq& s, uint2 key, int h, int i0, int j0, int ty, int tx,
                                          float (&keep)[Geo<DT>::M][Geo<DT>::M]) {
    using G = Geo<DT>;
#pragma unroll
    for (int a = 0; a < G::M; ++a)
#pragma unroll
        for (int b = 0; b < G::M; b += 2) {          // columns j0 + tx + 16 b and + 16: one block of draws
            if (p.drop.thr) {
                const int j = j0 + tx + 16 * b;
                const Words4 w = draw_block(p.drop, key, draw_row(s, h, i0 + ty * G::M + a) + (uint64_t)((j >> 5) * 4 + ((j >> 1) & 3)));
                const uint32_t lo = (j & 8) ? w.w[1] : w.w[0], hi = (j & 8) ? w.w[3] : w.w[2];
                const int shift = 16 * (j & 1);
                keep[a][b] = ((lo >> shift) & 0xFFFFu) < p.drop.thr ? 0.0f : p.drop.scale;
                keep[a][b + 1] = ((hi >> shift) & 0xFFFFu) < p.drop.thr ? 0.0f : p.drop.scale;
            } else {
                keep[a][b] = keep[a][b + 1] = 1.0f;
            }
        }
}

__device__ __forceinline__ float half_warp_max(float x) {
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, o));
    return x;
}
__device__ __forceinline__ float half_warp_sum(float x) {
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, o);
    return x;
}

template <typename T, int DT>
__device__ __forceinline__ void store_rows(const RelParams& p, const TokArg& a, int head, int64_t row0, int n, int ty, int tx,
                                           const float (&acc)[Geo<DT>::M][Geo<DT>::W], const float (&f)[Geo<DT>::M]) {
    using G = Geo<DT>;
#pragma unroll
    for (int r = 0; r < G::M; ++r) {
        if (ty * G::M + r >= n) continue;
        T* out = const_cast<T*>(static_cast<const T*>(a.data)) + (row0 + ty * G::M + r) * a.tok + (int64_t)head * a.head;
#pragma unroll
        for (int w = 0; w < G::W; ++w)
            if (tx + 16 * w < p.dim) store1(out + tx + 16 * w, acc[r][w] * f[r]);
    }
}

template <typename T, int DT>
__global__ void __launch_bounds__(kThreads) forward_kernel(RelParams p, int tiles) {
    using G = Geo<DT>;
    extern __shared__ float4 smem4[];
    float* Qs = reinterpret_cast<float*>(smem4);
    float* Ks = Qs + G::B * G::LD;
    float* Vs = Ks + G::B * G::LD;
    float* Ps = Vs + G::B * G::LD;
    float* bias = Ps + G::B * G::LP;
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t sn = blockIdx.x / tiles;
    const int i0 = (int)(blockIdx.x % tiles) * G::B, h = blockIdx.y;
    Seq s;
    if (!load_seq(p, sn, s) || i0 >= s.lq) return;
    const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
    const uint2 key = p.drop.thr ? instance_key(p.drop, sn) : make_uint2(0, 0);
    fill_bias<0>(p, h, bias);
    const int nq = min(G::B, s.lq - i0), end = keys_seen(p, s, i0 + nq);
    load_tile<T, DT>(p, p.q, h, s.q0 + i0, nq, Qs);
    float m[G::M], l[G::M], acc[G::M][G::W];
#pragma unroll
    for (int a = 0; a < G::M; ++a) {
        m[a] = -INFINITY;
        l[a] = 0.0f;
#pragma unroll
        for (int w = 0; w < G::W; ++w) acc[a][w] = 0.0f;
    }
    for (int j0 = 0; j0 < end; j0 += G::B) {
        __syncthreads();                     // the previous tile's products are done
        load_tile<T, DT>(p, p.k, h / p.group, s.k0 + j0, min(G::B, s.lk - j0), Ks);
        load_tile<T, DT>(p, p.v, h / p.group, s.k0 + j0, min(G::B, s.lk - j0), Vs);
        __syncthreads();
        float t[G::M][G::M], keep[G::M][G::M];
        dot_tile<DT>(Qs, Ks, ty, tx, t);
        finish_scores<DT>(p, s, bias, i0, j0, ty, tx, t);
        draw_tile<DT>(p, s, key, h, i0, j0, ty, tx, keep);
#pragma unroll
        for (int a = 0; a < G::M; ++a) {
            float top = t[a][0];
#pragma unroll
            for (int b = 1; b < G::M; ++b) top = fmaxf(top, t[a][b]);
            top = fmaxf(m[a], half_warp_max(top));
            const float ref = top == -INFINITY ? 0.0f : top, corr = ex2_approx(m[a] - ref);
            float sum = 0.0f;
#pragma unroll
            for (int b = 0; b < G::M; ++b) {
                const float e = ex2_approx(t[a][b] - ref);
                sum += e;
                Ps[(ty * G::M + a) * G::LP + tx + 16 * b] = e * keep[a][b];
            }
            l[a] = l[a] * corr + half_warp_sum(sum);
            m[a] = top;
#pragma unroll
            for (int w = 0; w < G::W; ++w) acc[a][w] *= corr;
        }
        __syncwarp();                        // a row's probabilities come from its own half-warp
        rows_times<DT>(Ps, Vs, ty, tx, acc);
    }
#pragma unroll
    for (int a = 0; a < G::M; ++a) l[a] = l[a] == 0.0f ? 0.0f : 1.0f / l[a];
    store_rows<T, DT>(p, p.out, h, s.q0 + i0, nq, ty, tx, acc, l);
}

// dq, the row statistics (m, 1 / l, D) and this CTA's share of the table's gradient.  grid (parts, heads): a CTA walks query tiles of
// its head.  First pass: m, l and D = sum_j p_ij dp_ij from unrounded probabilities; second pass: dS, its diagonal sums, dq.
template <typename T, int DT>
__global__ void __launch_bounds__(kThreads, DT == 64 ? 2 : 1) grad_q_kernel(RelParams p, int tiles) {
    using G = Geo<DT>;
    extern __shared__ float4 smem4[];
    float* Qs = reinterpret_cast<float*>(smem4);
    float* Os = Qs + G::B * G::LD;
    float* Ks = Os + G::B * G::LD;
    float* Vs = Ks + G::B * G::LD;
    float* Ps = Vs + G::B * G::LD;
    float* bias = Ps + G::B * G::LP;
    float* bins = bias + (p.table ? 2 * p.reach + 1 : 0);
    grid_dependency_wait();
    grid_dependency_release();
    const int h = blockIdx.y, ty = threadIdx.x / 16, tx = threadIdx.x % 16;
    const bool want_table = p.table && p.dtable;
    fill_bias<0>(p, h, bias);
    if (want_table)
        for (int i = threadIdx.x; i < 2 * p.reach; i += kThreads) bins[i] = 0.0f;
    FarSums far = {0.0f, 0.0f};
    const int64_t items = counted(p.count_dev, p.n_seq) * tiles;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t sn = item / tiles;
        const int i0 = (int)(item % tiles) * G::B;
        Seq s;
        if (!load_seq(p, sn, s) || i0 >= s.lq) continue;
        const uint2 key = p.drop.thr ? instance_key(p.drop, sn) : make_uint2(0, 0);
        const int nq = min(G::B, s.lq - i0), end = keys_seen(p, s, i0 + nq);
        __syncthreads();                     // the previous item's tiles have been read
        load_tile<T, DT>(p, p.q, h, s.q0 + i0, nq, Qs);
        load_tile<T, DT>(p, p.dout, h, s.q0 + i0, nq, Os);
        float m[G::M], l[G::M], D[G::M], acc[G::M][G::W];
#pragma unroll
        for (int a = 0; a < G::M; ++a) {
            m[a] = -INFINITY;
            l[a] = D[a] = 0.0f;
#pragma unroll
            for (int w = 0; w < G::W; ++w) acc[a][w] = 0.0f;
        }
#pragma unroll 1
        for (int pass = 0; pass < 2; ++pass) {
            for (int j0 = 0; j0 < end; j0 += G::B) {
                __syncthreads();
                load_tile<T, DT>(p, p.k, h / p.group, s.k0 + j0, min(G::B, s.lk - j0), Ks);
                load_tile<T, DT>(p, p.v, h / p.group, s.k0 + j0, min(G::B, s.lk - j0), Vs);
                __syncthreads();
                float t[G::M][G::M], dp[G::M][G::M], keep[G::M][G::M];
                dot_tile<DT>(Qs, Ks, ty, tx, t);
                finish_scores<DT>(p, s, bias, i0, j0, ty, tx, t);
                dot_tile<DT>(Os, Vs, ty, tx, dp);
                draw_tile<DT>(p, s, key, h, i0, j0, ty, tx, keep);
#pragma unroll
                for (int a = 0; a < G::M; ++a)
#pragma unroll
                    for (int b = 0; b < G::M; ++b) dp[a][b] = __fmul_rn(dp[a][b], keep[a][b]);
                if (pass == 0) {
#pragma unroll
                    for (int a = 0; a < G::M; ++a) {
                        float top = t[a][0];
#pragma unroll
                        for (int b = 1; b < G::M; ++b) top = fmaxf(top, t[a][b]);
                        top = fmaxf(m[a], half_warp_max(top));
                        const float ref = top == -INFINITY ? 0.0f : top, corr = ex2_approx(m[a] - ref);
                        float sum = 0.0f, dsum = 0.0f;
#pragma unroll
                        for (int b = 0; b < G::M; ++b) {
                            const float e = ex2_approx(t[a][b] - ref);
                            sum += e;
                            dsum = fmaf(e, dp[a][b], dsum);
                        }
                        l[a] = l[a] * corr + half_warp_sum(sum);
                        D[a] = D[a] * corr + half_warp_sum(dsum);
                        m[a] = top;
                    }
                } else {
#pragma unroll
                    for (int a = 0; a < G::M; ++a)
#pragma unroll
                        for (int b = 0; b < G::M; ++b)
                            Ps[(ty * G::M + a) * G::LP + tx + 16 * b] = ex2_approx(t[a][b] - m[a]) * l[a] * (dp[a][b] - D[a]);
                    __syncthreads();
                    rows_times<DT>(Ps, Ks, ty, tx, acc);
                    if (want_table && threadIdx.x < 2 * G::B - 1) {
                        const int d = (int)threadIdx.x - (G::B - 1);           // column - row of a diagonal
                        float sum = 0.0f;
                        for (int i = max(0, -d); i < min(G::B, G::B - d); ++i) sum += Ps[i * G::LP + i + d];
                        bin_diagonal(p, bins, far, j0 - (i0 + s.lk - s.lq) + d, sum);
                    }
                }
            }
            if (pass == 0) {
#pragma unroll
                for (int a = 0; a < G::M; ++a) {
                    l[a] = l[a] == 0.0f ? 0.0f : 1.0f / l[a];                  // a row that sees nothing: p = 0 * 2^(-inf)
                    if (m[a] == -INFINITY) m[a] = 0.0f;
                    D[a] *= l[a];
                    if (tx == 0 && ty * G::M + a < nq)
                        p.stats[(int64_t)h * p.q_rows + s.q0 + i0 + ty * G::M + a] = make_float4(m[a], l[a], D[a], 0.0f);
                }
            }
        }
        float f[G::M];
#pragma unroll
        for (int a = 0; a < G::M; ++a) f[a] = p.scale;
        store_rows<T, DT>(p, p.dq, h, s.q0 + i0, nq, ty, tx, acc, f);
    }
    if (!want_table) return;
    bins[2 * p.reach + threadIdx.x] = far.neg;
    bins[2 * p.reach + kThreads + threadIdx.x] = far.pos;
    __syncthreads();
    write_table_part(p, blockIdx.x, h, bins, 0, 1, kThreads);
}

// dk and dv of one key tile and key head: the query heads that share it and the query tiles that see it, in order.
template <typename T, int DT>
__global__ void __launch_bounds__(kThreads, DT == 64 ? 2 : 1) grad_kv_kernel(RelParams p, int tiles) {
    using G = Geo<DT>;
    extern __shared__ float4 smem4[];
    float* Qs = reinterpret_cast<float*>(smem4);
    float* Os = Qs + G::B * G::LD;
    float* Ks = Os + G::B * G::LD;
    float* Vs = Ks + G::B * G::LD;
    float* Ps = Vs + G::B * G::LD;
    float* bias = Ps + G::B * G::LP;
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t sn = blockIdx.x / tiles;
    const int j0 = (int)(blockIdx.x % tiles) * G::B, hk = blockIdx.y;
    Seq s;
    if (!load_seq(p, sn, s) || j0 >= s.lk) return;
    const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
    const uint2 key = p.drop.thr ? instance_key(p.drop, sn) : make_uint2(0, 0);
    const int nk = min(G::B, s.lk - j0);
    load_tile<T, DT>(p, p.k, hk, s.k0 + j0, nk, Ks);
    load_tile<T, DT>(p, p.v, hk, s.k0 + j0, nk, Vs);
    float gk[G::M][G::W], gv[G::M][G::W];
#pragma unroll
    for (int a = 0; a < G::M; ++a)
#pragma unroll
        for (int w = 0; w < G::W; ++w) gk[a][w] = gv[a][w] = 0.0f;
    for (int h = hk * p.group; h < (hk + 1) * p.group; ++h) {
        __syncthreads();
        fill_bias<0>(p, h, bias);
        for (int i0 = first_query(p, s, j0) / G::B * G::B; i0 < s.lq; i0 += G::B) {
            const int nq = min(G::B, s.lq - i0);
            __syncthreads();
            load_tile<T, DT>(p, p.q, h, s.q0 + i0, nq, Qs);
            load_tile<T, DT>(p, p.dout, h, s.q0 + i0, nq, Os);
            __syncthreads();
            float t[G::M][G::M], dp[G::M][G::M], keep[G::M][G::M];
            dot_tile<DT>(Qs, Ks, ty, tx, t);
            finish_scores<DT>(p, s, bias, i0, j0, ty, tx, t);
            dot_tile<DT>(Os, Vs, ty, tx, dp);
            draw_tile<DT>(p, s, key, h, i0, j0, ty, tx, keep);
#pragma unroll
            for (int a = 0; a < G::M; ++a) {
                const int i = ty * G::M + a;
                const float4 st = i < nq ? p.stats[(int64_t)h * p.q_rows + s.q0 + i0 + i] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
                for (int b = 0; b < G::M; ++b) {
                    const float prob = ex2_approx(t[a][b] - st.x) * st.y;
                    dp[a][b] = prob * (__fmul_rn(dp[a][b], keep[a][b]) - st.z);
                    Ps[i * G::LP + tx + 16 * b] = prob * keep[a][b];
                }
            }
            __syncthreads();
            cols_times<DT>(Ps, Os, ty, tx, gv);
            __syncthreads();
#pragma unroll
            for (int a = 0; a < G::M; ++a)
#pragma unroll
                for (int b = 0; b < G::M; ++b) Ps[(ty * G::M + a) * G::LP + tx + 16 * b] = dp[a][b];
            __syncthreads();
            cols_times<DT>(Ps, Qs, ty, tx, gk);
        }
    }
    float f[G::M], one[G::M];
#pragma unroll
    for (int a = 0; a < G::M; ++a) {
        f[a] = p.scale;
        one[a] = 1.0f;
    }
    store_rows<T, DT>(p, p.dk, hk, s.k0 + j0, nk, ty, tx, gk, f);
    store_rows<T, DT>(p, p.dv, hk, s.k0 + j0, nk, ty, tx, gv, one);
}

// dtable[b][h] = sum of the parts: a warp per entry, lanes over the parts, joined in a fixed order.
__global__ void __launch_bounds__(256) table_grad_kernel(RelParams p) {
    grid_dependency_wait();
    grid_dependency_release();
    const int n = p.buckets * p.heads, lane = threadIdx.x & 31;
    for (int i = (blockIdx.x * 256 + threadIdx.x) >> 5; i < n; i += gridDim.x * 8) {
        const int h = i / p.buckets, b = i % p.buckets;
        double sum = 0.0;
        for (int g = lane; g < p.n_parts; g += 32) sum += (double)p.parts[((int64_t)g * p.heads + h) * p.buckets + b];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        if (lane == 0) p.dtable[b * p.heads + h] = (float)sum;
    }
}

template <typename T, int DT>
aa_status forward(aa_ctx_impl* c, RelParams p) {
    using G = Geo<DT>;
    const void* kernel = (const void*)forward_kernel<T, DT>;
    const size_t smem = G::smem(3, p.table ? 2 * p.reach + 1 : 0);
    if (allow_smem(c, kernel, smem) != AA_OK) return AA_ERR_CUDA;
    int tiles = p.max_q > 0 ? (int)((p.max_q + G::B - 1) / G::B) : 1;      // one: sequences are looked over even if none may have a query
    if (p.n_seq * tiles > 0x7FFFFFFFll) return AA_ERR_UNSUPPORTED;
    void* args[] = {&p, &tiles};
    if (launch_overlapped(c, kernel, dim3((unsigned)(p.n_seq * tiles), p.heads), dim3(kThreads), args, smem, false) != cudaSuccess)
        return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

template <typename T, int DT>
aa_status backward(aa_ctx_impl* c, RelParams p) {
    using G = Geo<DT>;
    const void* kq = (const void*)grad_q_kernel<T, DT>;
    const void* kkv = (const void*)grad_kv_kernel<T, DT>;
    const int reach = p.table ? 2 * p.reach + 1 : 0;
    const size_t smem_q = G::smem(4, reach + (p.table && p.dtable ? 2 * p.reach + 2 * kThreads : 0)), smem_kv = G::smem(4, reach);
    if (allow_smem(c, kq, smem_q) != AA_OK || allow_smem(c, kkv, smem_kv) != AA_OK) return AA_ERR_CUDA;
    int tiles_q = p.max_q > 0 ? (int)((p.max_q + G::B - 1) / G::B) : 1, tiles_k = (int)((p.max_k + G::B - 1) / G::B);
    if (p.n_seq * tiles_k > 0x7FFFFFFFll) return AA_ERR_UNSUPPORTED;
    void* args_q[] = {&p, &tiles_q};
    void* args_kv[] = {&p, &tiles_k};
    if (launch_overlapped(c, kq, dim3(p.n_parts, p.heads), dim3(kThreads), args_q, smem_q, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    if (tiles_k > 0) {
        if (launch_overlapped(c, kkv, dim3((unsigned)(p.n_seq * tiles_k), p.kv_heads), dim3(kThreads), args_kv, smem_kv, false) != cudaSuccess)
            return AA_ERR_CUDA;
        ++c->launches;
    }
    return AA_OK;
}

}  // namespace

// Operand tiles of 64, 128 or 256 columns (48 as a fourth was slower for a width of 40, at the time: 436 against 401 us for 24 sentences of up to 301 tokens,
// 5 heads, forward and every gradient).
template <typename T>
aa_status forward_width(aa_ctx_impl* c, const RelParams& p) {
    return p.dim <= 64 ? forward<T, 64>(c, p) : p.dim <= 128 ? forward<T, 128>(c, p) : forward<T, 256>(c, p);
}
template <typename T>
aa_status backward_width(aa_ctx_impl* c, const RelParams& p) {
    return p.dim <= 64 ? backward<T, 64>(c, p) : p.dim <= 128 ? backward<T, 128>(c, p) : backward<T, 256>(c, p);
}

aa_status launch_rel_attention_plain(aa_ctx_impl* c, const RelParams& p, int dtype) {
    return dtype == AA_BF16 ? forward_width<uint16_t>(c, p) : forward_width<float>(c, p);
}

aa_status launch_rel_attention_grad_plain(aa_ctx_impl* c, const RelParams& p, int dtype) {
    return dtype == AA_BF16 ? backward_width<uint16_t>(c, p) : backward_width<float>(c, p);
}

aa_status launch_rel_table_grad(aa_ctx_impl* c, const RelParams& p) {
    RelParams q = p;
    void* args[] = {&q};
    const int n = p.buckets * p.heads;
    if (launch_overlapped(c, (const void*)table_grad_kernel, dim3((n + 7) / 8), dim3(256), args, 0, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

}  // namespace aa
