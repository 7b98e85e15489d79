// Layer normalisation of rows and its gradients.
//
//   c = x - mean(x),  r = 1 / sqrt(mean(c^2) + eps),  h = c r,  out = h gamma + beta
//   g = dout gamma,   dx = r (g - mean(g) - h mean(g h)) + residual,   dgamma = sum_rows dout h,  dbeta = sum_rows dout
//
// Bound by memory where rows are short or fp32 (25,000 x 512 fp32: forward 18.8 us, 5.4 TB/s, backward 29 us, 5.3 TB/s; bf16 with residual 23 us, 4.5 TB/s), by
// instructions and the latency of sums where an SM's warps share a row (3,001 x 4,099 fp32 backward: 41 us with both launches, the floor is 22).
// 2 values a column pass forward, 3 or 4 backward.  A row stays in the registers of a group of threads (8 or 16 columns each) between its sums and its
// result, so that memory is touched once; mean and variance are two rounds over registers, so that nothing cancels.  A mean of fp32 numbers is off by a few parts in
// 2^24, which is much where it is large against their spread (a constant row of 1,000.1 would get h = 0.02 with eps = 1e-5).  So the second round adds up c too:
// with d = mean(c), c - d are the distances from the mean and mean(c^2) - d^2 is the variance.  bf16 numbers of one size add up exactly (8 bits, 8,192 columns).
// Backward the rounds carry (sum x, sum g) and (sum c^2, sum g c, sum c): mean(g h) = r mean(g (c - d)), and no statistics are kept from the forward pass (two floats a row would save one round of
// shuffles and no memory).  A group walks over rows of its own and adds up dout h and dout of its columns; the sums of a CTA's groups are joined in
// shared memory, those of the CTAs by a second kernel, both in a fixed order.
// Rows too long for registers are swept three times, and their columns are summed by a kernel of their own.
#include <type_traits>

#include "async_copy.cuh"
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
        if constexpr (G >= 256) {            // a number a lane and a tree: a third of the instructions of 16 loads
            s = mine[threadIdx.x % (G / 32)];
#pragma unroll
            for (int o = G / 64; o > 0; o >>= 1) {
                s.x += __shfl_xor_sync(0xFFFFFFFFu, s.x, o);
                s.y += __shfl_xor_sync(0xFFFFFFFFu, s.y, o);
            }
        } else {
            s = mine[0];
#pragma unroll
            for (int w = 1; w < G / 32; ++w) {
                s.x += mine[w].x;
                s.y += mine[w].y;
            }
        }
    }
    return s;
}

// The same for K values.
template <int G, int K>
__device__ __forceinline__ void group_sums(float (&s)[K], float* buf) {
    static_assert(K == 2 || K == 4 || K == 8, "");
    if constexpr (K == 2 && G > 32) {        // the shorter chain of steps
        const float2 t = group_sum<G>(make_float2(s[0], s[1]), reinterpret_cast<float2*>(buf));
        s[0] = t.x;
        s[1] = t.y;
        return;
    }
    const int lane = threadIdx.x & 31;
    // a warp halves the number of values a lane has with the first steps: value q ends up in the lanes with q = lane % K
    float w[K];
#pragma unroll
    for (int q = 0; q < K; ++q) w[q] = s[q];
#pragma unroll
    for (int o = K / 2; o > 0; o /= 2) {
        const bool up = lane & o;
#pragma unroll
        for (int q = 0; q < o; ++q) w[q] = (up ? w[q + o] : w[q]) + __shfl_xor_sync(0xFFFFFFFFu, up ? w[q] : w[q + o], o);
    }
    float t = w[0];
#pragma unroll
    for (int o = K; o < (G < 32 ? G : 32); o *= 2) t += __shfl_xor_sync(0xFFFFFFFFu, t, o);
    if constexpr (G > 32) {
        constexpr int WARPS = G / 32, ALL = WARPS * K;
        const int group = threadIdx.x / G;
        float* mine = buf + group * ALL;
        if (lane < K) mine[(threadIdx.x % G >> 5) * K + lane] = t;
        if constexpr (kThreadsOf<G> == G) __syncthreads();
        else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(G) : "memory");
        t = mine[lane % ALL];
#pragma unroll
        for (int i = 32; i < ALL; i += 32) t += mine[lane + i];
#pragma unroll
        for (int o = K; o < (ALL < 32 ? ALL : 32); o *= 2) t += __shfl_xor_sync(0xFFFFFFFFu, t, o);
    }
#pragma unroll
    for (int q = 0; q < K; ++q) s[q] = __shfl_sync(0xFFFFFFFFu, t, G < 32 ? (lane & ~(G - 1)) | q : q);
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
    constexpr bool FINE = sizeof(T) == 4;    // the mean is corrected
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
        for (int j = 0; j < E; ++j) s.x += v[j];
        const float mean = __fdiv_rn(group_sum<G>(s, buf[0]).x, (float)cols);
        s = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            v[j] = first + j / V * step < cols ? v[j] - mean : 0.0f;
            s.x = fmaf(v[j], v[j], s.x);
            if (FINE) s.y += v[j];
        }
        s = group_sum<G>(s, buf[1]);
        const float d = FINE ? s.y * inv : 0.0f, r = rsqrtf((FINE ? fmaxf(fmaf(-d, s.y, s.x), 0.0f) : s.x) * inv + p.eps);
        T* out = static_cast<T*>(const_cast<void*>(p.out.data)) + row * p.out.stride;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = first + i * step;
            if (c >= cols || row >= live) continue;
#pragma unroll
            for (int e = 0; e < V; ++e) v[i * V + e] = fmaf((FINE ? v[i * V + e] - d : v[i * V + e]) * r, gm[i * V + e], bt[i * V + e]);
            store_elems<T, V>(out + c, v + i * V);
        }
    }
}

// A row's columns of this thread in shared memory, fetched by asynchronous copies that only this thread waits for: [word][thread], so that the threads of a
// warp read neighbouring words.
template <typename T, int V, int E, int TH>
struct Slot {
    using Word = typename Raw<T, V, E>::Word;
    static constexpr int N = E / V, BYTES = N * TH * (int)sizeof(Word);
    __device__ static __forceinline__ void clear(char* at) {
#pragma unroll
        for (int i = 0; i < N; ++i) reinterpret_cast<Word*>(at)[i * TH + threadIdx.x] = Word{};
    }
    __device__ static __forceinline__ void fetch(char* at, const T* row, int first, int step, int cols) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t to = smem_u32(reinterpret_cast<Word*>(at) + i * TH + threadIdx.x);
            if (first + i * step >= cols) continue;
            if constexpr (sizeof(Word) == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(row + first + i * step) : "memory");
            else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(row + first + i * step) : "memory");
        }
    }
    __device__ static __forceinline__ void read(const char* at, Raw<T, V, E>& x) {
#pragma unroll
        for (int i = 0; i < N; ++i) x.w[i] = reinterpret_cast<const Word*>(at)[i * TH + threadIdx.x];
    }
};

// The same for rows that start anywhere (V = 1, groups of whole warps): a warp has 32 E neighbouring columns, lane l those numbered l, l + 32, ...; it fetches
// the 16-byte words that cover them and finds its elements behind a shift.  Words that reach beyond the row lie in the matrix all the same
// (`lo`, `hi`: its ends); the few that do not are fetched element by element.
template <typename T, int E, int TH>
struct Shifted {
    static constexpr int WARP = 32 * E * (int)sizeof(T) + 16, BYTES = TH / 32 * WARP, TRIPS = (WARP / 16 + 31) / 32;
    // n: columns of the warp that count, 32 E at most
    __device__ static __forceinline__ void fetch(char* at, const T* seg, int n, const char* lo, const char* hi) {
        if (n <= 0) return;
        const int lane = threadIdx.x & 31;
        const uint32_t shift = (uint32_t)(uintptr_t)seg & 15u;
        const char* from = reinterpret_cast<const char*>(seg) - shift;
        char* to = at + (threadIdx.x >> 5) * WARP;
        const int words = (n * (int)sizeof(T) + (int)shift + 15) / 16;
        if (from >= lo && from + words * 16 <= hi) {
            const uint32_t at32 = smem_u32(to) + lane * 16;
            const char* src = from + lane * 16;
#pragma unroll
            for (int q = 0; q < TRIPS; ++q)
                if (lane + 32 * q < words) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at32 + 512 * q), "l"(src + 512 * q) : "memory");
            return;
        }
        for (int j = lane; j < words; j += 32) {
            const char* src = from + j * 16;
            if (src >= lo && src + 16 <= hi) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to + j * 16)), "l"(src) : "memory");
            } else {
                for (int e = 0; e < 16; e += (int)sizeof(T))
                    if (src + e >= lo && src + e + (int)sizeof(T) <= hi) *reinterpret_cast<T*>(to + j * 16 + e) = *reinterpret_cast<const T*>(src + e);
            }
        }
    }
    // seg: the low bits of the address
    __device__ static __forceinline__ void read(const char* at, uint32_t seg, Raw<T, 1, E>& x) {
        const T* from = reinterpret_cast<const T*>(at + (threadIdx.x >> 5) * WARP + (seg & 15u)) + (threadIdx.x & 31);
#pragma unroll
        for (int i = 0; i < E; ++i) x.w[i] = from[32 * i];
    }
};

// R rows of a group are worked on at a time - two where all warps of an SM are one group and registers hold both (10 columns a thread; with 11 they spill): barriers and the
// latency of sums come once for both (3,001 x 4,099 fp32: 43.3 us one by one, 40.9 in twos; 2,600 x 4,700 bf16 35.0 and 34.4; groups of 256 threads gain nothing).  `steps` times R rows are under way; a step's place is
// filled again as soon as its numbers are in registers.
template <typename T, int V, int E, int G, int R>
__global__ void __launch_bounds__(kThreadsOf<G>, 512 / kThreadsOf<G>) norm_grad_kernel(NormParams p, int steps) {
    constexpr int TH = kThreadsOf<G>, N = E / V;
    constexpr bool SHIFT = V == 1, FINE = sizeof(T) == 4;
    constexpr int K = FINE ? 4 : 2;          // sums of a row's second round
    static_assert(R == 1 || G >= 32, "a group's second row is skipped by whole warps");
    using S = Slot<T, V, E, TH>;
    using U = Shifted<T, E, TH>;
    constexpr int BYTES = SHIFT ? U::BYTES : S::BYTES;
    __shared__ __align__(8) float buf[2][TH / 32 * K * R];
    extern __shared__ __align__(16) char ring[];     // [steps, 1 or 2][R][x, dout, residual if there is one]; at the end the column sums
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, blockIdx.x == 0 && threadIdx.x == 0);
    const int l = threadIdx.x % G, groups = TH / G;
    const int cols = (int)p.cols, seg = (l & ~31) * E, first = SHIFT ? seg + (l & 31) : l * V, step = SHIFT ? 32 : G * V;
    const int n_warp = min(cols - seg, 32 * E);
    // every column of the warp (of the row, where lanes hold vectors) is one: no tests on the way
    const bool full = SHIFT ? n_warp == 32 * E : N * step <= cols, extra = p.residual.data != nullptr;
    const int row_bytes = (extra ? 3 : 2) * BYTES;
    const float inv = 1.0f / (float)cols;
    float gm[E], dg[E], db[E];
#pragma unroll
    for (int j = 0; j < E; ++j) {
        const int c = first + j / V * step + j % V;
        gm[j] = c < cols ? (p.gamma ? p.gamma[c] : 1.0f) : 0.0f;
        dg[j] = db[j] = 0.0f;
    }
    const int64_t jump = (int64_t)gridDim.x * groups;
    // the lanes of a warp keep step: rows past the end are looked at as the last one and not written
    const int64_t mine = (int64_t)blockIdx.x * groups + threadIdx.x / G;
    const auto row_of = [&](const MatArg& m, int64_t row) { return static_cast<const T*>(m.data) + row * m.stride; };
    const auto end_of = [&](const MatArg& m) { return reinterpret_cast<const char*>(row_of(m, live - 1) + cols); };
    const auto fetch_one = [&](char* at, const MatArg& m, int64_t row) {
        if constexpr (SHIFT) U::fetch(at, row_of(m, row) + seg, n_warp, static_cast<const char*>(m.data), end_of(m));
        else S::fetch(at, row_of(m, row), first, step, cols);
    };
    const auto read_one = [&](const char* at, const MatArg& m, int64_t row, Raw<T, V, E>& w) {
        if constexpr (SHIFT) U::read(at, (uint32_t)(uintptr_t)m.data + ((uint32_t)row * (uint32_t)m.stride + (uint32_t)seg) * (uint32_t)sizeof(T), w);
        else S::read(at, w);
    };
    // a group goes on while the first of its warp's rows does
    const int64_t lead = G >= 32 ? mine : (int64_t)blockIdx.x * groups + (threadIdx.x & ~31) / G;
    const auto fetch = [&](int64_t r, int slot) {
#pragma unroll
        for (int q = 0; q < R; ++q) {
            if (lead + r + q * jump >= live) continue;
            const int64_t row = G >= 32 ? mine + r + q * jump : min(mine + r, live - 1);
            char* at = ring + (slot * R + q) * row_bytes;
            fetch_one(at, p.x, row);
            fetch_one(at + BYTES, p.dout, row);
            if (extra) fetch_one(at + 2 * BYTES, p.residual, row);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if constexpr (!SHIFT)
        for (int a = 0; a < steps * row_bytes / BYTES * R; ++a) S::clear(ring + a * BYTES);
    for (int a = 0; a < steps; ++a) fetch(a * R * jump, a);
    int slot = 0;
    for (int64_t r = 0; lead + r < live; r += R * jump) {
        if (steps == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
        else asm volatile("cp.async.wait_group 0;" ::: "memory");
        if (SHIFT) __syncwarp();
        Raw<T, V, E> res[R];
        float v[R][E], u[R][E], s[2 * R] = {};
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const int64_t row = mine + r + q * jump;
            const char* at = ring + (slot * R + q) * row_bytes;
            Raw<T, V, E> x, d;
            read_one(at, p.x, row, x);
            read_one(at + BYTES, p.dout, row, d);
            if (extra) read_one(at + 2 * BYTES, p.residual, row, res[q]);
            // (the values of vectors behind the end are zeros already)
            const auto first_sums = [&](auto all) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    x.values(i, v[q] + i * V);
                    d.values(i, u[q] + i * V);
                    if constexpr (SHIFT && !all.value) {
                        const bool has = first + i * step < cols;
                        v[q][i] = has ? v[q][i] : 0.0f;
                        u[q][i] = has ? u[q][i] : 0.0f;
                    }
                }
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    s[2 * q] += v[q][j];
                    s[2 * q + 1] = fmaf(u[q][j], gm[j], s[2 * q + 1]);
                }
            };
            if (full) first_sums(std::true_type{});
            else first_sums(std::false_type{});
        }
        if (SHIFT) __syncwarp();             // the slot's readers are done
        fetch(r + steps * R * jump, slot);
        slot = slot + 1 == steps ? 0 : slot + 1;
        group_sums<G>(s, buf[0]);
        float mg[R], t[K * R] = {};          // t: sums of c^2, c g, c
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const float mean = __fdiv_rn(s[2 * q], (float)cols);
            mg[q] = s[2 * q + 1] * inv;
            const auto second_sums = [&](auto all) {
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    v[q][j] = all.value || first + j / V * step < cols ? v[q][j] - mean : 0.0f;
                    t[K * q] = fmaf(v[q][j], v[q][j], t[K * q]);
                    t[K * q + 1] = fmaf(v[q][j], u[q][j] * gm[j], t[K * q + 1]);
                    if (FINE) t[K * q + 2] += v[q][j];
                }
            };
            if (full) second_sums(std::true_type{});
            else second_sums(std::false_type{});
        }
        group_sums<G>(t, buf[1]);
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const int64_t row = mine + r + q * jump;
            const bool on = (G >= 32 && q == 0) || row < live;
            if (q > 0 && !on) continue;
            const float sum_c = FINE ? t[K * q + K - 2] : 0.0f, d = sum_c * inv;
            const float rs = rsqrtf((FINE ? fmaxf(fmaf(-d, sum_c, t[K * q]), 0.0f) : t[K * q]) * inv + p.eps);
            const float k = (FINE ? fmaf(-mg[q], sum_c, t[K * q + 1]) : t[K * q + 1]) * inv * rs;
            T* out = static_cast<T*>(const_cast<void*>(p.out.data)) + row * p.out.stride;
            const auto finish = [&](auto all) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const int c = first + i * step;
                    float y[V];
                    if (extra) res[q].values(i, y);
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const int j = i * V + e;
                        const float h = (FINE ? v[q][j] - d : v[q][j]) * rs, w = on ? u[q][j] : 0.0f;
                        dg[j] = fmaf(w, h, dg[j]);
                        db[j] += w;
                        const float z = rs * (fmaf(u[q][j], gm[j], -mg[q]) - h * k);
                        y[e] = extra ? z + y[e] : z;
                    }
                    if ((all.value || c < cols) && on) store_elems<T, V>(out + c, y);
                }
            };
            if (full) finish(std::true_type{});
            else finish(std::false_type{});
        }
    }
    if (!p.parts) return;
    float* to = p.parts + (int64_t)blockIdx.x * 2 * cols;
    if constexpr (TH == G) {
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const int c = first + j / V * step + j % V;
            if (c < cols) {
                to[c] = dg[j];
                to[cols + c] = db[j];
            }
        }
    } else {
        // [group][2][columns]: a CTA's groups one after the other
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();
        float* sums = reinterpret_cast<float*>(ring) + (threadIdx.x / G) * 2 * G * E;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const int c = first + j / V * step + j % V;
            sums[c] = dg[j];
            sums[G * E + c] = db[j];
        }
        __syncthreads();
        for (int c = threadIdx.x; c < 2 * cols; c += TH) {
            const int at = c < cols ? c : G * E + c - cols;
            float t = 0.0f;
            for (int w = 0; w < groups; ++w) t += reinterpret_cast<const float*>(ring)[w * 2 * G * E + at];
            to[c] = t;
        }
    }
}

// ---------------------------------------------------------------------- rows too long for registers

constexpr int kSweep = 512;

// f(first column, its V values) over a row by the CTA.
template <typename T, int V, typename F>
__device__ __forceinline__ void sweep(const T* row, int64_t cols, F f) {
#pragma unroll 4
    for (int64_t c = threadIdx.x * V; c < cols; c += kSweep * V) {
        float x[V];
        load_elems<T, V>(row + c, x);
        f(c, x);
    }
}

template <typename T, int V>
__device__ __forceinline__ NormStats row_stats(const NormParams& p, const T* x, float2 (*buf)[32]) {
    float2 s = make_float2(0.0f, 0.0f);
    sweep<T, V>(x, p.cols, [&](int64_t, const float* v) {
#pragma unroll
        for (int e = 0; e < V; ++e) s.x += v[e];
    });
    const float mean = __fdiv_rn(group_sum<kSweep>(s, buf[0]).x, (float)p.cols);
    s = make_float2(0.0f, 0.0f);
    sweep<T, V>(x, p.cols, [&](int64_t, const float* v) {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            s.x = fmaf(v[e] - mean, v[e] - mean, s.x);
            s.y += v[e] - mean;
        }
    });
    s = group_sum<kSweep>(s, buf[1]);
    const float d = s.y / (float)p.cols;
    return NormStats{mean, d, 1.0f / sqrtf(fmaxf(fmaf(-d, s.y, s.x), 0.0f) / (float)p.cols + p.eps), 0.0f};
}

template <typename T, int V>
__global__ void __launch_bounds__(kSweep) norm_sweep_kernel(NormParams p) {
    __shared__ float2 buf[2][32];
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, blockIdx.x == 0 && threadIdx.x == 0);
    for (int64_t row = blockIdx.x; row < live; row += gridDim.x) {
        const T* x = static_cast<const T*>(p.x.data) + row * p.x.stride;
        T* out = static_cast<T*>(const_cast<void*>(p.out.data)) + row * p.out.stride;
        const NormStats st = row_stats<T, V>(p, x, buf);
        sweep<T, V>(x, p.cols, [&](int64_t c, float* v) {
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = fmaf(st.h(v[e]), p.gamma ? p.gamma[c + e] : 1.0f, p.beta ? p.beta[c + e] : 0.0f);
            store_elems<T, V>(out + c, v);
        });
    }
}

// Sums of dout h and dout over runs of rows, before the rows' own kernel may overwrite x or dout.
template <typename T, int V>
__global__ void __launch_bounds__(128) norm_columns_kernel(NormParams p) {
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, false);
    const int64_t c = ((int64_t)blockIdx.x * 128 + threadIdx.x) * V;
    if (c >= p.cols) return;
    const int64_t run = (p.live.rows + kSweepParts - 1) / kSweepParts, r0 = run * blockIdx.y, r1 = min(live, r0 + run);
    float a[V] = {}, b[V] = {};
#pragma unroll 4
    for (int64_t row = r0; row < r1; ++row) {
        const NormStats st = p.stats[row];
        float d[V], x[V];
        load_elems<T, V>(static_cast<const T*>(p.dout.data) + row * p.dout.stride + c, d);
        load_elems<T, V>(static_cast<const T*>(p.x.data) + row * p.x.stride + c, x);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            a[e] = fmaf(d[e], st.h(x[e]), a[e]);
            b[e] += d[e];
        }
    }
    float* to = p.parts + (int64_t)blockIdx.y * 2 * p.cols;
#pragma unroll
    for (int e = 0; e < V; ++e) {
        to[c + e] = a[e];
        to[p.cols + c + e] = b[e];
    }
}

template <typename T, int V>
__global__ void __launch_bounds__(kSweep) norm_stats_kernel(NormParams p) {
    __shared__ float2 buf[2][32];
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, blockIdx.x == 0 && threadIdx.x == 0);
    for (int64_t row = blockIdx.x; row < live; row += gridDim.x) {
        const NormStats st = row_stats<T, V>(p, static_cast<const T*>(p.x.data) + row * p.x.stride, buf);
        if (threadIdx.x == 0) p.stats[row] = st;
    }
}

template <typename T, int V>
__global__ void __launch_bounds__(kSweep) norm_grad_sweep_kernel(NormParams p) {
    __shared__ float2 buf[32];
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, false);
    const float inv = 1.0f / (float)p.cols;
    for (int64_t row = blockIdx.x; row < live; row += gridDim.x) {
        const T *x = static_cast<const T*>(p.x.data) + row * p.x.stride, *d = static_cast<const T*>(p.dout.data) + row * p.dout.stride;
        const T* res = p.residual.data ? static_cast<const T*>(p.residual.data) + row * p.residual.stride : nullptr;
        T* out = static_cast<T*>(const_cast<void*>(p.out.data)) + row * p.out.stride;
        const NormStats st = p.stats[row];
        float2 s = make_float2(0.0f, 0.0f);
        sweep<T, V>(d, p.cols, [&](int64_t c, const float* u) {
            float v[V];
            load_elems<T, V>(x + c, v);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float g = u[e] * (p.gamma ? p.gamma[c + e] : 1.0f);
                s.x += g;
                s.y = fmaf(g, st.h(v[e]), s.y);
            }
        });
        s = group_sum<kSweep>(s, buf);
        const float mg = s.x * inv, k = s.y * inv;
        sweep<T, V>(d, p.cols, [&](int64_t c, const float* u) {
            float v[V], y[V];
            load_elems<T, V>(x + c, v);
            if (res) load_elems<T, V>(res + c, y);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float z = st.r * (u[e] * (p.gamma ? p.gamma[c + e] : 1.0f) - mg - st.h(v[e]) * k);
                y[e] = res ? z + y[e] : z;
            }
            store_elems<T, V>(out + c, y);
        });
        __syncthreads();                     // buf is read by all before the next row writes it
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
    constexpr int TH = kThreadsOf<G>, groups = TH / G, R = G >= 512 && E <= 10 ? 2 : 1;
    const void* kernel = grad ? (const void*)norm_grad_kernel<T, V, E, G, R> : (const void*)norm_kernel<T, V, E, G>;
    // two steps, one where two would hold more than 150 KB an SM: more are slower (25,000 x 512 fp32: 29.1 us with two, 29.9 with three, 32.1 with four, 33.3 with
    // one; 6,000 x 2,048 with residual, 98 KB a step: 38.8 with one, 42.6 with two)
    const size_t sums = TH == G ? 1 : 2 * sizeof(float) * E * TH, room = (size_t)150 * 1024 * TH / 512;
    const size_t one = (size_t)R * (p.residual.data ? 3 : 2) * (V == 1 ? Shifted<T, E, TH>::BYTES : Slot<T, V, E, TH>::BYTES);
    int steps = (int)(room / one);
    steps = steps > 2 ? 2 : (steps < 1 ? 1 : steps);
    const size_t smem = !grad ? 0 : (sums > steps * one ? sums : steps * one);
    if (smem && allow_smem(c, kernel, smem) != AA_OK) return AA_ERR_CUDA;
    int ctas = resident_ctas(c, kernel, TH, smem);
    if (ctas < 1) return AA_ERR_CUDA;
    const int64_t wanted = (p.live.rows + groups - 1) / groups;
    if (grad && ctas > kNormParts) ctas = kNormParts;
    if (ctas > wanted) ctas = (int)wanted;
    void* args[] = {&p, &steps};             // (the forward kernel takes the first alone)
    if (launch_overlapped(c, kernel, dim3(ctas), dim3(TH), args, smem, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    *n_parts = ctas;
    return AA_OK;
}

// 512 threads with E columns each or, if the row has more, with the next multiple of V.
template <typename T, int V, int E>
aa_status launch_wide(aa_ctx_impl* c, const NormParams& p, bool grad, int* n) {
    if constexpr (E < 16)
        if (p.cols > 512 * E) return launch_wide<T, V, E + V>(c, p, grad, n);
    return launch_rows<T, V, E, 512>(c, p, grad, n);
}

// The smallest group whose threads have 16 columns of bf16 each, or 8 of fp32 (more where no group is that wide, 8 where rows go in twos).
template <typename T, int V>
aa_status launch_width(aa_ctx_impl* c, const NormParams& p, bool grad, int* n) {
    if constexpr (V == 1) {                  // whole warps, see Shifted
        if (p.cols <= 128) return launch_rows<T, V, 4, 32>(c, p, grad, n);
        if (p.cols <= 256) return launch_rows<T, V, 8, 32>(c, p, grad, n);
    } else if constexpr (V == 8) {
        if (p.cols <= 128) return launch_rows<T, V, 16, 8>(c, p, grad, n);
        if (p.cols <= 256) return launch_rows<T, V, 16, 16>(c, p, grad, n);
    } else {
        if (p.cols <= 128) return launch_rows<T, V, 8, 16>(c, p, grad, n);
        if (p.cols <= 256) return launch_rows<T, V, 8, 32>(c, p, grad, n);
    }
    if constexpr (sizeof(T) == 2) {
        if (p.cols <= 512) return launch_rows<T, V, 16, 32>(c, p, grad, n);
        if (p.cols <= 1024) return launch_rows<T, V, 16, 64>(c, p, grad, n);
        if (p.cols <= 2048) return launch_rows<T, V, 16, 128>(c, p, grad, n);
        // backward, rows in twos: 3,000 x 4,096 takes 30 us, 32 with 16 columns a thread
        if (p.cols <= 4096) return grad && V == 8 ? launch_rows<T, V, 8, 512>(c, p, grad, n) : launch_rows<T, V, 16, 256>(c, p, grad, n);
    } else {
        if (p.cols <= 512) return launch_rows<T, V, 8, 64>(c, p, grad, n);
        if (p.cols <= 1024) return launch_rows<T, V, 8, 128>(c, p, grad, n);
        if (p.cols <= 2048) return launch_rows<T, V, 8, 256>(c, p, grad, n);
        if (p.cols <= 4096) return launch_rows<T, V, 8, 512>(c, p, grad, n);
    }
    // all of a CTA's threads hold the row: as many columns each as it takes (1,900 x 6,501 fp32, backward: 37.8 us with 13, 41.6 with 16; 2,400 x 5,100 bf16 34 with 10, 36 with 12)
    return launch_wide<T, V, (8 / V + 1) * V>(c, p, grad, n);
}

template <typename T, int V>
aa_status launch_sweeps(aa_ctx_impl* c, NormParams p, bool grad, int* n_parts) {
    const int grid = (int)(p.live.rows < 4 * c->sm_count ? p.live.rows : 4 * c->sm_count);
    void* args[] = {&p};
    const void* first = grad ? (const void*)norm_stats_kernel<T, V> : (const void*)norm_sweep_kernel<T, V>;
    if (launch_overlapped(c, first, dim3(grid), dim3(kSweep), args, 0, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    if (!grad) return AA_OK;
    if (p.parts) {
        if (launch_overlapped(c, (const void*)norm_columns_kernel<T, V>, dim3((unsigned)((p.cols + 128 * V - 1) / (128 * V)), kSweepParts), dim3(128), args, 0, false) != cudaSuccess)
            return AA_ERR_CUDA;
        ++c->launches;
    }
    if (launch_overlapped(c, (const void*)norm_grad_sweep_kernel<T, V>, dim3(grid), dim3(kSweep), args, 0, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    *n_parts = kSweepParts;
    return AA_OK;
}

template <typename T, int V>
aa_status launch_norm(aa_ctx_impl* c, const NormParams& p, bool grad, int* n) {
    return p.cols > kNormInRegisters ? launch_sweeps<T, V>(c, p, grad, n) : launch_width<T, V>(c, p, grad, n);
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
    if (dtype == AA_BF16) st = vec ? launch_norm<uint16_t, 8>(c, p, grad, &n_parts) : launch_norm<uint16_t, 1>(c, p, grad, &n_parts);
    else st = vec ? launch_norm<float, 4>(c, p, grad, &n_parts) : launch_norm<float, 1>(c, p, grad, &n_parts);
    if (st != AA_OK || !grad || !p.parts) return st;
    float* parts = p.parts;
    int64_t cols = p.cols;
    void* args[] = {&parts, &n_parts, &cols, &dgamma, &dbeta};
    if (launch_overlapped(c, (const void*)norm_join_kernel, dim3((unsigned)((2 * cols + 31) / 32)), dim3(256), args, 0, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

}  // namespace aa
