// Tiles of the tensor-core products: in which order a launch takes them, and which it cuts along the contraction so that the last round of SMs is full.
#pragma once

#include "cta_pair.cuh"
#include "linear.cuh"

namespace aa {

constexpr int kSlice = 64, kGroupM = 16;

// What a launch does in which order: the first `whole` tiles at once, the others in `splits` parts each.
struct Plan {
    int nt, whole, splits;
    float* parts;                        // [part][rows of a tile][columns of a tile]
    float* sum_parts;                    // [part][rows of a tile]
    int cluster;                         // above 1: the parts of a tile are the CTAs of a cluster, which join them themselves (no scratch memory)
};

// CTAs that share a tile as a cluster, where there are few tiles and no scratch memory: as many as run at once, up to eight, with a
// slice or more apiece (fp32, 200 x 300 -> 700 from a flushed L2: 33 us with four slices at least, 28 with two, 25 with one; bf16, 24 x 512 -> 512: 12, 10, 10).
inline int tile_cluster(aa_ctx_impl* c, const void* kernel, int threads, size_t smem, const ProductParams& p, int64_t tiles) {
    const int64_t slices = (p.k + kSlice - 1) / kSlice;
    int n = 8;
    while (n > 1 && (tiles * n > c->sm_count || slices < n || resident_clusters(c, kernel, threads, smem, n) < tiles)) n /= 2;
    return p.parts ? 1 : n;
}

// Splits of the tiles that do not fill a round of `teams`: the fewest slices one after the other, counting the parts' way through memory.
// slice_us: what a slice of a tile takes.
inline Plan make_plan(const ProductParams& p, int64_t tiles, int nt, int teams, int64_t tile_floats, int tile_rows, double slice_us, int cluster) {
    Plan plan{nt, (int)tiles, 1, p.parts, nullptr, cluster};
    const int64_t slices = (p.k + kSlice - 1) / kSlice, whole = tiles / teams * teams, tail = tiles - whole;
    if (cluster > 1) plan.whole = 0, plan.splits = cluster;
    if (!p.parts) return plan;
    if (tail == 0) return plan;
    double best = (double)slices;
    for (int s = 2; s <= 16 && slices / s >= 4; ++s) {
        const int64_t parts = tail * s;
        if (parts * (tile_floats + tile_rows) > p.part_floats) break;
        // the parts are written and read at about 5 TB/s, behind a launch of about 4 us
        const double cost = (double)((parts + teams - 1) / teams) * (double)((slices + s - 1) / s) + (4.0 + (double)(parts * tile_floats) * 8.0 / 5e6) / slice_us;
        if (cost < best) {
            best = cost;
            plan.whole = (int)whole;
            plan.splits = s;
            plan.sum_parts = p.parts + parts * tile_floats;
        }
    }
    return plan;
}

#ifdef __CUDACC__

struct Unit {
    int m, n, s0, s1, part;              // slices [s0, s1); part < 0: the whole tile
};

__device__ __forceinline__ void tile_at(int mt, int nt, int i, int& m, int& n) {
    const int per = kGroupM * nt, g = i / per, in = i - g * per, rows = min(kGroupM, mt - g * kGroupM);
    n = in / rows;
    m = g * kGroupM + (in - n * rows);
}
__device__ __forceinline__ int units_of(const Plan& p, int mt) {
    const int tiles = mt * p.nt;
    return tiles <= p.whole ? tiles : p.whole + (tiles - p.whole) * p.splits;
}
__device__ __forceinline__ Unit unit_at(const Plan& p, int mt, int slices, int i) {
    Unit u;
    if (i < p.whole) {
        tile_at(mt, p.nt, i, u.m, u.n);
        u.s0 = 0;
        u.s1 = slices;
        u.part = -1;
    } else {
        const int j = i - p.whole, t = j / p.splits, q = j - t * p.splits;
        tile_at(mt, p.nt, p.whole + t, u.m, u.n);
        u.s0 = (int)((uint32_t)slices * (uint32_t)q / (uint32_t)p.splits);       // 2^25 slices in 16 parts at most
        u.s1 = (int)((uint32_t)slices * (uint32_t)(q + 1) / (uint32_t)p.splits);
        u.part = j;
    }
    return u;
}

// The bias of the columns from `col` on that count.
__device__ __forceinline__ void load_bias(const ProductParams& p, int64_t col, float (&bias)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) bias[e] = p.bias && col + e < p.n ? p.bias[col + e] : 0.0f;
}

// Bias, pre, activation, residual and the rounding of four neighbouring columns (those below p.n count) of N rows `step` apart (those below `end`).
// vec: pointers allow vectors.  The residuals are loaded first, so that the rows' loads are under way together.
template <typename T, int N>
__device__ __forceinline__ void finish_quads(const ProductParams& p, float (&z)[N * 4], const float (&bias)[4], int64_t row, int64_t step, int64_t end, int64_t col, bool vec) {
    T* out = static_cast<T*>(const_cast<void*>(p.out.data)) + row * p.out.stride + col;
    T* pre = p.pre.data ? static_cast<T*>(const_cast<void*>(p.pre.data)) + row * p.pre.stride + col : nullptr;
    const T* res = p.residual.data ? static_cast<const T*>(p.residual.data) + row * p.residual.stride + col : nullptr;
    const int rows = (int)min((int64_t)N, (end - row + step - 1) / step), cols = (int)min((int64_t)4, p.n - col);
    if (rows <= 0 || cols <= 0) return;
    float y[N * 4];
#pragma unroll
    for (int i = 0; i < N * 4; ++i) y[i] = 0.0f;
    if (vec && cols == 4) {
        if (res) {
#pragma unroll
            for (int q = 0; q < N; ++q) {
                float v[4];
                load_quad(res + (int64_t)min(q, rows - 1) * step * p.residual.stride, v);
#pragma unroll
                for (int e = 0; e < 4; ++e) y[q * 4 + e] = v[e];
            }
        }
    } else if (res) {
#pragma unroll
        for (int i = 0; i < N * 4; ++i) y[i] = load1(res + (int64_t)min(i / 4, rows - 1) * step * p.residual.stride + min(i % 4, cols - 1));
    }
#pragma unroll
    for (int i = 0; i < N * 4; ++i) z[i] += bias[i % 4];
    const auto put = [&](T* to, int64_t stride) {
#pragma unroll
        for (int q = 0; q < N; ++q) {
            if (q >= rows) continue;
            T* at = to + (int64_t)q * step * stride;
            if (vec && cols == 4) {
                const float v[4] = {z[q * 4], z[q * 4 + 1], z[q * 4 + 2], z[q * 4 + 3]};
                store_quad(at, v);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < cols) store1(at + e, z[q * 4 + e]);
            }
        }
    };
    if (pre) put(pre, p.pre.stride);
    activate_all<sizeof(T) == 4>(z, p.act);
#pragma unroll
    for (int i = 0; i < N * 4; ++i) z[i] += y[i];
    put(out, p.out.stride);
}

// A warp's 32 rows of 32 columns (a lane has 32 columns of row `lane` of them in sum[32 C..]) through its stage, so that eight lanes write a row's 128 bytes
// together: as a part (`part`: its first row and column, BN apart) or finished.  row0, col: of the warp's first row and of this lane's four columns.
template <typename T, int C, int BN>
__device__ __forceinline__ void finish_chunk(const ProductParams& p, float* part, float* stage, const float (&sum)[64], const float (&bias)[4], int64_t row0, int64_t end, int64_t col, bool vec) {
    constexpr int kAtOnce = 4;
    const int lane = threadIdx.x & 31, sub = lane & 7, r8 = lane >> 3;
    __syncwarp();                            // the stage's readers of the chunk before are done
#pragma unroll
    for (int w = 0; w < 8; ++w)
        *reinterpret_cast<float4*>(stage + lane * 32 + ((w ^ (lane & 7)) << 2)) =
            make_float4(sum[C * 32 + 4 * w], sum[C * 32 + 4 * w + 1], sum[C * 32 + 4 * w + 2], sum[C * 32 + 4 * w + 3]);
    __syncwarp();
#pragma unroll 1
    for (int q0 = 0; q0 < 8; q0 += kAtOnce) {
        float z[kAtOnce * 4];
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
            const int r = (q0 + q) * 4 + r8;
            const float4 f = *reinterpret_cast<const float4*>(stage + r * 32 + ((sub ^ (r & 7)) << 2));
            z[q * 4] = f.x, z[q * 4 + 1] = f.y, z[q * 4 + 2] = f.z, z[q * 4 + 3] = f.w;
            if (part) *reinterpret_cast<float4*>(part + r * BN + sub * 4) = f;
        }
        if (!part) finish_quads<T, kAtOnce>(p, z, bias, row0 + q0 * 4 + r8, 4, end, col, vec);
    }
}

// The CTAs of a cluster have the parts of a tile of 128 rows in [CTA][128 / cluster rows][BN] of everybody's `parts` (shared memory): this CTA finishes its rows.
// `threads` threads (a multiple of BN / 4) from `tid` on; after a cluster barrier.
template <typename T, int BN>
__device__ __forceinline__ void finish_cluster(const ProductParams& p, const Plan& plan, const Unit& u, const float* parts, int64_t m_end, bool vec, int tid, int threads) {
    constexpr int kAtOnce = 2, kQuads = BN / 4;
    const int rows = 128 / plan.cluster, rank = (int)cluster_rank(), step = threads / kQuads, c = tid % kQuads * 4;
    const int64_t row0 = (int64_t)u.m * 128 + rank * rows, end = min(m_end, row0 + rows), col = (int64_t)u.n * BN + c;
    float bias[4];
    load_bias(p, col, bias);
    for (int r = tid / kQuads; r < rows; r += kAtOnce * step) {
        float z[kAtOnce * 4] = {};
        for (int s = 0; s < plan.cluster; ++s)
#pragma unroll
            for (int q = 0; q < kAtOnce; ++q) {
                const float4 f = *reinterpret_cast<const float4*>(parts + ((int64_t)s * rows + min(r + q * step, rows - 1)) * BN + c);
                z[q * 4] += f.x;
                z[q * 4 + 1] += f.y;
                z[q * 4 + 2] += f.z;
                z[q * 4 + 3] += f.w;
            }
        finish_quads<T, kAtOnce>(p, z, bias, row0 + r, step, end, col, vec);
    }
}

// Adds the parts of the cut tiles up in order and finishes them.  A thread takes four columns of a row.
template <typename T, int ROWS, int BN>
__global__ void __launch_bounds__(256) product_join_kernel(const __grid_constant__ ProductParams p, const __grid_constant__ Plan plan, bool vec) {
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, false);
    const int64_t m_end = p.live_k ? p.m : min(p.m, live);
    const int mt = (int)((m_end + ROWS - 1) / (ROWS)), tail = mt * plan.nt - plan.whole;
    constexpr int kPerTile = ROWS * BN / 4;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, t = at / kPerTile;
    if (t >= tail) return;
    const int in = (int)(at - t * kPerTile), r = in / (BN / 4), q = in - r * (BN / 4);
    int m, n;
    tile_at(mt, plan.nt, plan.whole + (int)t, m, n);
    const int64_t row = (int64_t)m * ROWS + r, col = (int64_t)n * BN + q * 4;
    if (row >= m_end || col >= p.n) return;
    if (p.a_sums && col == 0) {
        float sum = 0.0f;
        for (int s = 0; s < plan.splits; ++s) sum += plan.sum_parts[(t * plan.splits + s) * ROWS + r];
        p.a_sums[row] = sum;
    }
    float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const float4* from = reinterpret_cast<const float4*>(plan.parts + t * plan.splits * ROWS * BN) + in;
    for (int s = 0; s < plan.splits; ++s) {
        const float4 f = from[(int64_t)s * kPerTile];
        z[0] += f.x;
        z[1] += f.y;
        z[2] += f.z;
        z[3] += f.w;
    }
    T* out = static_cast<T*>(const_cast<void*>(p.out.data)) + row * p.out.stride + col;
    const T* res = p.residual.data ? static_cast<const T*>(p.residual.data) + row * p.residual.stride + col : nullptr;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (res && col + e < p.n) z[e] += load1(res + e);
    if (vec && col + 4 <= p.n) {
        store_quad(out, z);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (col + e < p.n) store1(out + e, z[e]);
    }
}

#endif  // __CUDACC__

}  // namespace aa
