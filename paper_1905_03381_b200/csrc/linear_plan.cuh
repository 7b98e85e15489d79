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

// Splits of the tiles that do not fill a round of `teams`: the fewest slices one after the other, counting the parts' way through memory.
// slice_us: what a slice of a tile takes.
inline Plan make_plan(const ProductParams& p, int64_t tiles, int nt, int teams, int64_t tile_floats, int tile_rows, double slice_us, bool may_cluster) {
    Plan plan{nt, (int)tiles, 1, p.parts, nullptr, 1};
    const int64_t slices = (p.k + kSlice - 1) / kSlice, whole = tiles / teams * teams, tail = tiles - whole;
    if (!p.parts) {
        // few tiles and no scratch memory: as many CTAs on each as the SMs give, with four slices or more apiece
        int c = 8;
        while (c > 1 && (tiles * c > teams || slices < 4 * c)) c /= 2;
        if (may_cluster && c > 1) plan.whole = 0, plan.splits = plan.cluster = c;
        return plan;
    }
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
        u.s0 = (int)((int64_t)slices * q / p.splits);
        u.s1 = (int)((int64_t)slices * (q + 1) / p.splits);
        u.part = j;
    }
    return u;
}

// Bias, pre, activation, residual and the rounding of four neighbouring columns (cols of them count; vec: pointers allow vectors).
template <typename T>
__device__ __forceinline__ void finish_quad(const ProductParams& p, float (&z)[4], int64_t row, int64_t col, int cols, bool vec) {
    T* out = static_cast<T*>(const_cast<void*>(p.out.data)) + row * p.out.stride + col;
    T* pre = p.pre.data ? static_cast<T*>(const_cast<void*>(p.pre.data)) + row * p.pre.stride + col : nullptr;
    const T* res = p.residual.data ? static_cast<const T*>(p.residual.data) + row * p.residual.stride + col : nullptr;
    if (p.bias) {
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] += e < cols ? p.bias[col + e] : 0.0f;
    }
    if (vec && cols == 4) {
        if (pre) store_quad(pre, z);
        activate_all(z, p.act);
        if (res) {
            float y[4];
            load_quad(res, y);
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] += y[e];
        }
        store_quad(out, z);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (pre && e < cols) store1(pre + e, z[e]);
        activate_all(z, p.act);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < cols) store1(out + e, res ? z[e] + load1(res + e) : z[e]);
    }
}

// The CTAs of a cluster have the parts of a tile of 128 rows in [CTA][128 / cluster rows][BN] of everybody's `parts` (shared memory): this CTA finishes its rows.
// `threads` threads from `tid` on; after a cluster barrier.
template <typename T, int BN>
__device__ __forceinline__ void finish_cluster(const ProductParams& p, const Plan& plan, const Unit& u, const float* parts, int64_t m_end, bool vec, int tid, int threads) {
    const int rows = 128 / plan.cluster, rank = (int)cluster_rank();
    for (int i = tid; i < rows * (BN / 4); i += threads) {
        const int r = i / (BN / 4), c = (i - r * (BN / 4)) * 4;
        const int64_t row = (int64_t)u.m * 128 + rank * rows + r, col = (int64_t)u.n * BN + c;
        if (row >= m_end || col >= p.n) continue;
        float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int s = 0; s < plan.cluster; ++s) {
            const float4 f = *reinterpret_cast<const float4*>(parts + ((int64_t)s * rows + r) * BN + c);
            z[0] += f.x;
            z[1] += f.y;
            z[2] += f.z;
            z[3] += f.w;
        }
        finish_quad<T>(p, z, row, col, (int)min((int64_t)4, p.n - col), vec);
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
