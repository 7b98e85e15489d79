// Tiles of the tensor-core products: in which order a launch takes them, and which it cuts along the contraction so that the last round of SMs is full.
#pragma once

#include "linear.cuh"

namespace aa {

constexpr int kSlice = 64, kGroupM = 16;

// What a launch does in which order: the first `whole` tiles at once, the others in `splits` parts each.
struct Plan {
    int nt, whole, splits;
    float* parts;                        // [part][rows of a tile][columns of a tile]
    float* sum_parts;                    // [part][rows of a tile]
};

// Splits of the tiles that do not fill a round of `teams`: the fewest slices one after the other, counting the parts' way through memory.
// slice_us: what a slice of a tile takes.
inline Plan make_plan(const ProductParams& p, int64_t tiles, int nt, int teams, int64_t tile_floats, int tile_rows, double slice_us) {
    Plan plan{nt, (int)tiles, 1, p.parts, nullptr};
    const int64_t slices = (p.k + kSlice - 1) / kSlice, whole = tiles / teams * teams, tail = tiles - whole;
    if (!p.parts || tail == 0) return plan;
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
