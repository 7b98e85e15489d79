// Building blocks of the bf16 attention kernels on the warp-level matrix instructions (mma.sync m16n8k16, fp32 accumulation): operand
// tiles in shared memory, fragments, the score block of a warp and the diagonal sums of the bias gradient.
//
// Why warp-level instructions: a score element costs 4 D flops forward but also a bias look-up, an exponential and, in training, a
// share of a Philox block, and the sentences of a batch are 8..128 tokens long, so tiles adapt to a sentence in steps of 16 rows and 16
// keys and the probabilities go from accumulator to operand without leaving the registers.
#pragma once

#include "async_copy.cuh"
#include "rel_attention.cuh"

namespace aa {

#ifdef __CUDACC__

// Row pitch of an operand tile in elements: one 16-byte chunk more than the row, an odd number of chunks for widths 32, 64, 128, so
// the eight rows of an ldmatrix phase fall on distinct banks.
__host__ __device__ constexpr int pitch_of(int width) { return width + 8; }

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool live) {
    const int n = live ? 16 : 0;         // 0: the destination is filled with zeros, src is not read
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Tokens [row0, row0 + ROWS) of one head into a tile of DT columns; rows from n up to the next multiple of ROUND and columns from p.dim on are
// zero, rows behind that are left as they are (nothing may read them: not even a masked score's product, which would pass a NaN on).  A
// thread keeps its column and walks down the rows: an address is one 32 x 32 + 64 bit multiply-add (strides are below 2^30 elements).
template <int ROWS, int DT, int THREADS, int ROUND = ROWS>
__device__ __forceinline__ void load_tile_async(const RelParams& p, const TokArg& a, int head, int64_t row0, int n, uint16_t* dst) {
    constexpr int CH = DT / 8, STEP = THREADS / CH;
    static_assert(STEP <= ROWS && ROWS % STEP == 0, "a pass of the threads covers whole rows");
    const int c = threadIdx.x % CH, r0 = threadIdx.x / CH;
    const char* base = reinterpret_cast<const char*>(static_cast<const uint16_t*>(a.data) + row0 * a.tok + (int64_t)head * a.head + (c * 8 < p.dim ? c * 8 : 0));
    const uint32_t d = smem_u32(dst) + (uint32_t)(r0 * pitch_of(DT) + c * 8) * 2u, pitch = (uint32_t)a.tok * 2u;
    const int live = c * 8 < p.dim ? n : 0, rows = ROUND == ROWS ? ROWS : (n + ROUND - 1) / ROUND * ROUND;
#pragma unroll
    for (int i = 0; i < ROWS / STEP; ++i) {
        const int r = r0 + i * STEP;
        if (ROUND == ROWS || r < rows) cp_async16(d + (uint32_t)(i * STEP * pitch_of(DT)) * 2u, base + (uint64_t)(uint32_t)max(0, min(r, n - 1)) * pitch, r < live);
    }
}

// Addresses of this lane's row for the four 8 x 8 matrices of an ldmatrix.x4.
// A operand 16 x 16 (rows r0.., contraction from k): plain; also the transposed B operand (contraction rows r0.., columns from k).
template <int PITCH>
__device__ __forceinline__ uint32_t frag_rows(uint32_t tile, int r0, int k, int lane) {
    return tile + (uint32_t)((r0 + (lane & 15)) * PITCH + k + ((lane >> 4) << 3)) * 2u;
}
// B operand of two 8-column tiles (columns = tile rows n0..n0+15, contraction from k): plain.  Registers 0,1: first tile; 2,3: second.
template <int PITCH>
__device__ __forceinline__ uint32_t frag_cols(uint32_t tile, int n0, int k, int lane) {
    return tile + (uint32_t)((n0 + (lane & 7) + ((lane >> 4) << 3)) * PITCH + k + (((lane >> 3) & 1) << 3)) * 2u;
}
// A operand 16 x 16 that is the transpose of what the tile holds (contraction rows k.., operand rows = tile columns from m): transposed.
template <int PITCH>
__device__ __forceinline__ uint32_t frag_trans(uint32_t tile, int k, int m, int lane) {
    return tile + (uint32_t)((k + (lane & 7) + ((lane >> 4) << 3)) * PITCH + m + (((lane >> 3) & 1) << 3)) * 2u;
}

// A score block is 16 rows x 8 NT keys, NT = 4 or 8, fully unrolled and without a test per group of keys: groups that see nothing are masked
// like any other key (a test each made the block's code twice as long in instructions executed).
// acc = A (16 x DT from registers) . tile rows [n0, n0 + 8 NT)^T
template <int DT, int NT>
__device__ __forceinline__ void block_dot(const RelParams& p, const uint32_t (&a)[DT / 16][4], uint32_t tile, int n0, int lane, float (&acc)[NT][4]) {
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][e] = 0.0f;
    const uint32_t at = frag_cols<pitch_of(DT)>(tile, n0, 0, lane);
#pragma unroll
    for (int k = 0; k < DT / 16; ++k) {
        if (DT > 64 && k * 16 >= p.dim) continue;
#pragma unroll
        for (int g = 0; g < NT / 2; ++g) {
            uint32_t b[4];
            ldsm4(b, at + (uint32_t)(g * 16 * pitch_of(DT) + k * 16) * 2u);
            mma16816(acc[2 * g], a[k], b[0], b[1]);
            mma16816(acc[2 * g + 1], a[k], b[2], b[3]);
        }
    }
}

template <int DT>
__device__ __forceinline__ void load_frags(const RelParams& p, uint32_t (&a)[DT / 16][4], uint32_t tile, int r0, int lane) {
#pragma unroll
    for (int k = 0; k < DT / 16; ++k) {
        if (DT > 64 && k * 16 >= p.dim) continue;
        ldsm4(a[k], frag_rows<pitch_of(DT)>(tile, r0, k * 16, lane));
    }
}

// Where a block lies: lane (g, t) holds query rows i0 + g, i0 + g + 8 and keys j0 + 8 nt + 2 t + {0, 1}.
struct Block {
    int i0, j0;
};

// A block that touches the reach of the bias holds distances up to 78 beyond it.
constexpr int kBiasMargin = 80;

// Products -> base-2 scores with bias and masks.
template <int NT>
__device__ __forceinline__ void block_scores(const RelParams& p, const Seq& s, const float* bias, const Block& b, int lane, float (&acc)[NT][4]) {
    const int shift = s.lk - s.lq, g = lane >> 2, t = lane & 3;
    const int dmin = b.j0 - (b.i0 + 15 + shift), dmax = b.j0 + 8 * NT - 1 - (b.i0 + shift);
    const bool whole = b.j0 + 8 * NT <= s.lk && b.i0 + 16 <= s.lq && (!p.causal || dmax <= 0);
    if (!p.table) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[n][e] *= p.scale2;
    } else if (dmax <= -p.reach || dmin >= p.reach) {      // one bucket for the whole block
        const float far = bias[dmax <= -p.reach ? 0 : 2 * (p.reach + kBiasMargin)];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[n][e] = fmaf(acc[n][e], p.scale2, far);
    } else {
        const float* at = bias + (b.j0 + 2 * t - (b.i0 + g + shift) + p.reach + kBiasMargin);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[n][e] = fmaf(acc[n][e], p.scale2, at[8 * n + (e & 1) - 8 * (e >> 1)]);
    }
    if (!whole) {
        int lim[2];                                        // keys of this lane's columns that row r sees: those below lim[r]
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int i = b.i0 + g + 8 * r;
            lim[r] = i < s.lq ? min(s.lk, p.causal ? i + shift + 1 : s.lk) - (b.j0 + 2 * t) : -0x40000000;
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[n][e] = 8 * n + (e & 1) >= lim[e >> 1] ? -INFINITY : acc[n][e];
    }
}

// Calls drop(n, e, dropped) for every element of the block.  Four draw blocks per lane: two rows, two chunks of 32 keys.  Draw x of a
// block is key tile 4 c + x / 2, element x % 2 of its row; the high half of a word compares in place, the low half shifted up.
template <int NT, typename F>
__device__ __forceinline__ void block_drops(const RelParams& p, const Seq& s, uint2 key, int h, const Block& b, int lane, F drop) {
    const uint32_t top = p.drop.thr << 16;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const uint64_t first = draw_row(s, h, b.i0 + (lane >> 2) + 8 * r) + (uint64_t)((b.j0 >> 5) * 4 + (lane & 3));
#pragma unroll
        for (int c = 0; c < NT / 4; ++c) {
            const Words4 w = draw_block(p.drop, key, first + 4 * c);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                drop(4 * c + x, 2 * r, (w.w[x] << 16) < top);
                drop(4 * c + x, 2 * r + 1, w.w[x] < top);
            }
        }
    }
}

__device__ __forceinline__ float quad_max(float x) {
    x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 1));
    return fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 2));
}
__device__ __forceinline__ float quad_sum(float x) {
    x += __shfl_xor_sync(0xFFFFFFFFu, x, 1);
    return x + __shfl_xor_sync(0xFFFFFFFFu, x, 2);
}

// ---- softmax and gradient steps of a block

// Running maximum and sum of rows g and g + 8, t -> 2^(t - m), earlier output rescaled.
template <int DT, int NT>
__device__ __forceinline__ void block_softmax(float (&t)[NT][4], float (&m)[2], float (&l)[2], float (&o)[DT / 8][4]) {
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        float top = m[r];
#pragma unroll
        for (int n = 0; n < NT; ++n) top = fmaxf(top, fmaxf(t[n][2 * r], t[n][2 * r + 1]));
        top = quad_max(top);
        const float ref = top == -INFINITY ? 0.0f : top, corr = ex2_approx(m[r] - ref);
        float sum = 0.0f;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const float e = ex2_approx(t[n][2 * r + c] - ref);
                sum += e;
                t[n][2 * r + c] = e;
            }
        l[r] = fmaf(l[r], corr, sum);                      // this lane's part of the row
        m[r] = top;
#pragma unroll
        for (int j = 0; j < DT / 8; ++j) {
            o[j][2 * r] *= corr;
            o[j][2 * r + 1] *= corr;
        }
    }
}
// o += x . tile rows [n0, n0 + 8 NT).  x (probabilities of at most 1, or score gradients) is rounded to bf16 as the left operand: 2^-9 of each
// term of a result that is bf16 itself.
template <int DT, int NT>
__device__ __forceinline__ void block_times(const RelParams& p, const float (&x)[NT][4], uint32_t tile, int n0, int lane, float (&o)[DT / 8][4]) {
    const uint32_t at = frag_rows<pitch_of(DT)>(tile, n0, 0, lane);
#pragma unroll
    for (int k = 0; k < NT / 2; ++k) {
        const uint32_t a[4] = {pack_bf16(x[2 * k][0], x[2 * k][1]), pack_bf16(x[2 * k][2], x[2 * k][3]), pack_bf16(x[2 * k + 1][0], x[2 * k + 1][1]),
                               pack_bf16(x[2 * k + 1][2], x[2 * k + 1][3])};
#pragma unroll
        for (int j = 0; j < DT / 16; ++j) {
            if (DT > 64 && j * 16 >= p.dim) continue;
            uint32_t v[4];
            ldsm4t(v, at + (uint32_t)(k * 16 * pitch_of(DT) + j * 16) * 2u);
            mma16816(o[2 * j], a, v[0], v[1]);
            mma16816(o[2 * j + 1], a, v[2], v[3]);
        }
    }
}

// Row statistics of lane (g, t)'s rows g and g + 8.
struct RowStats {
    float m[2], rl[2], D[2];
};
// this lane's maximum of row r
template <int NT>
__device__ __forceinline__ float block_max(const float (&t)[NT][4], int r, float top) {
#pragma unroll
    for (int n = 0; n < NT; ++n) top = fmaxf(top, fmaxf(t[n][2 * r], t[n][2 * r + 1]));
    return top;
}
// t -> e = 2^(t - ref); adds this lane's sums
template <int NT>
__device__ __forceinline__ void block_exp(const float (&ref)[2], float (&t)[NT][4], float (&sum)[2]) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            t[n][e] = ex2_approx(t[n][e] - ref[e >> 1]);
            sum[e >> 1] += t[n][e];
        }
}
// dp of dropped probabilities is 0, of kept ones scaled; the sign of e (which is not negative) remembers which were dropped.
template <int NT>
__device__ __forceinline__ void block_drop(const RelParams& p, const Seq& s, uint2 key, int h, const Block& b, int lane, float (&t)[NT][4], float (&dp)[NT][4]) {
    if (!p.drop.thr) return;
    block_drops<NT>(p, s, key, h, b, lane, [&](int n, int e, bool d) {
        dp[n][e] = d ? 0.0f : __fmul_rn(dp[n][e], p.drop.scale);
        t[n][e] = d ? -t[n][e] : t[n][e];
    });
}
// this lane's sums of e dp
template <int NT>
__device__ __forceinline__ void block_dsum(const float (&t)[NT][4], const float (&dp)[NT][4], float (&dsum)[2]) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) dsum[e >> 1] = fmaf(fabsf(t[n][e]), dp[n][e], dsum[e >> 1]);
}
// e (signed) -> p, dropped and scaled, in t;  dp -> ds = p (dp - D).  rl includes whatever turns e into p.
template <int NT>
__device__ __forceinline__ void block_ds(const RelParams& p, const RowStats& st, float (&t)[NT][4], float (&dp)[NT][4]) {
    const float f[2] = {st.rl[0] * p.drop.scale, st.rl[1] * p.drop.scale};
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = e >> 1;
            dp[n][e] = fabsf(t[n][e]) * st.rl[r] * (dp[n][e] - st.D[r]);
            t[n][e] = fmaxf(t[n][e], 0.0f) * f[r];
        }
}
// t and dp (p and ds by now) as bf16 into rows g and g + 8 of two tiles, at this lane's columns
template <int NT>
__device__ __forceinline__ void store_scores(uint16_t* prow, uint16_t* srow, int pitch, const float (&t)[NT][4], const float (&dp)[NT][4]) {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        *reinterpret_cast<uint32_t*>(prow + 8 * n) = pack_bf16(t[n][0], t[n][1]);
        *reinterpret_cast<uint32_t*>(prow + 8 * pitch + 8 * n) = pack_bf16(t[n][2], t[n][3]);
        *reinterpret_cast<uint32_t*>(srow + 8 * n) = pack_bf16(dp[n][0], dp[n][1]);
        *reinterpret_cast<uint32_t*>(srow + 8 * pitch + 8 * n) = pack_bf16(dp[n][2], dp[n][3]);
    }
}

// ---- diagonal sums.  A lane's elements of one 16 x 64 block are first added along the diagonal inside the lane (row g + 8 of key tile
// nt + 1 lies on the diagonal of row g of key tile nt); the 8 x 72 values left are stored skewed, row g shifted by 7 - g, so that a column
// of the staging area is a diagonal: column key - row + 15 (rows and keys relative to the block), columns 0..78.
constexpr int kDiagPitch = 89;           // two lanes per bank on the skewed store
constexpr int kDiagFloats = 8 * kDiagPitch;
constexpr int kDiagCols = 79;

__device__ __forceinline__ void stage_diagonals(float* stage, const float (&ds)[8][4], int lane) {
    const int g = lane >> 2, t = lane & 3;
    float* at = stage + g * kDiagPitch + 2 * t + 7 - g;
#pragma unroll
    for (int u = -1; u < 8; ++u)
#pragma unroll
        for (int c = 0; c < 2; ++c) at[8 * (u + 1) + c] = (u >= 0 ? ds[u < 0 ? 0 : u][c] : 0.0f) + (u < 7 ? ds[u < 7 ? u + 1 : 7][2 + c] : 0.0f);
}
// Row r holds columns 7 - r .. 78 - r.
__device__ __forceinline__ float diagonal_sum(const float* stage, int col) {
    float sum = 0.0f;
#pragma unroll
    for (int r = 0; r < 8; ++r) {
        const float x = stage[r * kDiagPitch + col];
        sum += col + r >= 7 && col + r < 79 ? x : 0.0f;
    }
    return sum;
}

// The same 18 values of a lane, added up over blocks that lie at the same distances: acc[u + 1][lane] of 9 x 32 pairs, this lane's own.
constexpr int kDiagAccFloats = 9 * 64;
template <int NT>
__device__ __forceinline__ void add_diagonals(float* acc, const float (&ds)[NT][4], int lane) {
    float2* mine = reinterpret_cast<float2*>(acc) + lane;
#pragma unroll
    for (int u = -1; u < NT; ++u) {
        float2 x = mine[(u + 1) * 32];
        x.x += (u >= 0 ? ds[u < 0 ? 0 : u][0] : 0.0f) + (u < NT - 1 ? ds[u < NT - 1 ? u + 1 : NT - 1][2] : 0.0f);
        x.y += (u >= 0 ? ds[u < 0 ? 0 : u][1] : 0.0f) + (u < NT - 1 ? ds[u < NT - 1 ? u + 1 : NT - 1][3] : 0.0f);
        mine[(u + 1) * 32] = x;
    }
}
__device__ __forceinline__ void stage_accumulated(float* stage, float* acc, int lane) {
    const int g = lane >> 2, t = lane & 3;
    float* at = stage + g * kDiagPitch + 2 * t + 7 - g;
    float2* mine = reinterpret_cast<float2*>(acc) + lane;
#pragma unroll
    for (int u = 0; u < 9; ++u) {
        const float2 x = mine[u * 32];
        mine[u * 32] = make_float2(0.0f, 0.0f);
        at[8 * u] = x.x;
        at[8 * u + 1] = x.y;
    }
}

// acc rows (g, g + 8 of a 16-row block) times f, as bf16, into DT columns from c0 on; rows from n on are not written.
template <int DT>
__device__ __forceinline__ void store_block(const RelParams& p, const TokArg& a, int head, int64_t row0, int n, int lane, const float (&acc)[DT / 8][4], float f0, float f1,
                                            int c0 = 0) {
    const int g = lane >> 2, t = lane & 3;
    uint16_t* base = const_cast<uint16_t*>(static_cast<const uint16_t*>(a.data)) + row0 * a.tok + (int64_t)head * a.head + c0 + 2 * t;
#pragma unroll
    for (int j = 0; j < DT / 8; ++j) {
        if (c0 + j * 8 >= p.dim) continue;
        if (g < n) *reinterpret_cast<uint32_t*>(base + (int64_t)g * a.tok + j * 8) = pack_bf16(acc[j][0] * f0, acc[j][1] * f0);
        if (g + 8 < n) *reinterpret_cast<uint32_t*>(base + (int64_t)(g + 8) * a.tok + j * 8) = pack_bf16(acc[j][2] * f1, acc[j][3] * f1);
    }
}

#endif  // __CUDACC__

}  // namespace aa
