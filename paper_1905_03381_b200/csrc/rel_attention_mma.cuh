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

// Tokens [row0, row0 + ROWS) of one head into a tile of DT columns; rows from n on and columns from p.dim on are zero.
template <int ROWS, int DT, int THREADS>
__device__ __forceinline__ void load_tile_async(const RelParams& p, const TokArg& a, int head, int64_t row0, int n, uint16_t* dst) {
    constexpr int CH = DT / 8;
    const uint16_t* base = static_cast<const uint16_t*>(a.data) + row0 * a.tok + (int64_t)head * a.head;
    const uint32_t d = smem_u32(dst);
#pragma unroll
    for (int i = 0; i < (ROWS * CH + THREADS - 1) / THREADS; ++i) {
        const int at = i * THREADS + (int)threadIdx.x;
        if ((ROWS * CH) % THREADS == 0 || at < ROWS * CH) {
            const int r = at / CH, c = at % CH;
            const bool live = r < n && c * 8 < p.dim;
            cp_async16(d + (uint32_t)(r * pitch_of(DT) + c * 8) * 2u, live ? base + (int64_t)r * a.tok + c * 8 : base, live);
        }
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

// acc (16 rows x 64 columns) = A (16 x DT from registers) . tile rows^T, for the first n16 groups of 16 columns.
template <int DT>
__device__ __forceinline__ void block_dot(const RelParams& p, const uint32_t (&a)[DT / 16][4], uint32_t tile, int n0, int n16, int lane, float (&acc)[8][4]) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][e] = 0.0f;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        if (g >= n16) continue;
#pragma unroll
        for (int k = 0; k < DT / 16; ++k) {
            if (DT > 64 && k * 16 >= p.dim) continue;
            uint32_t b[4];
            ldsm4(b, frag_cols<pitch_of(DT)>(tile, n0 + g * 16, k * 16, lane));
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

// Where a warp's 16 x 64 score block lies: query rows i0 + g, i0 + g + 8 and keys j0 + 8 nt + 2 t + {0, 1} of lane (g, t).
struct Block {
    int i0, j0;
};

// Products -> base-2 scores with bias and masks.
__device__ __forceinline__ void block_scores(const RelParams& p, const Seq& s, const float* bias, const Block& b, int lane, float (&acc)[8][4]) {
    const int shift = s.lk - s.lq, g = lane >> 2, t = lane & 3;
    const int dmin = b.j0 - (b.i0 + 15 + shift), dmax = b.j0 + 63 - (b.i0 + shift);
    const bool whole = b.j0 + 64 <= s.lk && b.i0 + 16 <= s.lq && (!p.causal || dmax <= 0);
    if (!p.table) {
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[n][e] *= p.scale2;
    } else if (dmax <= -p.reach || dmin >= p.reach) {      // one bucket for the whole block
        const float far = bias[dmax <= -p.reach ? 0 : 2 * p.reach];
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[n][e] = fmaf(acc[n][e], p.scale2, far);
    } else {
        const int d0 = b.j0 + 2 * t - (b.i0 + g + shift) + p.reach, top = 2 * p.reach;
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int at = d0 + 8 * n + (e & 1) - 8 * (e >> 1);
                acc[n][e] = fmaf(acc[n][e], p.scale2, bias[min(max(at, 0), top)]);
            }
    }
    if (!whole) {
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = b.i0 + g + 8 * (e >> 1), j = b.j0 + 8 * n + 2 * t + (e & 1);
                if (i >= s.lq || j >= s.lk || (p.causal && j > i + shift)) acc[n][e] = -INFINITY;
            }
    }
}

// Bits of dropped elements: bit 4 nt + e of the answer.  Four draw blocks per lane: two rows, two chunks of 32 keys.
__device__ __forceinline__ uint32_t block_drops(const RelParams& p, const Seq& s, uint2 key, int h, const Block& b, int lane) {
    uint32_t bits = 0;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const uint64_t first = draw_row(s, h, b.i0 + (lane >> 2) + 8 * r) + (uint64_t)((b.j0 >> 5) * 4 + (lane & 3));
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const Words4 w = draw_block(p.drop, key, first + 4 * c);
#pragma unroll
            for (int x = 0; x < 8; ++x)                     // draw x: key tile 4 c + x / 2, element x % 2 of row r
                if (draw_half(w, x) < p.drop.thr) bits |= 1u << (4 * (4 * c + (x >> 1)) + 2 * r + (x & 1));
        }
    }
    return bits;
}

// 16-key groups of the block that hold an unmasked pair.
__device__ __forceinline__ int block_groups(const RelParams& p, const Seq& s, const Block& b) {
    if (b.i0 >= s.lq) return 0;
    int end = s.lk;
    if (p.causal) end = min(end, min(b.i0 + 16, s.lq) + s.lk - s.lq);
    return min(4, max(0, (end - b.j0 + 15) >> 4));
}

__device__ __forceinline__ float quad_max(float x) {
    x = fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 1));
    return fmaxf(x, __shfl_xor_sync(0xFFFFFFFFu, x, 2));
}
__device__ __forceinline__ float quad_sum(float x) {
    x += __shfl_xor_sync(0xFFFFFFFFu, x, 1);
    return x + __shfl_xor_sync(0xFFFFFFFFu, x, 2);
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
__device__ __forceinline__ float diagonal_sum(const float* stage, int col) {
    float sum = 0.0f;
#pragma unroll
    for (int r = 0; r < 8; ++r) sum += stage[r * kDiagPitch + col];
    return sum;
}

// acc rows (g, g + 8 of a 16-row block) times f, as bf16; rows from n on are not written.
template <int DT>
__device__ __forceinline__ void store_block(const RelParams& p, const TokArg& a, int head, int64_t row0, int n, int lane, const float (&acc)[DT / 8][4], float f0, float f1) {
    const int g = lane >> 2, t = lane & 3;
    uint16_t* base = const_cast<uint16_t*>(static_cast<const uint16_t*>(a.data)) + row0 * a.tok + (int64_t)head * a.head + 2 * t;
#pragma unroll
    for (int j = 0; j < DT / 8; ++j) {
        if (j * 8 >= p.dim) continue;
        if (g < n) *reinterpret_cast<uint32_t*>(base + (int64_t)g * a.tok + j * 8) = pack_bf16(acc[j][0] * f0, acc[j][1] * f0);
        if (g + 8 < n) *reinterpret_cast<uint32_t*>(base + (int64_t)(g + 8) * a.tok + j * 8) = pack_bf16(acc[j][2] * f1, acc[j][3] * f1);
    }
}

#endif  // __CUDACC__

}  // namespace aa
