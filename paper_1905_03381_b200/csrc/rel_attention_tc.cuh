// Building blocks of the attention kernels on the 5th-generation tensor cores (tcgen05): operand tiles in the 128-byte-swizzled layout,
// products between them into TMEM, and a thread's row of a score tile.
//
// A score tile is 128 query rows x 64 keys; thread r of a warpgroup holds row r (TMEM lane r), so that maxima and sums stay in the thread.
// Operand tiles are fetched by ordinary 16-byte asynchronous copies, which zero what lies behind a sequence's end: the next sequence's
// tokens must not reach a product, not even times zero.
#pragma once

#include "rel_attention_mma.cuh"
#include "tensor_core.cuh"

namespace aa {

#ifdef __CUDACC__

constexpr int kTcKeys = 64;              // keys of a tile
constexpr int kTcMargin = 96;            // distances of a warp's 32 x 64 part beyond one that touches the reach
constexpr int kTcTmem = 512;

// [ROWS x DT] bf16 tile: DT / 64 blocks of [ROWS x 128 bytes], 16-byte chunk c of row r at position c ^ (r & 7).
template <int ROWS, int DT, int THREADS>
__device__ __forceinline__ void load_swizzled(const RelParams& p, const TokArg& a, int head, int64_t row0, int n, uint32_t dst, int tid) {
    constexpr int CH = DT / 8, STEP = THREADS / CH;
    static_assert(ROWS % STEP == 0 && STEP % 8 == 0 || STEP < 8, "rows");
    const int c = tid % CH, r0 = tid / CH;
    const char* base = reinterpret_cast<const char*>(static_cast<const uint16_t*>(a.data) + row0 * a.tok + (int64_t)head * a.head + (c * 8 < p.dim ? c * 8 : 0));
    const uint32_t pitch = (uint32_t)a.tok * 2u, block = dst + (uint32_t)((c >> 3) * ROWS * 128);
    const int live = c * 8 < p.dim ? n : 0;
#pragma unroll 8
    for (int i = 0; i < ROWS / STEP; ++i) {
        const int r = r0 + i * STEP;
        cp_async16(block + (uint32_t)(r * 128 + (((c & 7) ^ (r & 7)) << 4)), base + (uint64_t)(uint32_t)max(0, min(r, n - 1)) * pitch, r < live);
    }
}

// D[128 x N] (+)= A . B^T, both K-major tiles of DT columns (A_ROWS and N rows).
template <int DT, int A_ROWS, int N>
__device__ __forceinline__ void mma_rows(const RelParams& p, uint32_t d, uint32_t a, uint32_t b) {
    constexpr uint32_t idesc = umma_idesc_bf16(128, N, false, false);
#pragma unroll
    for (int k = 0; k < DT / 16; ++k) {
        if (k * 16 >= p.dim) break;
        umma_bf16(d, umma_smem_desc(a + (k >> 2) * A_ROWS * 128 + (k & 3) * 32, 16, 1024), umma_smem_desc(b + (k >> 2) * N * 128 + (k & 3) * 32, 16, 1024), idesc, k > 0);
    }
}

// 32 fp32 columns of this thread's TMEM lane from registers.
__device__ __forceinline__ void tmem_st_32cols(uint32_t taddr, const uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
        "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
        "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// A thread's 64 products -> base-2 scores.  i: its query row (i >= Lq: all masked), w0: first row of its warp.
__device__ __forceinline__ void row_scores(const RelParams& p, const Seq& s, const float* bias, int w0, int i, int j0, float (&t)[64]) {
    const int shift = s.lk - s.lq, pos = i + shift;
    const int dmin = j0 - (w0 + 31 + shift), dmax = j0 + 63 - (w0 + shift);
    if (!p.table) {
#pragma unroll
        for (int c = 0; c < 64; ++c) t[c] *= p.scale2;
    } else if (dmax <= -p.reach || dmin >= p.reach) {
        const float far = bias[dmax <= -p.reach ? 0 : 2 * (p.reach + kTcMargin)];
#pragma unroll
        for (int c = 0; c < 64; ++c) t[c] = fmaf(t[c], p.scale2, far);
    } else {
        const float* at = bias + (j0 - pos + p.reach + kTcMargin);
#pragma unroll
        for (int c = 0; c < 64; ++c) t[c] = fmaf(t[c], p.scale2, at[c]);
    }
    if (j0 + 64 > s.lk || w0 + 32 > s.lq || (p.causal && dmax > 0)) {
        const int lim = i < s.lq ? min(s.lk, p.causal ? pos + 1 : s.lk) - j0 : 0;
#pragma unroll
        for (int c = 0; c < 64; ++c) t[c] = c >= lim ? -INFINITY : t[c];
    }
}

// drop(c, dropped) for the row's 64 elements.
template <typename F>
__device__ __forceinline__ void row_drops(const RelParams& p, const Seq& s, uint2 key, int h, int i, int j0, F drop) {
    const uint32_t top = p.drop.thr << 16;
    const uint64_t first = draw_row(s, h, i) + (uint64_t)((j0 >> 5) * 4);
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const Words4 w = draw_block(p.drop, key, first + (uint64_t)(4 * c + q));
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                drop(32 * c + 8 * x + 2 * q, (w.w[x] << 16) < top);
                drop(32 * c + 8 * x + 2 * q + 1, w.w[x] < top);
            }
        }
}

// The row's 64 values as bf16 into row r of a [128 x 128 bytes] swizzled block.
__device__ __forceinline__ void store_row(char* tile, int r, const float (&t)[64]) {
    char* row = tile + r * 128;
#pragma unroll
    for (int c = 0; c < 8; ++c)
        *reinterpret_cast<uint4*>(row + ((c ^ (r & 7)) << 4)) =
            make_uint4(pack_bf16(t[8 * c], t[8 * c + 1]), pack_bf16(t[8 * c + 2], t[8 * c + 3]), pack_bf16(t[8 * c + 4], t[8 * c + 5]), pack_bf16(t[8 * c + 6], t[8 * c + 7]));
}

__device__ __forceinline__ void load_row(uint32_t tmem, float (&t)[64]) {
    uint32_t a[32], b[32];
    tmem_ld_32cols(tmem, a);
    tmem_ld_32cols(tmem + 32, b);
    tmem_ld_wait();
#pragma unroll
    for (int c = 0; c < 32; ++c) {
        t[c] = __uint_as_float(a[c]);
        t[32 + c] = __uint_as_float(b[c]);
    }
}

// COLS accumulator columns of this thread's lane times f, as bf16, to `out` from element `from` on (nullptr: read only, the instruction is the warp's).
template <int COLS>
__device__ __forceinline__ void store_accumulator(const RelParams& p, uint32_t tmem, uint16_t* out, float f, int from = 0) {
#pragma unroll
    for (int c0 = 0; c0 < COLS; c0 += 32) {
        uint32_t v[32];
        tmem_ld_32cols(tmem + (uint32_t)c0, v);
        tmem_ld_wait();
        if (out) {
#pragma unroll
            for (int c = 0; c < 32; c += 8) {
                if (from + c0 + c >= p.dim) continue;
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = pack_bf16(__uint_as_float(v[c + 2 * k]) * f, __uint_as_float(v[c + 2 * k + 1]) * f);
                *reinterpret_cast<uint4*>(out + from + c0 + c) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
        __syncwarp();                      // the next load is the whole warp's
    }
}

#endif  // __CUDACC__

}  // namespace aa
