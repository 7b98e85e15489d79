// Linear layers on up to 16 rows: single new tokens and short prompts.
//
// Bound by the weights' way from memory: 2 bytes for at most 32 flops.  A warp takes 16 outputs as the M side of warp-level matrix instructions (m16n8k16) and 8 or
// 16 rows of x as their N side; nothing is staged.  The order of the terms of a sum is free, so a lane fetches 8 neighbouring weights of two outputs
// (16 or 32 bytes) and the 8 values of x that belong to them, and they are taken for the terms that the instruction's layout gives the
// lane.  Where the outputs alone do not fill the GPU, the warps of a CTA share a sum's range and join in shared memory.
// fp32 numbers go in as three bf16 terms (see linear_split.cu), which costs six instructions a weight whatever the rows; sums of 64 terms
// (bf16: 128) leave the matrix unit's accumulator for ordinary additions.
// 1 x 512 -> 32,000 bf16 (33 MB of weights, 5.0 us at the copy rate) takes 8.3 us behind other launches and 11 alone, both from a cold L2 (14 by 128-row tiles on the tensor cores); 16 x 512 -> 32,000 fp32
// 24 and 54, 16 x 8,192 -> 1,024 fp32 30 and 53.
#include <type_traits>

#include "linear_plan.cuh"

namespace aa {

namespace {

constexpr int kFewRows = 16, kFewWarps = 8;

__device__ __forceinline__ void mma_few(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Eight neighbouring elements as they lie in memory, zeros where `n` says that fewer count.
template <typename T, bool VEC>
struct Eight {
    static constexpr int N = VEC ? (int)sizeof(T) / 2 : 8;
    using Word = typename std::conditional<VEC, uint4, T>::type;
    Word w[N];
    __device__ __forceinline__ void load(const T* at, int n) {
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = n > 0 ? reinterpret_cast<const uint4*>(at)[i] : make_uint4(0, 0, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = i < n ? at[i] : T(0);
        }
    }
    // Packed pairs, in TERMS bf16 terms.
    template <int TERMS>
    __device__ __forceinline__ void pairs(uint32_t (&t)[TERMS][4]) const {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (sizeof(T) == 2 && VEC) {
                t[0][q] = (&w[0].x)[q];
            } else if constexpr (sizeof(T) == 2) {
                t[0][q] = (uint32_t)w[2 * q] | (uint32_t)w[2 * q + 1] << 16;
            } else {
                float a, b;
                if constexpr (VEC) a = __uint_as_float((&w[q / 2].x)[q % 2 * 2]), b = __uint_as_float((&w[q / 2].x)[q % 2 * 2 + 1]);
                else a = w[2 * q], b = w[2 * q + 1];
                t[0][q] = pack_bf16(a, b);
                a -= bf16_lo(t[0][q]);
                b -= bf16_hi(t[0][q]);
                t[1][q] = pack_bf16(a, b);
                a -= bf16_lo(t[1][q]);
                b -= bf16_hi(t[1][q]);
                t[2][q] = pack_bf16(a, b);
            }
        }
    }
};

// NT groups of 8 rows of x; `share` warps of a CTA have the same outputs.
template <typename T, bool VEC, int NT>
__global__ void __launch_bounds__(kFewWarps * 32, NT == 1 || sizeof(T) == 2 ? 2 : 1) linear_few_kernel(const __grid_constant__ ProductParams p, int share, bool out_vec) {
    constexpr int TERMS = sizeof(T) == 4 ? 3 : 1, DEPTH = TERMS == 3 ? 2 : 4;      // blocks of 32 terms that are under way
    __shared__ float tile[kFewWarps][NT * 8][16 + 4];
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, blockIdx.x == 0 && threadIdx.x == 0), m_end = min(p.m, live);
    if (m_end == 0) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int groups = kFewWarps / share;                       // of 16 outputs in this CTA
    const int64_t n0 = ((int64_t)blockIdx.x * groups + warp / share) * 16;
    const int64_t blocks = (p.k + 31) / 32, part = warp % share;
    const int64_t b0 = blocks * part / share, b1 = blocks * (part + 1) / share;
    // rows that do not exist are stood in for by the last one; their results are not used
    const T* w[2];
    const T* x[NT];
#pragma unroll
    for (int i = 0; i < 2; ++i) w[i] = static_cast<const T*>(p.b.data) + min(n0 + g + 8 * i, p.n - 1) * p.b.stride + 8 * t;
#pragma unroll
    for (int i = 0; i < NT; ++i) x[i] = static_cast<const T*>(p.a.data) + min((int64_t)(g + 8 * i), m_end - 1) * p.a.stride + 8 * t;
    float sum[NT][4] = {};
    Eight<T, VEC> wa[DEPTH][2], xa[DEPTH][NT];
    const auto fetch = [&](int64_t b, int d) {
        const int64_t k = b * 32;
        const int n = b < b1 ? (int)max((int64_t)0, min((int64_t)8, p.k - k - 8 * t)) : 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) wa[d][i].load(w[i] + k, n);
#pragma unroll
        for (int i = 0; i < NT; ++i) xa[d][i].load(x[i] + k, n);
    };
    for (int64_t b = b0; b < b1; b += DEPTH) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) fetch(b + d, d);
        float big[NT][4] = {}, rest[NT][4] = {};
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            uint32_t u[2][TERMS][4];
#pragma unroll
            for (int i = 0; i < 2; ++i) wa[d][i].template pairs<TERMS>(u[i]);
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                uint32_t v[TERMS][4];
                xa[d][i].template pairs<TERMS>(v);
#pragma unroll
                for (int h = 0; h < 2; ++h) {                   // terms 2 h, 2 h + 1 of the lane's four pairs
                    const auto a = [&](int s, uint32_t (&f)[4]) { f[0] = u[0][s][2 * h], f[1] = u[1][s][2 * h], f[2] = u[0][s][2 * h + 1], f[3] = u[1][s][2 * h + 1]; };
                    uint32_t f[4];
                    a(0, f);
                    mma_few(big[i], f, v[0][2 * h], v[0][2 * h + 1]);
                    if constexpr (TERMS == 3) {
                        mma_few(rest[i], f, v[2][2 * h], v[2][2 * h + 1]);
                        mma_few(rest[i], f, v[1][2 * h], v[1][2 * h + 1]);
                        a(1, f);
                        mma_few(rest[i], f, v[1][2 * h], v[1][2 * h + 1]);
                        mma_few(rest[i], f, v[0][2 * h], v[0][2 * h + 1]);
                        a(2, f);
                        mma_few(rest[i], f, v[0][2 * h], v[0][2 * h + 1]);
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[i][e] += big[i][e] + rest[i][e];
    }
    // lane: outputs g and g + 8 of the group against rows 2 t and 2 t + 1
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) tile[warp][8 * i + 2 * t + (e & 1)][g + 8 * (e >> 1)] = sum[i][e];
    __syncthreads();
    const int quads = groups * 4;                               // of neighbouring outputs in this CTA
    for (int i = threadIdx.x; i < (int)m_end * quads; i += kFewWarps * 32) {
        const int row = i / quads, q = i - row * quads;
        const int64_t col = (int64_t)blockIdx.x * groups * 16 + q * 4;
        if (col >= p.n) continue;
        float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int s = 0; s < share; ++s) {
            const float4 f = *reinterpret_cast<const float4*>(&tile[q / 4 * share + s][row][q % 4 * 4]);
            z[0] += f.x;
            z[1] += f.y;
            z[2] += f.z;
            z[3] += f.w;
        }
        float bias[4];
        load_bias(p, col, bias);
        finish_quads<T, 1>(p, z, bias, row, 1, p.m, col, out_vec);
    }
}

template <typename T, bool VEC>
aa_status launch_few(aa_ctx_impl* c, const ProductParams& in, bool out_vec) {
    ProductParams p = in;
    // warps that share a sum: until every SM has eight warps, and no more than there are blocks
    const int64_t groups = (p.n + 15) / 16, blocks = (p.k + 31) / 32;
    int share = 1;
    while (share < kFewWarps && groups * share < 8ll * c->sm_count && blocks >= 4 * share) share *= 2;
    const int64_t grid = (groups * share + kFewWarps - 1) / kFewWarps;
    if (grid > 0x7FFFFFFF) return AA_ERR_UNSUPPORTED;
    const void* kernel = p.m <= 8 ? (const void*)linear_few_kernel<T, VEC, 1> : (const void*)linear_few_kernel<T, VEC, 2>;
    void* args[] = {&p, &share, &out_vec};
    if (launch_overlapped(c, kernel, dim3((unsigned)grid), dim3(kFewWarps * 32), args, 0, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

}  // namespace

bool product_few_fits(const ProductParams& p) { return p.m <= kFewRows && !p.a_across && !p.b_across; }

aa_status launch_product_few(aa_ctx_impl* c, const ProductParams& p, int dtype) {
    const int64_t es = dtype == AA_BF16 ? 2 : 4;
    const auto lies = [&](const MatArg& a, int64_t bytes) { return !a.data || ((uintptr_t)a.data % bytes == 0 && a.stride * es % bytes == 0); };
    const bool vec = lies(p.a, 16) && lies(p.b, 16) && p.k % 8 == 0;
    const bool out_vec = lies(p.out, 4 * es) && lies(p.pre, 4 * es) && lies(p.residual, 4 * es);
    if (dtype == AA_BF16) return vec ? launch_few<uint16_t, true>(c, p, out_vec) : launch_few<uint16_t, false>(c, p, out_vec);
    return vec ? launch_few<float, true>(c, p, out_vec) : launch_few<float, false>(c, p, out_vec);
}

}  // namespace aa
