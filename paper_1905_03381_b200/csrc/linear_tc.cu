// Products of linear layers on the 5th-generation tensor cores (tcgen05), bf16 operands that TMA can fetch.
//
// A persistent CTA per SM takes 128 x BN tiles of C = A B^T.  One warp fetches 64-wide slices of both operands into a ring (128-byte swizzle; an operand
// whose contraction runs across its stored rows is fetched as it lies and read by the matrix unit in its other orientation, so nothing is
// ever transposed in memory), one warp issues the products (M = 128, N = BN, K = 16, four a slice) into one of two accumulators in TMEM, and eight warps
// take the finished accumulator through a 32 x 32 stage of their own - a thread holds a row of the accumulator but has to store along
// rows - while the next tile's products run.  Bias, activation, residual and the single rounding happen on that way.
#include "linear.cuh"
#include "tensor_core.cuh"

namespace aa {

namespace {

constexpr int kBM = 128, kSlice = 64, kGroupM = 16;
constexpr int kTcThreads = 384;          // producer, issuer, allocator, one idle warp, eight epilogue warps
constexpr int kEpilogue = 8;
constexpr int kStageFloats = 32 * 32;    // per epilogue warp
constexpr int kMaxStages = 8;

template <int BN>
struct Geo {
    static constexpr int A = kBM * 128, B = BN * 128, STAGE = A + B;
    static constexpr int STAGES = BN == 256 ? 4 : (BN == 128 ? 6 : 8);
    static constexpr int TMEM = 2 * BN < 32 ? 32 : 2 * BN;
    static constexpr size_t SMEM = 1024 + (size_t)STAGES * STAGE + kEpilogue * kStageFloats * sizeof(float);
};

struct Ctl {
    uint64_t full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2], drain;
    uint32_t tmem;
    int abort_flag;
};

struct Tiles {
    int mt, nt, n;                       // of this launch
};

__device__ __forceinline__ void tile_at(const Tiles& t, int i, int& m, int& n) {
    const int per = kGroupM * t.nt, g = i / per, in = i - g * per, rows = min(kGroupM, t.mt - g * kGroupM);
    n = in / rows;
    m = g * kGroupM + (in - n * rows);
}

template <int BN, bool A_ACROSS, bool B_ACROSS>
__global__ void __launch_bounds__(kTcThreads, 1)
product_tc_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ ProductParams p, int mt, int nt, bool vec) {
    using G = Geo<BN>;
    extern __shared__ unsigned char smem_raw[];
    __shared__ Ctl ctl;
    unsigned char* ring = reinterpret_cast<unsigned char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    float* stage_f = reinterpret_cast<float*>(ring + (size_t)G::STAGES * G::STAGE);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* abort_flag = &ctl.abort_flag;
    if (threadIdx.x == 0) {
        for (int s = 0; s < G::STAGES; ++s) {
            mbar_init(&ctl.full[s], 1);
            mbar_init(&ctl.empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&ctl.acc_full[b], 1);
            mbar_init(&ctl.acc_empty[b], kEpilogue);
        }
        mbar_init(&ctl.drain, 1);
        ctl.abort_flag = 0;
        mbar_fence_init();
        prefetch_tensormap(&map_a);
        prefetch_tensormap(&map_b);
    }
    if (warp == 2) tmem_alloc(&ctl.tmem, G::TMEM);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *(volatile uint32_t*)&ctl.tmem;
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, blockIdx.x == 0 && threadIdx.x == 0);
    const int64_t m_end = p.live_k ? p.m : min(p.m, live), k_end = p.live_k ? min(p.k, live) : p.k;
    const Tiles tiles{(int)((m_end + kBM - 1) / kBM), nt, (int)((m_end + kBM - 1) / kBM) * nt};
    const int slices = (int)((k_end + kSlice - 1) / kSlice);
    bool ok = true;
    if (slices == 0) {
        // no term at all: only the epilogue has work
    } else if (warp == 0) {
        // ---- producer
        int stage = 0, sent = 0;
        uint32_t phase = 0;
        for (int i = blockIdx.x; i < tiles.n && ok; i += gridDim.x) {
            int m, n;
            tile_at(tiles, i, m, n);
            for (int s = 0; s < slices; ++s) {
                if (!__all_sync(0xFFFFFFFFu, mbar_wait(&ctl.empty[stage], phase ^ 1u, abort_flag))) {
                    ok = false;
                    break;
                }
                if (lane == 0) {
                    unsigned char* a = ring + (size_t)stage * G::STAGE;
                    unsigned char* b = a + G::A;
                    mbar_arrive_expect_tx(&ctl.full[stage], G::STAGE);
                    if (A_ACROSS) {
#pragma unroll
                        for (int c = 0; c < kBM / 64; ++c) tma_load_2d(a + c * 8192, &map_a, m * kBM + c * 64, s * kSlice, &ctl.full[stage]);
                    } else {
                        tma_load_2d(a, &map_a, s * kSlice, m * kBM, &ctl.full[stage]);
                    }
                    if (B_ACROSS) {
#pragma unroll
                        for (int c = 0; c < BN / 64; ++c) tma_load_2d(b + c * 8192, &map_b, n * BN + c * 64, s * kSlice, &ctl.full[stage]);
                    } else {
                        tma_load_2d(b, &map_b, s * kSlice, n * BN, &ctl.full[stage]);
                    }
                }
                __syncwarp();
                ++sent;
                if (++stage == G::STAGES) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
        }
        if (!ok) {
            // copies still in flight land before the CTA's shared memory goes away
            const int pending = sent < G::STAGES ? sent : G::STAGES;
            for (int back = 1; back <= pending; ++back) {
                const int j = sent - back;
                const long long t0 = clock64();
                while (!mbar_try_wait(&ctl.full[j % G::STAGES], (uint32_t)((j / G::STAGES) & 1)) && clock64() - t0 < kWaitCycles) {
                }
            }
        }
    } else if (warp == 1) {
        // ---- issuer
        constexpr uint32_t idesc = umma_idesc_bf16(kBM, BN, A_ACROSS, B_ACROSS);
        int stage = 0, it = 0;
        uint32_t phase = 0;
        for (int i = blockIdx.x; i < tiles.n && ok; i += gridDim.x, ++it) {
            const int buf = it & 1;
            if (!__all_sync(0xFFFFFFFFu, mbar_wait(&ctl.acc_empty[buf], (uint32_t)(((it >> 1) & 1) ^ 1), abort_flag))) {
                ok = false;
                break;
            }
            tc_fence_after_sync();
            const uint32_t d = tmem + (uint32_t)(buf * BN);
            for (int s = 0; s < slices; ++s) {
                if (!__all_sync(0xFFFFFFFFu, mbar_wait(&ctl.full[stage], phase, abort_flag))) {
                    ok = false;
                    break;
                }
                unsigned char* at = ring + (size_t)stage * G::STAGE;
                const int left = (int)min((int64_t)kSlice, k_end - (int64_t)s * kSlice);
                if (A_ACROSS && B_ACROSS && left < kSlice && k_end < p.k) {
                    // stored rows past the counted ones may hold anything, and must not reach a sum, not even times zero
                    for (int u = lane; u < (kSlice - left) * 8 * (kBM + BN) / 64; u += 32) {
                        const int c = u / ((kSlice - left) * 8), r = u - c * (kSlice - left) * 8;
                        *reinterpret_cast<uint4*>(at + c * 8192 + left * 128 + r * 16) = make_uint4(0, 0, 0, 0);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                }
                tc_fence_after_sync();
                if (lane == 0) {
                    const uint32_t a = smem_u32(at), b = a + G::A;
#pragma unroll
                    for (int k = 0; k < kSlice / 16; ++k) {
                        const uint64_t ad = A_ACROSS ? umma_smem_desc(a + k * 2048, 8192, 1024) : umma_smem_desc(a + k * 32, 16, 1024);
                        const uint64_t bd = B_ACROSS ? umma_smem_desc(b + k * 2048, 8192, 1024) : umma_smem_desc(b + k * 32, 16, 1024);
                        umma_bf16(d, ad, bd, idesc, (s | k) != 0);
                    }
                    umma_commit(&ctl.empty[stage]);
                    if (s == slices - 1) umma_commit(&ctl.acc_full[buf]);
                }
                __syncwarp();
                if (++stage == G::STAGES) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
        }
        if (lane == 0) umma_commit(&ctl.drain);
        __syncwarp();
        const long long t0 = clock64();
        while (!mbar_try_wait(&ctl.drain, 0) && clock64() - t0 < kWaitCycles) {
        }
    }
    if (warp >= 4) {
        // ---- epilogue
        const int quad = warp & 3, half = (warp - 4) >> 2;
        float* mine = stage_f + (warp - 4) * kStageFloats;
        const int sub = lane & 7, r8 = lane >> 3;
        uint16_t* out = static_cast<uint16_t*>(const_cast<void*>(p.out.data));
        uint16_t* pre = static_cast<uint16_t*>(const_cast<void*>(p.pre.data));
        const uint16_t* res = static_cast<const uint16_t*>(p.residual.data);
        int it = 0;
        for (int i = blockIdx.x; i < tiles.n && ok; i += gridDim.x, ++it) {
            int m, n;
            tile_at(tiles, i, m, n);
            const int buf = it & 1;
            if (slices > 0) {
                if (!__all_sync(0xFFFFFFFFu, mbar_wait(&ctl.acc_full[buf], (uint32_t)((it >> 1) & 1), abort_flag))) {
                    ok = false;
                    break;
                }
                tc_fence_after_sync();
            }
            const int64_t row0 = (int64_t)m * kBM + quad * 32;
#pragma unroll 1
            for (int c = 0; c < BN / 64; ++c) {
                const int64_t col = (int64_t)n * BN + half * (BN / 2) + c * 32 + sub * 4;
                const bool whole = vec && col + 4 <= p.n;
                float bias[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) bias[e] = p.bias && col + e < p.n ? p.bias[col + e] : 0.0f;
                uint32_t v[32];
                if (slices > 0) {
                    tmem_ld_32cols(tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(buf * BN + half * (BN / 2) + c * 32), v);
                    tmem_ld_wait();
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = 0u;
                }
                if (c == BN / 64 - 1 && slices > 0) {
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&ctl.acc_empty[buf]);
                }
                __syncwarp();                // the stage's readers of the chunk before are done
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    *reinterpret_cast<uint4*>(mine + lane * 32 + ((u ^ (lane & 7)) << 2)) = make_uint4(v[4 * u], v[4 * u + 1], v[4 * u + 2], v[4 * u + 3]);
                __syncwarp();
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const int r = q * 4 + r8;
                    const int64_t row = row0 + r;
                    const float4 f = *reinterpret_cast<const float4*>(mine + r * 32 + ((sub ^ (r & 7)) << 2));
                    float z[4] = {f.x + bias[0], f.y + bias[1], f.z + bias[2], f.w + bias[3]};
                    if (row >= m_end) continue;
                    if (whole) {
                        if (pre) *reinterpret_cast<uint2*>(pre + row * p.pre.stride + col) = make_uint2(pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3]));
#pragma unroll
                        for (int e = 0; e < 4; ++e) z[e] = activate(z[e], p.act);
                        if (res) {
                            const uint2 w = *reinterpret_cast<const uint2*>(res + row * p.residual.stride + col);
                            z[0] += bf16_lo(w.x);
                            z[1] += bf16_hi(w.x);
                            z[2] += bf16_lo(w.y);
                            z[3] += bf16_hi(w.y);
                        }
                        *reinterpret_cast<uint2*>(out + row * p.out.stride + col) = make_uint2(pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3]));
                    } else {
                        for (int e = 0; e < 4; ++e) {
                            if (col + e >= p.n) break;
                            if (pre) store1(pre + row * p.pre.stride + col + e, z[e]);
                            float y = activate(z[e], p.act);
                            if (res) y += load1(res + row * p.residual.stride + col + e);
                            store1(out + row * p.out.stride + col + e, y);
                        }
                    }
                }
            }
        }
    }
    if (!ok) {
        *abort_flag = 1;
        if (lane == 0) latch(p.ctl, AA_ERR_SCAN_TIMEOUT);
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == 2) tmem_dealloc(tmem, G::TMEM);
}

template <int BN, bool AA, bool BA>
aa_status launch_tc(aa_ctx_impl* c, const ProductParams& in, bool vec) {
    using G = Geo<BN>;
    ProductParams p = in;
    alignas(64) CUtensorMap map_a, map_b;
    const int64_t a_rows = AA ? p.k : p.m, a_cols = AA ? p.m : p.k, b_rows = BA ? p.k : p.n, b_cols = BA ? p.n : p.k;
    if (!encode_bf16_tile_map(&map_a, p.a.data, a_rows, a_cols, p.a.stride, AA ? kSlice : kBM) ||
        !encode_bf16_tile_map(&map_b, p.b.data, b_rows, b_cols, p.b.stride, BA ? kSlice : BN))
        return AA_ERR_CUDA;
    int mt = (int)((p.m + kBM - 1) / kBM), nt = (int)((p.n + BN - 1) / BN);
    const void* kernel = (const void*)product_tc_kernel<BN, AA, BA>;
    if (allow_smem(c, kernel, G::SMEM) != AA_OK) return AA_ERR_CUDA;
    const int64_t n = (int64_t)mt * nt;
    const int grid = (int)(n < c->sm_count ? n : c->sm_count);
    void* args[] = {&map_a, &map_b, &p, &mt, &nt, &vec};
    if (launch_overlapped(c, kernel, dim3(grid), dim3(kTcThreads), args, G::SMEM, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

template <int BN>
aa_status launch_majors(aa_ctx_impl* c, const ProductParams& p, bool vec) {
    if (p.a_across) return launch_tc<BN, true, true>(c, p, vec);
    return p.b_across ? launch_tc<BN, false, true>(c, p, vec) : launch_tc<BN, false, false>(c, p, vec);
}

}  // namespace

bool product_tc_fits(const ProductParams& p) {
    const auto tma = [](const MatArg& a) { return (uintptr_t)a.data % 16 == 0 && a.stride % 8 == 0; };
    const int64_t tiles = ((p.m + kBM - 1) / kBM) * ((p.n + 63) / 64);
    return tma(p.a) && tma(p.b) && p.m <= 0x3FFFFFFF && p.n <= 0x3FFFFFFF && p.k <= 0x3FFFFFFF && tiles < 0x3FFFFFFF;
}

aa_status launch_product_tc(aa_ctx_impl* c, const ProductParams& p) {
    const auto quad = [](const MatArg& a) { return !a.data || ((uintptr_t)a.data % 8 == 0 && a.stride % 4 == 0); };
    const bool vec = quad(p.out) && quad(p.pre) && quad(p.residual);
    // the widest tile moves the fewest bytes a product; narrower ones where it would leave SMs idle
    const int64_t mt = (p.m + kBM - 1) / kBM;
    const auto waves = [&](int bn) { return (double)((mt * ((p.n + bn - 1) / bn) + c->sm_count - 1) / c->sm_count) * bn; };
    if (p.n > 128 && waves(256) <= waves(128)) return launch_majors<256>(c, p, vec);
    if (p.n > 64 && waves(128) <= waves(64)) return launch_majors<128>(c, p, vec);
    return launch_majors<64>(c, p, vec);
}

}  // namespace aa
