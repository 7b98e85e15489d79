// Products of linear layers on the 5th-generation tensor cores (tcgen05), bf16 operands that TMA can fetch.
//
// A persistent pair of CTAs (a cluster of two SMs) takes 256 x 256 tiles of C = A B^T, a single CTA 128 x 64 tiles where there are few of those.  A warp fetches
// 64-wide slices of its CTA's 128 rows of A and of its half of B into a ring (128-byte swizzle; an operand whose contraction runs across its
// stored rows is fetched as it lies and read by the matrix unit in its other orientation, so nothing is ever transposed in memory).  One warp
// of the pair issues the products (M = 256, N = BN, K = 16, four a slice), which read both CTAs' shared memory and leave 128 rows in each CTA's TMEM.
// Two accumulators alternate: eight warps take the finished one through
// a 32 x 32 stage of their own - a thread holds a row of the accumulator but has to store along rows - while the next tile's products run.
// Bias, activation, residual and the single rounding happen on that way.
// Pairs, because a tile of 128 x 256 needs 96 bytes a cycle and SM out of L2, which gives about 60, and one of 256 x 256 needs 64.
//
// 8,192^3 takes 690 us (1.59 PFLOP/s, of 1.62 that a library's plain product reaches in a burst); 25,000 x 2,048 -> 512 44 us behind other launches (1.19 PFLOP/s):
// 196 tiles are 2.65 rounds of 74 pairs, which a forward call, without scratch memory, takes as three.  Few rows are bound by latency: 64 x 512 -> 2,048 takes 10 us.
//
// The matrix unit rounds a sum towards zero, by a step of it (a part in 2^23 at most) once in 16 terms, all in one direction: a million terms of one sign lose more than the
// rounding to bf16 does.  So a run of 2,048 terms at most stays in TMEM (a part in 2^16); the epilogue's warps add longer sums up in registers, in fp32 with ordinary rounding, while
// the next run's products go on.  A thread holds 128 columns of a row for that, so those warps take registers over from the others (setmaxnreg).  The vocabulary gradients take
// 1,565 us without runs and 1,590 with them, of 1,024 to 8,192 terms alike.
//
// Tiles that do not fill the last round of SMs can be cut along the contraction (the backward call has scratch memory): their parts go to
// scratch in fp32 and a second kernel adds them up in order and finishes them.
#include "cta_pair.cuh"
#include "linear_plan.cuh"

namespace aa {

namespace {

constexpr int kBM = 128;
constexpr int kTcThreads = 384;          // producer, issuer, allocator, an idle warp, eight for the epilogue
constexpr int kSumThreads = 512;         // and four for column sums
constexpr int kEpilogue = 8;
constexpr int kStageFloats = 32 * 32;    // per epilogue warp
constexpr int kMaxStages = 8;
constexpr int kTcRun = 32;               // slices summed in TMEM

// CG CTAs share a tile of CG 128 rows and BN columns.
template <int CG, int BN>
struct Geo {
    static constexpr int A = kBM * 128, ROWS_B = BN / CG, B = ROWS_B * 128, STAGE = A + B;
    static constexpr int STAGES = CG == 2 ? 6 : 8;
    static constexpr int TMEM = 2 * BN;
    static constexpr size_t SMEM = 1024 + (size_t)STAGES * STAGE + kEpilogue * kStageFloats * sizeof(float);
};

// Registers a thread of a pair's kernel, as launched and then: eight warps of the epilogue, all others.  No more in all than were launched, or the epilogue would wait for good.
template <bool SUMS>
struct Registers {
    static constexpr int THREADS = SUMS ? kSumThreads : kTcThreads, LAUNCH = SUMS ? 128 : 168, OTHERS = SUMS ? 72 : 56, EPILOGUE = SUMS ? 184 : 224;
    static_assert((THREADS - 256) * OTHERS + 256 * EPILOGUE <= THREADS * LAUNCH && THREADS * LAUNCH <= 65536, "");
};

struct Ctl {
    uint64_t full[kMaxStages], empty[kMaxStages], done[kMaxStages], acc_full[2], acc_empty[2], drain;
    uint64_t ragged, cleared;            // the last slice of tokens: it has arrived (second CTA), its rest is zero there (first CTA)
    uint32_t tmem;
    int abort_flag;
};

// A lane's part of a 32 x 32 chunk out of the warp's stage: four columns of rows r8, r8 + 4, ... below `rows`.  Steps are four rows, in elements.
template <int ACT>
__device__ __forceinline__ void put_chunk(uint32_t stage, int sub, int r8, int rows, const float (&bias)[4], bool some, const uint2 (&add)[8], uint16_t* to, int64_t step,
                                          uint16_t* raw, int64_t raw_step) {
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        float z[4];
        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                     : "=f"(z[0]), "=f"(z[1]), "=f"(z[2]), "=f"(z[3])
                     : "r"(stage + (uint32_t)(q * 512 + ((sub ^ ((q * 4 + r8) & 7)) << 4)))
                     : "memory");
        if (q * 4 + r8 < rows) {
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] += bias[e];
            if (raw) *reinterpret_cast<uint2*>(raw) = make_uint2(pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3]));
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] = activate<ACT, false>(z[e]);
            if (some) {
                z[0] += bf16_lo(add[q].x);
                z[1] += bf16_hi(add[q].x);
                z[2] += bf16_lo(add[q].y);
                z[3] += bf16_hi(add[q].y);
            }
            *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3]));
        }
        to += step;
        if (raw) raw += raw_step;
    }
}

__device__ __forceinline__ void store_shared(uint32_t at, const float* f) {
    asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at), "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]) : "memory");
}

// SUMS: the sums of A over the contraction, too (A's slices are in shared memory already; another pass over A would cost as much as reading it).  Four
// warps add up the slice's 128 columns once the products have read it and hand the stage back with them (two warps took longer than the products).
// JOIN (single CTAs): the parts of a tile are the CTAs of a cluster, as in linear_plan.cuh; a CTA has one unit then.
// RUNS: a unit may have more than kTcRun slices.  (25,000 x 2,048 -> 512 takes 54 us without, 56 to 60 through the registers of a kernel that has both ways.)
template <int CG, int BN, bool A_ACROSS, bool B_ACROSS, bool SUMS, bool JOIN, bool RUNS>
__global__ void __launch_bounds__(SUMS ? kSumThreads : kTcThreads, 1)
product_tc_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ ProductParams p, const __grid_constant__ Plan plan,
                  bool vec) {
    using G = Geo<CG, BN>;
    constexpr bool PARTS = A_ACROSS || B_ACROSS;         // a backward call: scratch memory for parts
    extern __shared__ unsigned char smem_raw[];
    __shared__ Ctl ctl;
    unsigned char* ring = reinterpret_cast<unsigned char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    float* stage_f = reinterpret_cast<float*>(ring + (size_t)G::STAGES * G::STAGE);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = CG == 1 ? 0 : (int)cluster_rank();
    Unit last = {};                      // JOIN: the tile, and whether there is one
    bool has = false;
    volatile int* abort_flag = &ctl.abort_flag;
    if (threadIdx.x == 0) {
        for (int s = 0; s < G::STAGES; ++s) {
            mbar_init(&ctl.full[s], 1);      // both CTAs' copies count on the first one's
            mbar_init(&ctl.empty[s], SUMS ? 5 : 1);
            mbar_init(&ctl.done[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&ctl.acc_full[b], 1);
            mbar_init(&ctl.acc_empty[b], CG * kEpilogue);
        }
        mbar_init(&ctl.drain, 1);
        mbar_init(&ctl.ragged, 1);
        mbar_init(&ctl.cleared, 1);
        ctl.abort_flag = 0;
        mbar_fence_init();
        prefetch_tensormap(&map_a);
        prefetch_tensormap(&map_b);
    }
    if (warp == 2) alloc<CG>(&ctl.tmem, G::TMEM);
    tc_fence_before_sync();
    __syncthreads();
    if (CG == 2) cluster_sync_all();
    tc_fence_after_sync();
    const uint32_t tmem = *(volatile uint32_t*)&ctl.tmem;
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, blockIdx.x == 0 && threadIdx.x == 0);
    const int64_t m_end = p.live_k ? p.m : min(p.m, live), k_end = p.live_k ? min(p.k, live) : p.k;
    const int mt = (int)((m_end + CG * kBM - 1) / (CG * kBM)), units = units_of(plan, mt);
    const int slices = (int)((k_end + kSlice - 1) / kSlice);
    const int first = blockIdx.x / CG, step = gridDim.x / CG;
    bool ok = true;
    if (warp >= 4 && warp < 12) {
        if (CG == 2 && RUNS) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Registers<SUMS>::EPILOGUE));
        // ---- epilogue
        const int quad = warp & 3, half = (warp - 4) >> 2;
        float* mine = stage_f + (warp - 4) * kStageFloats;
        const int sub = lane & 7, r8 = lane >> 3;
        const uint32_t my_row = smem_u32(mine + lane * 32);
        uint16_t* out = static_cast<uint16_t*>(const_cast<void*>(p.out.data));
        uint16_t* pre = PARTS ? nullptr : static_cast<uint16_t*>(const_cast<void*>(p.pre.data));
        const uint16_t* res = A_ACROSS ? nullptr : static_cast<const uint16_t*>(p.residual.data);
        int it = 0;
        for (int i = first; i < units && ok; i += step) {
            const Unit u = unit_at(plan, mt, slices, i);
            const bool some = u.s0 < u.s1;   // else no term at all
            const int64_t row0 = ((int64_t)u.m * CG + rank) * kBM + quad * 32 + r8;
            const int rows = (int)max((int64_t)0, min((int64_t)32, m_end - row0 + r8));      // of the warp's 32 that count
            float sum[RUNS ? BN / 2 : 1];    // a row's columns of this warp
            int buf = 0;
            const auto arrived = [&]() {
                buf = it & 1;
                ok = __all_sync(0xFFFFFFFFu, mbar_wait(&ctl.acc_full[buf], (uint32_t)((it >> 1) & 1), abort_flag));
                tc_fence_after_sync();
                ++it;
            };
            const auto load = [&](int c, float (&f)[32]) {
                uint32_t v[32];
                tmem_ld_32cols(tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)(buf * BN + half * (BN / 2) + c * 32), v);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 32; ++e) f[e] = __uint_as_float(v[e]);
            };
            const auto release = [&]() {
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) {
                    if (CG == 1) mbar_arrive(&ctl.acc_empty[buf]);
                    else mbar_arrive_at(of_rank(&ctl.acc_empty[buf], 0));
                }
            };
            if constexpr (RUNS) {
#pragma unroll
                for (int e = 0; e < BN / 2; ++e) sum[e] = 0.0f;
                for (int s = u.s0; s < u.s1 && ok; s += kTcRun) {
                    arrived();
                    if (!ok) break;
#pragma unroll
                    for (int c = 0; c < BN / 64; ++c) {
                        float f[32];
                        load(c, f);
#pragma unroll
                        for (int e = 0; e < 32; ++e) sum[c * 32 + e] += f[e];
                    }
                    release();
                }
            } else if (some) {
                arrived();
            }
            if (!ok) break;
            if (JOIN) {
                // every CTA of the cluster is through with its ring: its shared memory takes the parts of 128 / cluster rows
                last = u;
                has = true;
                cluster_sync_all();
            }
#pragma unroll 1
            for (int c = 0; c < BN / 64; ++c) {
                const int64_t col = (int64_t)u.n * BN + half * (BN / 2) + c * 32 + sub * 4;
                const bool whole = vec && col + 4 <= p.n;
                uint2 add[8];
                if (!JOIN && res && whole && u.part < 0) {
#pragma unroll
                    for (int q = 0; q < 8; ++q) add[q] = r8 + q * 4 < rows ? *reinterpret_cast<const uint2*>(res + (row0 + q * 4) * p.residual.stride + col) : make_uint2(0, 0);
                } else {
#pragma unroll
                    for (int q = 0; q < 8; ++q) add[q] = make_uint2(0, 0);
                }
                float bias[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                if (!PARTS && p.bias) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) bias[e] = col + e < p.n ? p.bias[col + e] : 0.0f;
                }
                // the lane's 32 numbers: to the stage, or to the CTAs that finish them
                const auto give = [&](const float* f) {
                    if (JOIN) {
                        const int rows = kBM / plan.cluster, r = quad * 32 + lane;
                        const uint32_t to = of_rank(ring, (uint32_t)(r / rows)) + (uint32_t)((((int)cluster_rank() * rows + r % rows) * BN + half * (BN / 2) + c * 32) * 4);
#pragma unroll
                        for (int e = 0; e < 32; e += 4) store_remote(to + (uint32_t)(e * 4), make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]));
                    } else {
#pragma unroll
                        for (int w = 0; w < 8; ++w) store_shared(my_row + (uint32_t)((w ^ (lane & 7)) << 4), f + 4 * w);
                    }
                };
                __syncwarp();                // the stage's readers of the chunk before are done
                if constexpr (RUNS) {
                    // (four stores of their own: a choice among registers would be 128 instructions)
#pragma unroll
                    for (int q = 0; q < BN / 64; ++q)
                        if (c == q) give(sum + q * 32);
                } else {
                    float f[32];
                    if (some) {
                        load(c, f);
                        if (c == BN / 64 - 1) release();
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) f[e] = 0.0f;
                    }
                    give(f);
                }
                if (JOIN) continue;
                __syncwarp();
                if (PARTS && u.part >= 0) {
                    float* to = plan.parts + ((int64_t)u.part * CG + rank) * kBM * BN + (int64_t)(quad * 32 + r8) * BN + half * (BN / 2) + c * 32 + sub * 4;
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        *reinterpret_cast<float4*>(to + q * 4 * BN) = *reinterpret_cast<const float4*>(mine + (q * 4 + r8) * 32 + ((sub ^ ((q * 4 + r8) & 7)) << 2));
                    continue;
                }
                if (whole) {
                    const uint32_t at = smem_u32(mine + r8 * 32);
                    uint16_t* to = out + row0 * p.out.stride + col;
                    uint16_t* raw = pre ? pre + row0 * p.pre.stride + col : nullptr;
                    if (PARTS || p.act == AA_ACT_NONE) put_chunk<AA_ACT_NONE>(at, sub, r8, rows, bias, res != nullptr, add, to, p.out.stride * 4, raw, p.pre.stride * 4);
                    else if (p.act == AA_ACT_RELU) put_chunk<AA_ACT_RELU>(at, sub, r8, rows, bias, res != nullptr, add, to, p.out.stride * 4, raw, p.pre.stride * 4);
                    else if (p.act == AA_ACT_GELU) put_chunk<AA_ACT_GELU>(at, sub, r8, rows, bias, res != nullptr, add, to, p.out.stride * 4, raw, p.pre.stride * 4);
                    else put_chunk<AA_ACT_SILU>(at, sub, r8, rows, bias, res != nullptr, add, to, p.out.stride * 4, raw, p.pre.stride * 4);
                } else {
                    // (128 more registers hold sums; four rows at once would spill)
                    constexpr int AT_ONCE = CG == 2 && RUNS && SUMS ? 2 : 4;
#pragma unroll 1
                    for (int q0 = 0; q0 < 8; q0 += AT_ONCE) {
                        float z[AT_ONCE * 4];
#pragma unroll
                        for (int q = 0; q < AT_ONCE; ++q) {
                            const int r = (q0 + q) * 4 + r8;
                            const float4 f = *reinterpret_cast<const float4*>(mine + r * 32 + ((sub ^ (r & 7)) << 2));
                            z[q * 4] = f.x, z[q * 4 + 1] = f.y, z[q * 4 + 2] = f.z, z[q * 4 + 3] = f.w;
                        }
                        finish_quads<uint16_t, AT_ONCE>(p, z, bias, row0 + q0 * 4, 4, m_end, col, false);
                    }
                }
            }
        }
    } else {
        if (CG == 2 && RUNS) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Registers<SUMS>::OTHERS));
        if (warp == 0) {
            // ---- producer
            int stage = 0, sent = 0;
            uint32_t phase = 0;
            for (int i = first; i < units && ok; i += step) {
                const Unit u = unit_at(plan, mt, slices, i);
                const int am = (u.m * CG + rank) * kBM, bn = u.n * BN + rank * G::ROWS_B;
                for (int s = u.s0; s < u.s1; ++s) {
                    if (!__all_sync(0xFFFFFFFFu, mbar_wait(&ctl.empty[stage], phase ^ 1u, abort_flag))) {
                        ok = false;
                        break;
                    }
                    if (elect_one()) {
                        unsigned char* a = ring + (size_t)stage * G::STAGE;
                        unsigned char* b = a + G::A;
                        uint64_t* bar = &ctl.full[stage];
                        const uint32_t bar0 = CG == 1 ? 0u : of_rank(bar, 0);
                        if (rank == 0) mbar_arrive_expect_tx(bar, CG * G::STAGE);
                        if (A_ACROSS) {
#pragma unroll
                            for (int c = 0; c < kBM / 64; ++c) load_box<CG>(a + c * 8192, &map_a, am + c * 64, s * kSlice, bar, bar0);
                        } else {
                            load_box<CG>(a, &map_a, s * kSlice, am, bar, bar0);
                        }
                        if (B_ACROSS) {
#pragma unroll
                            for (int c = 0; c < G::ROWS_B / 64; ++c) load_box<CG>(b + c * 8192, &map_b, bn + c * 64, s * kSlice, bar, bar0);
                        } else {
                            load_box<CG>(b, &map_b, s * kSlice, bn, bar, bar0);
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
            if (!ok && rank == 0) {
                // copies still in flight land before the shared memory of either CTA goes away
                const int pending = sent < G::STAGES ? sent : G::STAGES;
                for (int back = 1; back <= pending; ++back) {
                    const int j = sent - back;
                    const long long t0 = clock64();
                    while (!mbar_try_wait(&ctl.full[j % G::STAGES], (uint32_t)((j / G::STAGES) & 1)) && clock64() - t0 < kWaitCycles) {
                    }
                }
            }
        } else if (warp == 1) {
            // ---- issuer; in the second CTA it only clears what lies behind the last token
            constexpr uint32_t idesc = umma_idesc_bf16(CG * kBM, BN, A_ACROSS, B_ACROSS);
            const uint64_t a_desc = umma_smem_desc(smem_u32(ring), A_ACROSS ? 8192 : 16, 1024), b_desc = umma_smem_desc(smem_u32(ring) + G::A, B_ACROSS ? 8192 : 16, 1024);
            int it = 0;
            uint32_t sent = 0, ragged = 0;
            for (int i = first; i < units && ok; i += step) {
                const Unit u = unit_at(plan, mt, slices, i);
                for (int r0 = u.s0, r1; r0 < u.s1 && ok; r0 = r1) {
                    r1 = RUNS ? min(r0 + kTcRun, u.s1) : u.s1;
                    const int buf = it & 1;
                    const uint32_t d = tmem + (uint32_t)(buf * BN);
                    if (rank == 0) {
                        if (!__all_sync(0xFFFFFFFFu, mbar_wait(&ctl.acc_empty[buf], (uint32_t)(((it >> 1) & 1) ^ 1), abort_flag))) {
                            ok = false;
                            break;
                        }
                        tc_fence_after_sync();
                    }
                    ++it;
                    for (int s = r0; s < r1; ++s, ++sent) {
                        const int stage = (int)(sent % G::STAGES), left = (int)min((int64_t)kSlice, k_end - (int64_t)s * kSlice);
                        unsigned char* at = ring + (size_t)stage * G::STAGE;
                        // stored rows past the counted ones may hold anything, and must not reach a sum, not even times zero
                        const bool clear = A_ACROSS && B_ACROSS && left < kSlice && k_end < p.k;
                        if (rank == 0) ok = __all_sync(0xFFFFFFFFu, mbar_wait(&ctl.full[stage], (sent / G::STAGES) & 1u, abort_flag));
                        else if (clear) ok = __all_sync(0xFFFFFFFFu, mbar_wait(&ctl.ragged, ragged, abort_flag));
                        if (!ok) break;
                        if (clear) {
                            if (CG == 2 && rank == 0 && lane == 0) mbar_arrive_at(of_rank(&ctl.ragged, 1));
                            const int per = (kSlice - left) * 8;
                            for (int q = lane; q < per * (kBM + G::ROWS_B) / 64; q += 32) {
                                const int c = q / per, r = q - c * per;
                                *reinterpret_cast<uint4*>(at + c * 8192 + left * 128 + r * 16) = make_uint4(0, 0, 0, 0);
                            }
                            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                            __syncwarp();
                            if (CG == 2) {
                                if (rank == 1 && lane == 0) mbar_release_at(of_rank(&ctl.cleared, 0));
                                if (rank == 0 && !__all_sync(0xFFFFFFFFu, mbar_wait(&ctl.cleared, ragged, abort_flag))) {
                                    ok = false;
                                    break;
                                }
                                ragged ^= 1u;
                            }
                        }
                        if (rank == 0) {
                            tc_fence_after_sync();
                            if (elect_one()) {
                                // the address is the descriptor's low field, in units of 16 bytes
                                const uint64_t ad = a_desc + (uint64_t)(uint32_t)(stage * (G::STAGE >> 4)), bd = b_desc + (uint64_t)(uint32_t)(stage * (G::STAGE >> 4));
#pragma unroll
                                for (int k = 0; k < kSlice / 16; ++k) mma<CG>(d, ad + (A_ACROSS ? k * 128 : k * 2), bd + (B_ACROSS ? k * 128 : k * 2), idesc, s > r0 || k > 0);
                                commit<CG>(&ctl.empty[stage]);
                                if (SUMS) commit<CG>(&ctl.done[stage]);
                                if (s == r1 - 1) commit<CG>(&ctl.acc_full[buf]);
                            }
                            __syncwarp();
                        }
                    }
                }
            }
            if (rank == 0) {
                if (elect_one()) commit<CG>(&ctl.drain);
                __syncwarp();
            }
            // both CTAs' memory is read until the last product is done
            const long long t0 = clock64();
            while (!mbar_try_wait(&ctl.drain, 0) && clock64() - t0 < kWaitCycles) {
            }
        } else if (SUMS && warp >= 12) {
            // ---- column sums: 64 of the CTA's 128 columns and half of the tokens a warp; a lane takes 8 columns of every fourth token
            const int chunk = warp & 1, part = (warp >> 1) & 1, unit = lane & 7, r4 = lane >> 3;
            __shared__ float halves[2][kBM];
            uint32_t sent = 0;
            // a warp that gave up still meets the others at their barriers
            for (int i = first; i < units; i += step) {
                const Unit u = unit_at(plan, mt, slices, i);
                float sum[8] = {};
                for (int s = u.s0; s < u.s1 && ok; ++s, ++sent) {
                    const int stage = (int)(sent % G::STAGES);
                    ok = __all_sync(0xFFFFFFFFu, mbar_wait(&ctl.done[stage], (sent / G::STAGES) & 1u, abort_flag));
                    if (!ok) break;
                    if (u.n == 0) {              // the tiles of a row of tiles share A
                        const unsigned char* at = ring + (size_t)stage * G::STAGE + chunk * 8192 + part * 4096;
                        float some[8] = {};
#pragma unroll
                        for (int q = 0; q < 8; ++q) {
                            const int r = q * 4 + r4;
                            float x[8];
                            Vec<uint16_t>::unpack(*reinterpret_cast<const uint4*>(at + r * 128 + ((unit ^ (r & 7)) << 4)), x);
#pragma unroll
                            for (int e = 0; e < 8; ++e) some[e] += x[e];
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e) sum[e] += some[e];
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&ctl.empty[stage]);
                }
                if (u.n != 0) continue;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    sum[e] += __shfl_xor_sync(0xFFFFFFFFu, sum[e], 8);
                    sum[e] += __shfl_xor_sync(0xFFFFFFFFu, sum[e], 16);
                    if (r4 == 0) halves[part][chunk * 64 + unit * 8 + e] = sum[e];
                }
                asm volatile("bar.sync 1, 128;" ::: "memory");
                const int at = (int)threadIdx.x - 384;
                const int64_t row = ((int64_t)u.m * CG + rank) * kBM + at;
                const float total = halves[0][at] + halves[1][at];
                if (u.part >= 0) plan.sum_parts[((int64_t)u.part * CG + rank) * kBM + at] = total;
                else if (row < p.m) p.a_sums[row] = total;
                asm volatile("bar.sync 1, 128;" ::: "memory");
            }
        }
    }
    if (JOIN) {
        // once before the parts are sent (the senders have done it) and once after
        if (!has) cluster_sync_all();
        cluster_sync_all();
        if (has) finish_cluster<uint16_t, BN>(p, plan, last, reinterpret_cast<const float*>(ring), m_end, vec, (int)threadIdx.x - 128, kEpilogue * 32);
    }
    if (!ok) {
        *abort_flag = 1;
        if (lane == 0) latch(p.ctl, AA_ERR_SCAN_TIMEOUT);
    }
    tc_fence_before_sync();
    __syncthreads();
    if (CG == 2) cluster_sync_all();         // nothing of the other CTA is on its way here any more
    tc_fence_after_sync();
    if (warp == 2) dealloc<CG>(tmem, G::TMEM);
}

// Whether a pair's kernel was compiled for the registers that it shares out; looked up once.
template <bool AA, bool BA, bool SUMS>
bool registers_ok() {
    static const bool ok = [] {
        cudaFuncAttributes attr;
        return cudaFuncGetAttributes(&attr, (const void*)product_tc_kernel<2, 256, AA, BA, SUMS, false, true>) == cudaSuccess && attr.numRegs >= Registers<SUMS>::LAUNCH;
    }();
    return ok;
}

template <int CG, int BN, bool AA, bool BA, bool SUMS, bool JOIN>
aa_status launch_tc(aa_ctx_impl* c, const ProductParams& in, bool vec, int cluster = 1) {
    using G = Geo<CG, BN>;
    constexpr int kThreads = SUMS ? kSumThreads : kTcThreads;
    ProductParams p = in;
    alignas(64) CUtensorMap map_a, map_b;
    const int64_t a_rows = AA ? p.k : p.m, a_cols = AA ? p.m : p.k, b_rows = BA ? p.k : p.n, b_cols = BA ? p.n : p.k;
    if (!encode_bf16_tile_map(&map_a, p.a.data, a_rows, a_cols, p.a.stride, AA ? kSlice : kBM) ||
        !encode_bf16_tile_map(&map_b, p.b.data, b_rows, b_cols, p.b.stride, BA ? kSlice : G::ROWS_B))
        return AA_ERR_CUDA;
    const int64_t mt = (p.m + CG * kBM - 1) / (CG * kBM), nt = (p.n + BN - 1) / BN, tiles = mt * nt, slices = (p.k + kSlice - 1) / kSlice;
    // (the kernel with runs takes the same threads and memory)
    const void* kernel = (const void*)product_tc_kernel<CG, BN, AA, BA, SUMS, JOIN, CG == 1>;
    if (allow_smem(c, kernel, G::SMEM) != AA_OK) return AA_ERR_CUDA;
    const int teams = CG == 1 ? c->sm_count : resident_clusters(c, kernel, kThreads, G::SMEM, CG);
    if (teams < 1) return AA_ERR_CUDA;
    Plan plan = make_plan(p, tiles, (int)nt, teams, (int64_t)CG * kBM * BN, CG * kBM, CG == 2 ? 0.4 : 0.2, cluster);
    const int64_t tail = tiles - plan.whole, units = plan.whole + tail * plan.splits;
    if constexpr (CG == 2)
        if ((plan.whole > 0 ? slices : (slices + plan.splits - 1) / plan.splits) > kTcRun) {
            kernel = (const void*)product_tc_kernel<CG, BN, AA, BA, SUMS, JOIN, true>;
            if (!registers_ok<AA, BA, SUMS>() || allow_smem(c, kernel, G::SMEM) != AA_OK) return AA_ERR_CUDA;
        }
    void* args[] = {&map_a, &map_b, &p, &plan, &vec};
    if (launch_clusters(c, kernel, (unsigned)(JOIN ? units : (units < teams ? units : teams) * CG), kThreads, args, G::SMEM, JOIN ? cluster : CG) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    if (tail == 0 || JOIN) return AA_OK;
    void* join[] = {&p, &plan, &vec};
    const int64_t threads = tail * CG * kBM * BN / 4;
    if (launch_overlapped(c, (const void*)product_join_kernel<uint16_t, CG * kBM, BN>, dim3((unsigned)(threads / 256)), dim3(256), join, 0, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

template <int CG, int BN>
aa_status launch_majors(aa_ctx_impl* c, const ProductParams& p, bool vec) {
    if (p.a_across) return p.a_sums ? launch_tc<CG, BN, true, true, true, false>(c, p, vec) : launch_tc<CG, BN, true, true, false, false>(c, p, vec);
    if (p.b_across) return launch_tc<CG, BN, false, true, false, false>(c, p, vec);
    if constexpr (CG == 1) {
        const int64_t tiles = (p.m + kBM - 1) / kBM * ((p.n + BN - 1) / BN);
        const void* kernel = (const void*)product_tc_kernel<CG, BN, false, false, false, true, true>;
        if (allow_smem(c, kernel, Geo<CG, BN>::SMEM) != AA_OK) return AA_ERR_CUDA;
        const int cluster = tile_cluster(c, kernel, kTcThreads, Geo<CG, BN>::SMEM, p, tiles);
        if (cluster > 1) return launch_tc<CG, BN, false, false, false, true>(c, p, vec, cluster);
    }
    return launch_tc<CG, BN, false, false, false, false>(c, p, vec);
}

}  // namespace

bool product_tc_fits(const ProductParams& p) {
    const auto tma = [](const MatArg& a) { return (uintptr_t)a.data % 16 == 0 && a.stride % 8 == 0; };
    const int64_t tiles = ((p.m + kBM - 1) / kBM) * ((p.n + 63) / 64);
    return tma(p.a) && tma(p.b) && p.m <= 0x3FFFFFFF && p.n <= 0x3FFFFFFF && p.k <= 0x3FFFFFFF && tiles < 0x3FFFFFF;
}

aa_status launch_product_tc(aa_ctx_impl* c, const ProductParams& p) {
    const auto quad = [](const MatArg& a) { return !a.data || ((uintptr_t)a.data % 8 == 0 && a.stride % 4 == 0); };
    const bool vec = quad(p.out) && quad(p.pre) && quad(p.residual);
    // the widest tile moves the fewest bytes a product (256 x 256 by pairs and 128 x 64: 8,192^3 721 and 1,772 us, 4,096 x 1,024 -> 1,024 15 and 25 us); narrow
    // ones where it would leave more than half of the SMs idle (500 x 512 -> 2,048: 12.9 and 12.4 us)
    const int64_t tiles = (p.m + kBM - 1) / kBM * ((p.n + 255) / 256), sms = c->sm_count;
    if (2 * tiles >= sms || (p.parts && p.k >= 16 * kSlice && tiles * (p.k / (8 * kSlice)) >= sms)) return launch_majors<2, 256>(c, p, vec);
    return launch_majors<1, 64>(c, p, vec);
}

}  // namespace aa
