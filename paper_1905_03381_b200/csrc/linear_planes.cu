// Products of fp32 matrices that were taken apart into three planes of bf16 terms beforehand (backward calls have scratch memory for them): see linear_split.cu for
// the arithmetic, linear_tc.cu for the pair of CTAs, the ring and the cut tiles.
//
// A pair of CTAs takes 256 x 128 tiles.  A slice is 72 KB a CTA - 64 terms of 128 rows of A and 64 of B in three planes each - and 24 products
// a pair, so that every byte fetched serves six products.  Every four slices the two accumulators (the products of the leading terms, and the
// others) go to the epilogue's registers, where the runs are added with ordinary rounding.
// 4,099 x 515 x 1,001 (4.2 GFLOP): 38 us for dx and 35 for dw, 0.11 PFLOP/s, the tensor pipe busy 42 % of the launch - 20 slices of 0.8 us a pair at most,
// between the first copies and the last tile's way out;
// the whole backward call takes 95 us with copies and column sums, 173 by linear_split.cu.
#include "cta_pair.cuh"
#include "linear_plan.cuh"

namespace aa {

namespace {

constexpr int kM = 128, kBN = 128, kHalfB = 64, kTerms = 3, kStages = 2, kRun = 4;
constexpr int kPlaneA = kM * 128, kPlaneB = kHalfB * 128, kStage = kTerms * (kPlaneA + kPlaneB);
constexpr int kPlaneThreads = 384, kEpilogue = 8;       // producer, issuer, allocator, one idle warp, eight epilogue warps
constexpr int kAcc = 2 * kBN;
constexpr size_t kPlaneSmem = 1024 + (size_t)kStages * kStage + kEpilogue * 32 * 32 * sizeof(float);

struct PlaneCtl {
    uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], drain;
    uint32_t tmem;
    int abort_flag;
};

template <bool A_ACROSS, bool B_ACROSS>
__global__ void __launch_bounds__(kPlaneThreads, 1)
product_planes_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ ProductParams p, const __grid_constant__ Plan plan,
                      bool vec) {
    extern __shared__ unsigned char smem_raw[];
    __shared__ PlaneCtl ctl;
    unsigned char* ring = reinterpret_cast<unsigned char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    float* stage_f = reinterpret_cast<float*>(ring + (size_t)kStages * kStage);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = (int)cluster_rank();
    volatile int* abort_flag = &ctl.abort_flag;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&ctl.full[s], 1);      // both CTAs' copies count on the first one's
            mbar_init(&ctl.empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&ctl.acc_full[b], 1);
            mbar_init(&ctl.acc_empty[b], 2 * kEpilogue);
        }
        mbar_init(&ctl.drain, 1);
        ctl.abort_flag = 0;
        mbar_fence_init();
        prefetch_tensormap(&map_a);
        prefetch_tensormap(&map_b);
    }
    if (warp == 2) alloc<2>(&ctl.tmem, 2 * kAcc);
    tc_fence_before_sync();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after_sync();
    const uint32_t tmem = *(volatile uint32_t*)&ctl.tmem;
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, blockIdx.x == 0 && threadIdx.x == 0);
    const int64_t m_end = p.live_k ? p.m : min(p.m, live), k_end = p.live_k ? min(p.k, live) : p.k;
    const int mt = (int)((m_end + 2 * kM - 1) / (2 * kM)), units = units_of(plan, mt), slices = (int)((k_end + kSlice - 1) / kSlice);
    const int first = blockIdx.x / 2, step = gridDim.x / 2;
    bool ok = true;
    if (warp == 0) {
        // ---- producer
        uint32_t sent = 0;
        for (int i = first; i < units && ok; i += step) {
            const Unit u = unit_at(plan, mt, slices, i);
            const int am = (u.m * 2 + rank) * kM, bn = u.n * kBN + rank * kHalfB;
            for (int s = u.s0; s < u.s1; ++s, ++sent) {
                const int stage = (int)(sent % kStages);
                if (!__all_sync(0xFFFFFFFFu, mbar_wait(&ctl.empty[stage], ((sent / kStages) & 1u) ^ 1u, abort_flag))) {
                    ok = false;
                    break;
                }
                if (elect_one()) {
                    unsigned char* a = ring + (size_t)stage * kStage;
                    unsigned char* b = a + kTerms * kPlaneA;
                    const uint32_t bar = of_rank(&ctl.full[stage], 0);
                    if (rank == 0) mbar_arrive_expect_tx(&ctl.full[stage], 2 * kStage);
#pragma unroll
                    for (int t = 0; t < kTerms; ++t) {
                        if (A_ACROSS) {
                            load_plane_box_pair(a + t * kPlaneA, &map_a, am, s * kSlice, t, bar);
                            load_plane_box_pair(a + t * kPlaneA + 8192, &map_a, am + 64, s * kSlice, t, bar);
                        } else {
                            load_plane_box_pair(a + t * kPlaneA, &map_a, s * kSlice, am, t, bar);
                        }
                        if (B_ACROSS) load_plane_box_pair(b + t * kPlaneB, &map_b, bn, s * kSlice, t, bar);
                        else load_plane_box_pair(b + t * kPlaneB, &map_b, s * kSlice, bn, t, bar);
                    }
                }
                __syncwarp();
            }
        }
        if (!ok && rank == 0) {
            // copies still in flight land before the shared memory of either CTA goes away
            const uint32_t pending = sent < kStages ? sent : kStages;
            for (uint32_t back = 1; back <= pending; ++back) {
                const uint32_t j = sent - back;
                const long long t0 = clock64();
                while (!mbar_try_wait(&ctl.full[j % kStages], (j / kStages) & 1u) && clock64() - t0 < kWaitCycles) {
                }
            }
        }
    } else if (warp == 1) {
        // ---- issuer
        constexpr uint32_t idesc = umma_idesc_bf16(2 * kM, kBN, A_ACROSS, B_ACROSS);
        const uint64_t a_desc = umma_smem_desc(smem_u32(ring), A_ACROSS ? 8192 : 16, 1024), b_desc = umma_smem_desc(smem_u32(ring) + kTerms * kPlaneA, B_ACROSS ? 8192 : 16, 1024);
        uint32_t sent = 0;
        int it = 0;
        for (int i = first; i < units && ok && rank == 0; i += step) {
            const Unit u = unit_at(plan, mt, slices, i);
            for (int s = u.s0; s < u.s1; ++s, ++sent) {
                const int in_run = (s - u.s0) % kRun, stage = (int)(sent % kStages);
                if (in_run == 0 && !__all_sync(0xFFFFFFFFu, mbar_wait(&ctl.acc_empty[it & 1], (uint32_t)(((it >> 1) & 1) ^ 1), abort_flag))) {
                    ok = false;
                    break;
                }
                if (!__all_sync(0xFFFFFFFFu, mbar_wait(&ctl.full[stage], (sent / kStages) & 1u, abort_flag))) {
                    ok = false;
                    break;
                }
                tc_fence_after_sync();
                const bool end = in_run == kRun - 1 || s == u.s1 - 1;
                if (elect_one()) {
                    const uint32_t d = tmem + (uint32_t)((it & 1) * kAcc);
                    // the address is the descriptor's low field, in units of 16 bytes
                    const uint64_t at = (uint64_t)(uint32_t)(stage * (kStage >> 4));
#pragma unroll
                    for (int k = 0; k < kSlice / 16; ++k) {
                        const auto ad = [&](int t) { return a_desc + at + (uint64_t)(t * (kPlaneA >> 4) + (A_ACROSS ? k * 128 : k * 2)); };
                        const auto bd = [&](int t) { return b_desc + at + (uint64_t)(t * (kPlaneB >> 4) + (B_ACROSS ? k * 128 : k * 2)); };
                        const bool more = (in_run | k) != 0;
                        mma<2>(d, ad(0), bd(0), idesc, more);
                        mma<2>(d + kBN, ad(0), bd(2), idesc, more);
                        mma<2>(d + kBN, ad(2), bd(0), idesc, true);
                        mma<2>(d + kBN, ad(1), bd(1), idesc, true);
                        mma<2>(d + kBN, ad(0), bd(1), idesc, true);
                        mma<2>(d + kBN, ad(1), bd(0), idesc, true);
                    }
                    commit<2>(&ctl.empty[stage]);
                    if (end) commit<2>(&ctl.acc_full[it & 1]);
                }
                __syncwarp();
                if (end) ++it;
            }
        }
        if (rank == 0) {
            if (elect_one()) commit<2>(&ctl.drain);
            __syncwarp();
        }
        // both CTAs' memory is read until the last product is done
        const long long t0 = clock64();
        while (!mbar_try_wait(&ctl.drain, 0) && clock64() - t0 < kWaitCycles) {
        }
    } else if (warp >= 4) {
        // ---- epilogue: a warp has 32 rows and 64 columns
        const int quad = warp & 3, half = (warp - 4) >> 2;
        float* mine = stage_f + (warp - 4) * 32 * 32;
        const int sub = lane & 7;
        int it = 0;
        for (int i = first; i < units && ok; i += step) {
            const Unit u = unit_at(plan, mt, slices, i);
            float sum[64];
#pragma unroll
            for (int e = 0; e < 64; ++e) sum[e] = 0.0f;
            for (int s = u.s0; s < u.s1; s += kRun, ++it) {
                if (!__all_sync(0xFFFFFFFFu, mbar_wait(&ctl.acc_full[it & 1], (uint32_t)((it >> 1) & 1), abort_flag))) {
                    ok = false;
                    break;
                }
                tc_fence_after_sync();
                const uint32_t at = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)((it & 1) * kAcc + half * 64);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t v[16], w[16];
                    tmem_ld_16cols(at + (uint32_t)(c * 16), v);
                    tmem_ld_16cols(at + (uint32_t)(kBN + c * 16), w);
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 16; ++e) sum[c * 16 + e] += __uint_as_float(v[e]) + __uint_as_float(w[e]);
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive_at(of_rank(&ctl.acc_empty[it & 1], 0));
            }
            if (!ok) break;
            const int64_t row0 = ((int64_t)u.m * 2 + rank) * kM + quad * 32, col = (int64_t)u.n * kBN + half * 64 + sub * 4;
            float* part = u.part >= 0 ? plan.parts + (((int64_t)u.part * 2 + rank) * kM + quad * 32) * kBN + half * 64 : nullptr;
            constexpr float none[4] = {};                        // these products have no bias
            finish_chunk<float, 0, kBN>(p, part, mine, sum, none, row0, m_end, col, vec);
            finish_chunk<float, 1, kBN>(p, part ? part + 32 : nullptr, mine, sum, none, row0, m_end, col + 32, vec);
        }
    }
    if (!ok) {
        *abort_flag = 1;
        if (lane == 0) latch(p.ctl, AA_ERR_SCAN_TIMEOUT);
    }
    tc_fence_before_sync();
    __syncthreads();
    cluster_sync_all();                      // nothing of the other CTA is on its way here any more
    tc_fence_after_sync();
    if (warp == 2) dealloc<2>(tmem, 2 * kAcc);
}

template <bool AA, bool BA>
aa_status launch_planes(aa_ctx_impl* c, const ProductParams& in) {
    ProductParams p = in;
    alignas(64) CUtensorMap map_a, map_b;
    const int64_t a_rows = AA ? p.k : p.m, a_cols = AA ? p.m : p.k, b_rows = BA ? p.k : p.n, b_cols = BA ? p.n : p.k;
    if (!encode_bf16_planes_map(&map_a, p.a.data, kTerms, a_rows, a_cols, p.a.stride, p.plane_a, AA ? kSlice : kM) ||
        !encode_bf16_planes_map(&map_b, p.b.data, kTerms, b_rows, b_cols, p.b.stride, p.plane_b, BA ? kSlice : kHalfB))
        return AA_ERR_CUDA;
    const int64_t mt = (p.m + 2 * kM - 1) / (2 * kM), nt = (p.n + kBN - 1) / kBN, tiles = mt * nt;
    if (tiles > 0x3FFFFFF) return AA_ERR_UNSUPPORTED;
    const void* kernel = (const void*)product_planes_kernel<AA, BA>;
    if (allow_smem(c, kernel, kPlaneSmem) != AA_OK) return AA_ERR_CUDA;
    const int teams = resident_clusters(c, kernel, kPlaneThreads, kPlaneSmem, 2);
    if (teams < 1) return AA_ERR_CUDA;
    Plan plan = make_plan(p, tiles, (int)nt, teams, 2 * kM * kBN, 2 * kM, 1.2, 1);
    const int64_t tail = tiles - plan.whole, units = plan.whole + tail * plan.splits;
    bool vec = true;
    for (const MatArg* m : {&p.out, &p.residual}) vec = vec && (!m->data || ((uintptr_t)m->data % 16 == 0 && m->stride % 4 == 0));
    void* args[] = {&map_a, &map_b, &p, &plan, &vec};
    if (launch_clusters(c, kernel, (unsigned)((units < teams ? units : teams) * 2), kPlaneThreads, args, kPlaneSmem, 2) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    if (tail == 0) return AA_OK;
    void* join[] = {&p, &plan, &vec};
    if (launch_overlapped(c, (const void*)product_join_kernel<float, 2 * kM, kBN>, dim3((unsigned)(tail * 2 * kM * kBN / 4 / 256)), dim3(256), join, 0, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

}  // namespace

aa_status launch_product_planes(aa_ctx_impl* c, const ProductParams& p) { return p.a_across ? launch_planes<true, true>(c, p) : launch_planes<false, true>(c, p); }

}  // namespace aa
