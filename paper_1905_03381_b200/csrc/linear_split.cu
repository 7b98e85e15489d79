// Products of linear layers on the tensor cores for operands that TMA cannot feed to them: fp32, and bf16 rows that start at any alignment.
//
// The matrix unit takes bf16 factors.  An fp32 number is the sum of three of them, x = h + m + l with h = bf16(x), m = bf16(x - h), l = bf16(x - h - m): 24 bits in
// all, each difference exact.  Of the nine products of two numbers the six largest are summed - h h', h m', m h', m m', h l', l h' - the others are
// below 2^-22 of the product.  h h' has an accumulator of its own in TMEM, so that the large sum is rounded once for 16 terms.  The matrix unit rounds
// towards zero there (one part in 2^24 a step of 16 terms, all in one direction: 1.4e-5 of a sum of 4,096 positive terms), so that every 256 terms
// the accumulators go to registers, where the runs are added with ordinary rounding.
// Six products of bf16 at 1.6 PFLOP/s are 0.27 PFLOP/s of fp32, against 0.07 of the ordinary lanes.
//
// A persistent CTA takes 128 x 128 tiles.  Eight warps fetch 64-wide slices with ordinary loads a slice ahead, take them apart and store the terms in the
// layout that TMA would have left (128-byte swizzle); elements out of range are zeros, so strides, alignment and counted rows need nothing
// else.  The first of them issues a slice's products, a quarter at a time between the batches of the next one that it stores; eight other warps add
// the runs up and finish a tile, as in the kernel for bf16.
// 2,048 x 4,096 -> 2,048 fp32 takes 361 us, 95 TFLOP/s (a library's plain fp32 product: 56).  A slice takes about 5,000 cycles: 1,540 of products, and
// 64 KB that come through registers and shared memory (96 KB written there, 196 KB read by the products).  A tile's way out takes 6,000 cycles, which
// bounds short contractions (1,000 x 65 -> 1,000: 20 us from a flushed L2, the library's product without bias 13).
#include <type_traits>

#include "linear_plan.cuh"
#include "tensor_core.cuh"

namespace aa {

namespace {

constexpr int kTile = 128, kStages = 2;
constexpr int kLoaders = 8, kEpilogue = 8;
constexpr int kSplitThreads = 512;       // warps 0..7 load (the first of them issues, too), 8..15 finish: 128 registers a thread
constexpr int kRun = 4;                  // slices summed in TMEM
constexpr int kParts = kSlice / 16;      // steps of the matrix unit a slice
constexpr int kTermBytes = kTile * 128;

template <int TERMS>
struct Split {
    static constexpr int OPERAND = TERMS * kTermBytes, STAGE = 2 * OPERAND;
    static constexpr int ACC = TERMS == 1 ? kTile : 2 * kTile, TMEM = 2 * ACC;
    static constexpr size_t SMEM = 1024 + (size_t)kStages * STAGE + kEpilogue * 32 * 32 * sizeof(float);
};

struct SplitCtl {
    uint64_t full[kStages], empty[kStages], acc_full[2], acc_empty[2], drain;
    uint32_t tmem;
    int abort_flag;
};

// Stored rows and columns of an operand that count.
struct Box {
    const void* data;
    int64_t stride, rows, cols;
};

// The 16 numbers a lane fetches of a batch of 8 rows of 64 elements, as they lie in memory: runs of RUN elements at column RUN (l % LANES) of rows l / LANES, l / LANES + 32 /
// LANES, ...  VEC (16-byte aligned base and rows, columns in eights): a run is 16 bytes; otherwise it is two elements.  Neighbouring lanes read neighbouring runs.
// Nothing touches what the loads bring before it is stored, so that they stay under way.  Where an element does not count a stand-in is loaded (there is a
// row and a column at least); `in` says which numbers count.
template <typename T, bool VEC>
struct Batch {
    using Word = typename std::conditional<VEC, uint4, T>::type;
    static constexpr int RUN = VEC ? 16 / (int)sizeof(T) : 2, LANES = 64 / RUN, RUNS = 16 / RUN, ROWS = 32 / LANES;   // ROWS: between a lane's runs
    static constexpr int PER = VEC ? 1 : RUN;
    Word w[RUNS * PER];
    uint32_t in;

    __device__ __forceinline__ void load(const Box& b, int64_t row0, int64_t col0) {
        const int lane = threadIdx.x & 31;
        const int64_t col = col0 + (lane % LANES) * RUN;
        if constexpr (VEC) {
            asm volatile("" : "+l"(row0));   // the addresses are worked out here, not held in registers from slice to slice
            in = 0;
#pragma unroll
            for (int h = 0; h < RUNS; ++h) {
                const int64_t row = row0 + lane / LANES + ROWS * h;
                w[h] = *reinterpret_cast<const Word*>(static_cast<const T*>(b.data) + min(row, b.rows - 1) * b.stride + (col < b.cols ? col : 0));
                if (row < b.rows && col < b.cols) in |= ((1u << RUN) - 1) << (h * RUN);
            }
        } else if (row0 + 8 <= b.rows && col0 + 64 <= b.cols) {
            const T* at = static_cast<const T*>(b.data) + (row0 + lane / LANES) * b.stride + col;
            in = 0xFFFFu;
#pragma unroll
            for (int h = 0; h < RUNS; ++h) {
                w[2 * h] = at[0];
                w[2 * h + 1] = at[1];
                at += ROWS * b.stride;
            }
        } else {
            in = 0;
#pragma unroll
            for (int h = 0; h < RUNS; ++h) {
                const int64_t row = row0 + lane / LANES + ROWS * h;
                const T* at = static_cast<const T*>(b.data) + min(row, b.rows - 1) * b.stride;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    w[2 * h + e] = at[col + e < b.cols ? col + e : 0];
                    if (row < b.rows && col + e < b.cols) in |= 1u << (2 * h + e);
                }
            }
        }
    }
    __device__ __forceinline__ void values(float (&x)[16]) const {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            if constexpr (VEC && sizeof(T) == 4) x[e] = __uint_as_float((&w[e / 4].x)[e % 4]);
            else if constexpr (VEC) x[e] = e % 2 ? bf16_hi((&w[e / 8].x)[e / 2 % 4]) : bf16_lo((&w[e / 8].x)[e / 2 % 4]);
            else if constexpr (sizeof(T) == 4) x[e] = w[e];
            else x[e] = __uint_as_float((uint32_t)w[e] << 16);
        }
        if (!__all_sync(0xFFFFFFFFu, in == 0xFFFFu)) {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = (in >> e) & 1u ? x[e] : 0.0f;
        }
    }
};

// Two numbers' terms, packed.
template <int TERMS>
__device__ __forceinline__ void take_apart(float a, float b, uint32_t (&t)[TERMS]) {
    t[0] = pack_bf16(a, b);
    if constexpr (TERMS == 3) {
        a -= bf16_lo(t[0]);
        b -= bf16_hi(t[0]);
        t[1] = pack_bf16(a, b);
        a -= bf16_lo(t[1]);
        b -= bf16_hi(t[1]);
        t[2] = pack_bf16(a, b);
    }
}

// The batch into rows r0 .. r0 + 7 of a [rows x 128 bytes] swizzled block; r0 a multiple of 8.
template <typename T, int TERMS, bool VEC>
__device__ __forceinline__ void store_batch(unsigned char* block, int r0, const float (&x)[16]) {
    using B = Batch<T, VEC>;
    const int lane = threadIdx.x & 31, byte = (lane % B::LANES) * B::RUN * 2;        // of the row's 128
#pragma unroll
    for (int h = 0; h < B::RUNS; ++h) {
        const int r = lane / B::LANES + B::ROWS * h;
        uint32_t t[B::RUN / 2][TERMS];
#pragma unroll
        for (int q = 0; q < B::RUN / 2; ++q) take_apart<TERMS>(x[h * B::RUN + 2 * q], x[h * B::RUN + 2 * q + 1], t[q]);
        unsigned char* to = block + (r0 + r) * 128 + (((byte >> 4) ^ r) << 4) + (byte & 15);
#pragma unroll
        for (int k = 0; k < TERMS; ++k) {
            if constexpr (B::RUN == 8) *reinterpret_cast<uint4*>(to + k * kTermBytes) = make_uint4(t[0][k], t[1][k], t[2][k], t[3][k]);
            else if constexpr (B::RUN == 4) *reinterpret_cast<uint2*>(to + k * kTermBytes) = make_uint2(t[0][k], t[1][k]);
            else *reinterpret_cast<uint32_t*>(to + k * kTermBytes) = t[0][k];
        }
    }
}

template <typename T, int TERMS, bool VEC, bool A_ACROSS, bool B_ACROSS>
__global__ void __launch_bounds__(kSplitThreads, 1) product_split_kernel(const __grid_constant__ ProductParams p, const __grid_constant__ Plan plan, bool out_vec) {
    using S = Split<TERMS>;
    extern __shared__ unsigned char smem_raw[];
    __shared__ SplitCtl ctl;
    unsigned char* ring = reinterpret_cast<unsigned char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    float* stage_f = reinterpret_cast<float*>(ring + (size_t)kStages * S::STAGE);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* abort_flag = &ctl.abort_flag;
    Unit last = {};                      // of a cluster: the tile, and whether there is one
    bool has = false;
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(&ctl.full[s], kLoaders);
            mbar_init(&ctl.empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(&ctl.acc_full[b], 1);
            mbar_init(&ctl.acc_empty[b], kEpilogue);
        }
        mbar_init(&ctl.drain, 1);
        ctl.abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 8) tmem_alloc(&ctl.tmem, S::TMEM);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *(volatile uint32_t*)&ctl.tmem;
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t live = live_rows(p.live, p.ctl, blockIdx.x == 0 && threadIdx.x == 0);
    const int64_t m_end = p.live_k ? p.m : min(p.m, live), k_end = p.live_k ? min(p.k, live) : p.k;
    const int mt = (int)((m_end + kTile - 1) / kTile), units = units_of(plan, mt), slices = (int)((k_end + kSlice - 1) / kSlice);
    bool ok = true;
    if (warp < kLoaders) {
        // ---- loaders: a slice is 16 batches of 8 rows of each operand, two a warp; the next batch is under way while this one is stored
        const Box a{p.a.data, p.a.stride, A_ACROSS ? k_end : m_end, A_ACROSS ? m_end : k_end}, b{p.b.data, p.b.stride, B_ACROSS ? k_end : p.n, B_ACROSS ? p.n : k_end};
        int i = blockIdx.x, s = 0;
        Unit u = {};
        // the first slice from here on, over the units without one
        const auto settle = [&]() {
            for (; i < units; i += gridDim.x) {
                const Unit next = unit_at(plan, mt, slices, i);
                if (next.s0 == next.s1) continue;
                u = next;
                s = next.s0;
                return;
            }
        };
        const auto fetch = [&](int q, Batch<T, VEC>& x) {
            const int batch = warp * 2 + (q & 1);
            const bool of_a = q < 2, across = of_a ? A_ACROSS : B_ACROSS;
            const int64_t tile0 = (int64_t)(of_a ? u.m : u.n) * kTile;
            // across: the first 64 rows of the block are tokens against columns 0..63 of the tile, the others against 64..127
            const int64_t row = across ? (int64_t)s * kSlice + (batch & 7) * 8 : tile0 + batch * 8, col = across ? tile0 + (batch >> 3) * 64 : (int64_t)s * kSlice;
            x.load(of_a ? a : b, row, col);
        };
        // a quarter of the products of slice number `issued` of this CTA, by the first warp
        constexpr uint32_t idesc = umma_idesc_bf16(kTile, kTile, A_ACROSS, B_ACROSS);
        const uint64_t a_desc = umma_smem_desc(smem_u32(ring), A_ACROSS ? 8192 : 16, 1024), b_desc = umma_smem_desc(smem_u32(ring) + S::OPERAND, B_ACROSS ? 8192 : 16, 1024);
        uint32_t issued = 0;
        int in_run = 0, it = 0, of = blockIdx.x, togo = 0;
        bool last = false;
        const auto issue = [&](int k) -> bool {
            const int stage = (int)(issued % kStages);
            if (k == 0) {
                while (togo == 0) {
                    const Unit v = unit_at(plan, mt, slices, of);
                    of += gridDim.x;
                    togo = v.s1 - v.s0;
                }
                if (in_run == 0 && !__all_sync(0xFFFFFFFFu, mbar_wait(&ctl.acc_empty[it & 1], (uint32_t)(((it >> 1) & 1) ^ 1), abort_flag))) return false;
                if (!__all_sync(0xFFFFFFFFu, mbar_wait(&ctl.full[stage], (issued / kStages) & 1u, abort_flag))) return false;
                tc_fence_after_sync();
                last = in_run == kRun - 1 || togo == 1;
            }
            if (elect_one()) {
                const uint32_t d = tmem + (uint32_t)((it & 1) * S::ACC);
                // the address is the descriptor's low field, in units of 16 bytes
                const uint64_t at = (uint64_t)(uint32_t)(stage * (S::STAGE >> 4));
                const auto ad = [&](int t) { return a_desc + at + (uint64_t)(t * (kTermBytes >> 4) + (A_ACROSS ? k * 128 : k * 2)); };
                const auto bd = [&](int t) { return b_desc + at + (uint64_t)(t * (kTermBytes >> 4) + (B_ACROSS ? k * 128 : k * 2)); };
                const bool more = (in_run | k) != 0;
                umma_bf16(d, ad(0), bd(0), idesc, more);
                if (TERMS == 3) {
                    umma_bf16(d + kTile, ad(0), bd(2), idesc, more);
                    umma_bf16(d + kTile, ad(2), bd(0), idesc, true);
                    umma_bf16(d + kTile, ad(1), bd(1), idesc, true);
                    umma_bf16(d + kTile, ad(0), bd(1), idesc, true);
                    umma_bf16(d + kTile, ad(1), bd(0), idesc, true);
                }
                if (k == kParts - 1) umma_commit(&ctl.empty[stage]);
                if (k == kParts - 1 && last) umma_commit(&ctl.acc_full[it & 1]);
            }
            __syncwarp();
            if (k == kParts - 1) {
                ++issued;
                --togo;
                in_run = last ? 0 : in_run + 1;
                if (last) ++it;
            }
            return true;
        };
        Batch<T, VEC> x[4];
        uint32_t sent = 0;
        settle();
        if (i < units)
#pragma unroll
            for (int q = 0; q < 4; ++q) fetch(q, x[q]);
        while (i < units && ok) {
            const int stage = (int)(sent % kStages);
            if (!__all_sync(0xFFFFFFFFu, mbar_wait(&ctl.empty[stage], ((sent / kStages) & 1u) ^ 1u, abort_flag))) {
                ok = false;
                break;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (warp == 0 && sent > 0 && ok) ok = issue(q);
                unsigned char* block = ring + (size_t)stage * S::STAGE + (q < 2 ? 0 : S::OPERAND);
                float v[16];
                x[q].values(v);
                store_batch<T, TERMS, VEC>(block, (warp * 2 + (q & 1)) * 8, v);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.full[stage]);
            ++sent;
            // only now the next slice's loads: the fence waits for every load under way.  The last slice of all is fetched once more and not stored, rather than
            // have the loads behind a branch.
            if (++s >= u.s1) {
                i += gridDim.x;
                settle();
                if (i >= units) --s;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) fetch(q, x[q]);
        }
        if (warp == 0) {
            if (sent > 0)
#pragma unroll
                for (int q = 0; q < kParts; ++q)
                    if (ok) ok = issue(q);
            if (elect_one()) umma_commit(&ctl.drain);
            __syncwarp();
            const long long t0 = clock64();
            while (!mbar_try_wait(&ctl.drain, 0) && clock64() - t0 < kWaitCycles) {
            }
        }
    } else {
        // ---- epilogue: a warp has 32 rows and 64 columns
        const int quad = warp & 3, half = (warp - 8) >> 2;
        float* mine = stage_f + (warp - 8) * 32 * 32;
        const int sub = lane & 7;
        int it = 0;
        for (int i = blockIdx.x; i < units && ok; i += gridDim.x) {
            const Unit u = unit_at(plan, mt, slices, i);
            float sum[64], bias[2][4];
#pragma unroll
            for (int e = 0; e < 64; ++e) sum[e] = 0.0f;
#pragma unroll
            for (int c = 0; c < 2; ++c) load_bias(p, (int64_t)u.n * kTile + half * 64 + c * 32 + sub * 4, bias[c]);
            for (int s = u.s0; s < u.s1; s += kRun, ++it) {
                if (!__all_sync(0xFFFFFFFFu, mbar_wait(&ctl.acc_full[it & 1], (uint32_t)((it >> 1) & 1), abort_flag))) {
                    ok = false;
                    break;
                }
                tc_fence_after_sync();
                const uint32_t at = tmem + ((uint32_t)(quad * 32) << 16) + (uint32_t)((it & 1) * S::ACC + half * 64);
#pragma unroll
                for (int t = 0; t < (TERMS == 3 ? 2 : 1); ++t)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint32_t v[16];
                        tmem_ld_16cols(at + (uint32_t)(t * kTile + c * 16), v);
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 16; ++e) sum[c * 16 + e] += __uint_as_float(v[e]);
                    }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl.acc_empty[it & 1]);
            }
            if (!ok) break;
            if (plan.cluster > 1) {
                // every CTA of the cluster is through with its ring: its shared memory takes the parts of 128 / cluster rows
                last = u;
                has = true;
                cluster_sync_all();
                const int rows = kTile / plan.cluster, r = quad * 32 + lane;
                const uint32_t to = of_rank(ring, (uint32_t)(r / rows)) + (uint32_t)((((int)cluster_rank() * rows + r % rows) * kTile + half * 64) * 4);
#pragma unroll
                for (int e = 0; e < 64; e += 4) store_remote(to + (uint32_t)(e * 4), make_float4(sum[e], sum[e + 1], sum[e + 2], sum[e + 3]));
                break;
            }
            const int64_t row0 = (int64_t)u.m * kTile + quad * 32, col = (int64_t)u.n * kTile + half * 64 + sub * 4;
            float* part = u.part >= 0 ? plan.parts + ((int64_t)u.part * kTile + quad * 32) * kTile + half * 64 : nullptr;
            finish_chunk<T, 0, kTile>(p, part, mine, sum, bias[0], row0, m_end, col, out_vec);
            finish_chunk<T, 1, kTile>(p, part ? part + 32 : nullptr, mine, sum, bias[1], row0, m_end, col + 32, out_vec);
        }
    }
    if (plan.cluster > 1) {
        // once before the parts are sent (the senders have done it) and once after
        if (!has) cluster_sync_all();
        cluster_sync_all();
        if (has) finish_cluster<T, kTile>(p, plan, last, reinterpret_cast<const float*>(ring), m_end, out_vec, (int)threadIdx.x - kLoaders * 32, kEpilogue * 32);
    }
    if (!ok) {
        *abort_flag = 1;
        if (lane == 0) latch(p.ctl, AA_ERR_SCAN_TIMEOUT);
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == 8) tmem_dealloc(tmem, S::TMEM);
}

template <typename T, int TERMS, bool VEC>
aa_status launch_split(aa_ctx_impl* c, const ProductParams& in, bool out_vec) {
    ProductParams p = in;
    const int64_t mt = (p.m + kTile - 1) / kTile, nt = (p.n + kTile - 1) / kTile, tiles = mt * nt;
    if (tiles > 0x3FFFFFF) return AA_ERR_UNSUPPORTED;
    const void* kernel = p.a_across ? (const void*)product_split_kernel<T, TERMS, VEC, true, true>
                                    : (p.b_across ? (const void*)product_split_kernel<T, TERMS, VEC, false, true> : (const void*)product_split_kernel<T, TERMS, VEC, false, false>);
    if (allow_smem(c, kernel, Split<TERMS>::SMEM) != AA_OK) return AA_ERR_CUDA;
    const int cluster = tile_cluster(c, kernel, kSplitThreads, Split<TERMS>::SMEM, p, tiles);
    Plan plan = make_plan(p, tiles, (int)nt, c->sm_count, kTile * kTile, kTile, TERMS == 3 ? 2.6 : 1.5, cluster);
    const int64_t tail = tiles - plan.whole, units = plan.whole + tail * plan.splits;
    void* args[] = {&p, &plan, &out_vec};
    const unsigned grid = (unsigned)(units < c->sm_count || plan.cluster > 1 ? units : c->sm_count);
    if (launch_clusters(c, kernel, grid, kSplitThreads, args, Split<TERMS>::SMEM, plan.cluster) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    if (tail == 0 || plan.cluster > 1) return AA_OK;
    void* join[] = {&p, &plan, &out_vec};
    if (launch_overlapped(c, (const void*)product_join_kernel<T, kTile, kTile>, dim3((unsigned)(tail * kTile * kTile / 4 / 256)), dim3(256), join, 0, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

}  // namespace

aa_status launch_product_split(aa_ctx_impl* c, const ProductParams& p, int dtype) {
    const int64_t es = dtype == AA_BF16 ? 2 : 4;
    const auto lies = [&](const MatArg& a, int64_t bytes) { return !a.data || ((uintptr_t)a.data % bytes == 0 && a.stride * es % bytes == 0); };
    const bool vec = lies(p.a, 16) && lies(p.b, 16) && (p.a_across ? p.m : p.k) % 8 == 0 && (p.b_across ? p.n : p.k) % 8 == 0;
    const bool out_vec = lies(p.out, 4 * es) && lies(p.pre, 4 * es) && lies(p.residual, 4 * es);
    if (dtype == AA_BF16) return vec ? launch_split<uint16_t, 1, true>(c, p, out_vec) : launch_split<uint16_t, 1, false>(c, p, out_vec);
    return vec ? launch_split<float, 3, true>(c, p, out_vec) : launch_split<float, 3, false>(c, p, out_vec);
}

}  // namespace aa
