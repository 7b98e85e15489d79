// Forward pass of the bf16 attention with a relative position bias for long sequences, on the 5th-generation tensor cores.
//
// A CTA owns two tiles of 128 query rows of one head and streams 64-key tiles of K and V.  One warp issues every product; two warpgroups, one
// per query tile, turn scores into probabilities: while one works on its tile the products of the other run.  Per key tile and query tile:
// 4 D x 8192 flops on the tensor cores (512 cycles at D = 128) against 8192 exponentials (512 cycles of the special function units) and
// about eight instructions each.  The accumulated output stays in TMEM and is rescaled only when a row's maximum grew by more than 2^8 since
// its reference: until then probabilities are up to 256, which costs bf16 no accuracy, and sums stay in fp32.
// Two causal documents of 4,096 tokens, 16 heads of 128 on 4 key heads: 0.35 ms, 0.39 PFLOP/s of unmasked products; bound by the
// latency of the turn a score tile takes (product, a thread's 64 scores, product): tensor pipe 18 %, issue slots 23 % in use.  (On the warp-level instructions: 1.15 ms.)
#include "rel_attention_tc.cuh"

namespace aa {

namespace {

constexpr int kKvStages = 3;
constexpr int kFwdThreads = 352;         // 8 softmax warps, the issuing warp, 2 loading warps

struct FwdCtl {
    uint64_t q_full, kv_full[kKvStages], kv_empty[kKvStages], s_full[2], p_full[2], o_full[2], drain;
    uint32_t tmem;
    int abort_flag;
};

template <int DT>
struct FwdGeo {
    static constexpr int Q = 128 * DT * 2, KV = kTcKeys * DT * 2, P = 128 * 128;
    static size_t smem(int reach, bool bias) { return 1024 + 2 * Q + kKvStages * 2 * KV + 2 * P + (bias ? bias_floats(reach, kTcMargin) * sizeof(float) : 0); }
};

template <int DT>
__global__ void __launch_bounds__(kFwdThreads, 1) forward_tc_kernel(RelParams p, int lo, int tiles) {
    using G = FwdGeo<DT>;
    extern __shared__ char smem_raw[];
    __shared__ FwdCtl ctl;
    char* Qs = reinterpret_cast<char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);     // two tiles
    char* KV = Qs + 2 * G::Q;                                                                // [stage][K, V]
    char* Ps = KV + kKvStages * 2 * G::KV;                                                   // two tiles
    float* bias = reinterpret_cast<float*>(Ps + 2 * G::P);
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t sn = blockIdx.x / tiles;
    // later rows of a causal sequence see more keys: the longest first
    const int i0 = (tiles - 1 - (int)(blockIdx.x % tiles)) * 256, h = blockIdx.y, hk = h / p.group;
    Seq s;
    if (!load_seq(p, sn, s) || max(s.lq, s.lk) <= lo || i0 >= s.lq) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    volatile int* abort_flag = &ctl.abort_flag;
    if (threadIdx.x == 0) {
        mbar_init(&ctl.q_full, 64);
        for (int i = 0; i < kKvStages; ++i) {
            mbar_init(&ctl.kv_full[i], 64);
            mbar_init(&ctl.kv_empty[i], 1);
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(&ctl.s_full[t], 1);
            mbar_init(&ctl.p_full[t], 4);
            mbar_init(&ctl.o_full[t], 1);
        }
        mbar_init(&ctl.drain, 1);
        ctl.abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 8) tmem_alloc(&ctl.tmem, kTcTmem);
    fill_bias<kTcMargin>(p, h, bias);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *(volatile uint32_t*)&ctl.tmem;
    // key tiles that each query tile sees
    int n_tiles[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) n_tiles[t] = i0 + 128 * t < s.lq ? (keys_seen(p, s, min(i0 + 128 * t + 128, s.lq)) + kTcKeys - 1) / kTcKeys : 0;
    const int n = max(n_tiles[0], n_tiles[1]);
    const uint32_t qS = smem_u32(Qs), kvS = smem_u32(KV), pS = smem_u32(Ps);
    bool ok = true;
    if (warp >= 9) {
        // ---- loading warps
        const int tid = threadIdx.x - 288;
        for (int t = 0; t < 2; ++t)
            if (n_tiles[t] > 0) load_swizzled<128, DT, 64>(p, p.q, h, s.q0 + i0 + 128 * t, min(128, s.lq - i0 - 128 * t), qS + t * G::Q, tid);
        cp_async_commit();
        for (int i = 0; i <= n && ok; ++i) {
            if (i < n) {
                const int st = i % kKvStages;
                if (i >= kKvStages && !mbar_wait(&ctl.kv_empty[st], (uint32_t)((i / kKvStages - 1) & 1), abort_flag)) {
                    ok = false;
                    break;
                }
                load_swizzled<kTcKeys, DT, 64>(p, p.k, hk, s.k0 + i * kTcKeys, min(kTcKeys, s.lk - i * kTcKeys), kvS + st * 2 * G::KV, tid);
                load_swizzled<kTcKeys, DT, 64>(p, p.v, hk, s.k0 + i * kTcKeys, min(kTcKeys, s.lk - i * kTcKeys), kvS + (st * 2 + 1) * G::KV, tid);
            }
            cp_async_commit();
            cp_async_wait<1>();            // all but the newest group: the tile before this one (at first the queries)
            fence_async_shared();
            if (i == 0) mbar_arrive(&ctl.q_full);
            else mbar_arrive(&ctl.kv_full[(i - 1) % kKvStages]);
        }
        cp_async_wait<0>();
    } else if (warp == 8) {
        // ---- issuing warp
        constexpr uint32_t idesc_pv = umma_idesc_bf16(128, DT, false, true);
        const auto scores = [&](int t, int i) {
            if (lane == 0) {
                mma_rows<DT, 128, kTcKeys>(p, tmem + (uint32_t)(t * 256), qS + t * G::Q, kvS + (i % kKvStages) * 2 * G::KV);
                umma_commit(&ctl.s_full[t]);
            }
            __syncwarp();
        };
        if (n > 0) ok = mbar_wait(&ctl.q_full, 0, abort_flag) && mbar_wait(&ctl.kv_full[0], 0, abort_flag);
        if (n > 0 && ok) {
            tc_fence_after_sync();
            for (int t = 0; t < 2; ++t)
                if (n_tiles[t] > 0) scores(t, 0);
        }
        for (int i = 0; i < n && ok; ++i) {
            if (i + 1 < n && !mbar_wait(&ctl.kv_full[(i + 1) % kKvStages], (uint32_t)(((i + 1) / kKvStages) & 1), abort_flag)) {
                ok = false;
                break;
            }
            for (int t = 0; t < 2; ++t) {
                if (i >= n_tiles[t]) continue;
                if (!mbar_wait(&ctl.p_full[t], (uint32_t)(i & 1), abort_flag)) {
                    ok = false;
                    break;
                }
                tc_fence_after_sync();
                if (lane == 0) {
                    const uint32_t a = pS + t * G::P, b = kvS + ((i % kKvStages) * 2 + 1) * G::KV;
#pragma unroll
                    for (int k = 0; k < kTcKeys / 16; ++k)
                        umma_bf16(tmem + (uint32_t)(t * 256 + 64), umma_smem_desc(a + k * 32, 16, 1024), umma_smem_desc(b + k * 2048, kTcKeys * 128, 1024), idesc_pv, (i | k) != 0);
                    if (i + 1 == n_tiles[t]) umma_commit(&ctl.o_full[t]);
                }
                __syncwarp();
                if (i + 1 < n_tiles[t]) scores(t, i + 1);
            }
            if (lane == 0) umma_commit(&ctl.kv_empty[i % kKvStages]);
            __syncwarp();
        }
        if (lane == 0) umma_commit(&ctl.drain);
        __syncwarp();
        const long long t0 = clock64();
        while (!mbar_try_wait(&ctl.drain, 0) && clock64() - t0 < kWaitCycles) {
        }
    } else {
        // ---- softmax warpgroups
        const int t = warp >> 2, r = threadIdx.x & 127, w0 = i0 + 128 * t + (warp & 3) * 32, i = i0 + 128 * t + r;
        const uint32_t row = tmem + ((uint32_t)((warp & 3) * 32) << 16) + (uint32_t)(t * 256);
        const uint2 key = p.drop.thr ? instance_key(p.drop, sn) : make_uint2(0, 0);
        float m = -INFINITY, l = 0.0f;
        for (int k = 0; k < n_tiles[t]; ++k) {
            if (!mbar_wait(&ctl.s_full[t], (uint32_t)(k & 1), abort_flag)) ok = false;
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            tc_fence_after_sync();
            const int j0 = k * kTcKeys;
            float x[64];
            load_row(row, x);
            row_scores(p, s, bias, w0, i, j0, x);
            float top = x[0];
#pragma unroll
            for (int c = 1; c < 64; ++c) top = fmaxf(top, x[c]);
            // a new reference where the maximum has grown by more than 8; the products before this tile are complete (its scores came after)
            const bool grow = k == 0 ? true : top > m + 8.0f || (m == -INFINITY && top > -INFINITY);
            if (__any_sync(0xFFFFFFFFu, grow)) {
                const float next = grow ? fmaxf(m, top) : m, ref = next == -INFINITY ? 0.0f : next;
                const float corr = grow ? ex2_approx(m - ref) : 1.0f;
                l *= corr;
                m = next;
                if (k > 0) {
#pragma unroll
                    for (int c0 = 0; c0 < DT; c0 += 32) {
                        uint32_t v[32];
                        tmem_ld_32cols(row + 64 + c0, v);
                        tmem_ld_wait();
#pragma unroll
                        for (int c = 0; c < 32; ++c) v[c] = __float_as_uint(__uint_as_float(v[c]) * corr);
                        tmem_st_32cols(row + 64 + c0, v);
                    }
                    tmem_st_wait();
                }
            }
            const float ref = m == -INFINITY ? 0.0f : m;
            float a = 0.0f, b = 0.0f;
#pragma unroll
            for (int c = 0; c < 64; c += 2) {
                x[c] = ex2_approx(x[c] - ref);
                x[c + 1] = ex2_approx(x[c + 1] - ref);
                a += x[c];
                b += x[c + 1];
            }
            l += a + b;
            if (p.drop.thr) row_drops(p, s, key, h, i, j0, [&](int c, bool d) { x[c] = d ? 0.0f : x[c]; });
            store_row(Ps + t * G::P, r, x);
            fence_async_shared();
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.p_full[t]);
        }
        uint16_t* out = i < s.lq ? const_cast<uint16_t*>(static_cast<const uint16_t*>(p.out.data)) + (s.q0 + i) * p.out.tok + (int64_t)h * p.out.head : nullptr;
        if (n_tiles[t] > 0) {
            if (ok && !mbar_wait(&ctl.o_full[t], 0, abort_flag)) ok = false;
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (ok) {
                tc_fence_after_sync();
                store_accumulator<DT>(p, row + 64, out, l == 0.0f ? 0.0f : p.drop.scale / l);
            }
        } else if (out) {                  // rows that see no key
            for (int c = 0; c < p.dim; c += 8) *reinterpret_cast<uint4*>(out + c) = make_uint4(0, 0, 0, 0);
        }
    }
    if (!ok) {
        *abort_flag = 1;
        if (lane == 0) latch(p.ctl, AA_ERR_SCAN_TIMEOUT);
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == 8) tmem_dealloc(tmem, kTcTmem);
}

template <int DT>
aa_status forward(aa_ctx_impl* c, RelParams p, int lo) {
    const void* kernel = (const void*)forward_tc_kernel<DT>;
    const size_t smem = FwdGeo<DT>::smem(p.reach, p.table);
    if (allow_smem(c, kernel, smem) != AA_OK) return AA_ERR_CUDA;
    int tiles = (int)((p.max_q + 255) / 256);
    if (p.n_seq * tiles > 0x7FFFFFFFll) return AA_ERR_UNSUPPORTED;
    void* args[] = {&p, &lo, &tiles};
    if (launch_overlapped(c, kernel, dim3((unsigned)(p.n_seq * tiles), p.heads), dim3(kFwdThreads), args, smem, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

}  // namespace

aa_status launch_rel_attention_tc(aa_ctx_impl* c, const RelParams& p, int lo) { return p.dim <= 64 ? forward<64>(c, p, lo) : forward<128>(c, p, lo); }

}  // namespace aa
