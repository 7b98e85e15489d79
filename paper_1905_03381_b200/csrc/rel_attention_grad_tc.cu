// Backward pass of the bf16 attention with a relative position bias for long sequences, on the 5th-generation tensor cores.
//
// rows kernel: a CTA owns 128 query rows of one head and streams 64-key tiles twice: first the running maximum, sum and D = sum p dp, from
// unrounded probabilities (rounded ones would cost the fp32 bias gradient its digits), then dS, its diagonal sums and dQ.
// keys kernel: a CTA owns 64 keys of one key head and streams the 128-row query tiles of the heads that share it, with those statistics;
// dV^T and dK^T (head elements x keys) stay in TMEM, so that p and dS are right operands as the rows leave them.
//
// In both, one warp issues the products and two warpgroups take turns with the score tiles: one works on S and dP of a tile (a thread per query
// row) while the tensor cores make the other's.  ds = p (dp - D) and p are rounded to bf16 as operands of the products with K, Q and dO, whose
// results are bf16; the diagonal sums are taken before the rounding.
// Two causal documents of 4,096 tokens, 16 heads of 128 on 4 key heads: 2.1 ms both kernels (the warp-level instructions: 3.1 ms), bound by
// the latency of the turn a score tile takes: product, a thread's 64 scores, product; the tensor cores are busy for 13 to 15 % of it.
#include "rel_attention_tc.cuh"

namespace aa {

namespace {

constexpr int kGradThreads = 352;        // 8 warps with scores, the issuing warp, 2 loading warps
constexpr int kRowStages = 3;

// S and dP of a tile -> registers; TMEM columns `at` and `at + 64`.
__device__ __forceinline__ void load_pair(uint32_t at, float (&t)[64], float (&dp)[64]) {
    load_row(at, t);
    load_row(at + 64, dp);
}
// t: scores -> e = 2^(t - m) with the drop's sign, dp masked and scaled; returns the row's sums of e and e dp
__device__ __forceinline__ void row_exp(const RelParams& p, const Seq& s, uint2 key, int h, int i, int j0, float m, float (&t)[64], float (&dp)[64], float& sum, float& dsum) {
    float a = 0.0f, b = 0.0f;
#pragma unroll
    for (int c = 0; c < 64; c += 2) {
        t[c] = ex2_approx(t[c] - m);
        t[c + 1] = ex2_approx(t[c + 1] - m);
        a += t[c];
        b += t[c + 1];
    }
    sum = a + b;
    if (p.drop.thr)
        row_drops(p, s, key, h, i, j0, [&](int c, bool d) {
            dp[c] = d ? 0.0f : __fmul_rn(dp[c], p.drop.scale);
            t[c] = d ? -t[c] : t[c];
        });
    a = b = 0.0f;
#pragma unroll
    for (int c = 0; c < 64; c += 2) {
        a = fmaf(fabsf(t[c]), dp[c], a);
        b = fmaf(fabsf(t[c + 1]), dp[c + 1], b);
    }
    dsum = a + b;
}
__device__ __forceinline__ void row_ds(const RelParams& p, float rl, float D, float (&t)[64], float (&dp)[64]) {
    const float f = rl * p.drop.scale;
#pragma unroll
    for (int c = 0; c < 64; ++c) {
        dp[c] = fabsf(t[c]) * rl * (dp[c] - D);
        t[c] = fmaxf(t[c], 0.0f) * f;
    }
}

// ... and whether `ok` holds in all of them
__device__ __forceinline__ bool group_all(int id, int threads, bool ok) {
    int r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %1, 0;\n\tbarrier.red.and.pred q, %2, %3, p;\n\tselp.s32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"((int)ok), "r"(id), "r"(threads) : "memory");
    return r != 0;
}
__device__ __forceinline__ void group_barrier(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// ------------------------------------------------------------------------------------------------------------ rows kernel

struct RowsCtl {
    uint64_t q_full, q_empty, kv_full[kRowStages], kv_empty[kRowStages], s_full[2], s_free[2], ds_full[2], ds_empty[2], dq_full, dq_free, drain;
    uint32_t tmem;
    int abort_flag;
};

constexpr int kSkewRows = 4, kSkewCols = 67, kSkewPitch = 69;       // rows x 64 keys of a warp staged along their diagonals

template <int DT>
struct RowsTcGeo {
    static constexpr int Q = 128 * DT * 2, KV = kTcKeys * DT * 2, S = 128 * 128;
    static constexpr int kStat = 2 * 128 * 3, kStage = 8 * kSkewRows * kSkewPitch, kFar = 2 * 256;
    static size_t smem(int stages, int reach, bool bias, bool table) {
        size_t b = 1024 + 2 * Q + (size_t)stages * 2 * KV + 2 * S + sizeof(RowsCtl) + kStat * sizeof(float);
        if (bias) b += bias_floats(reach, kTcMargin) * sizeof(float);
        if (table) b += (kStage + 2 * 2 * reach + kFar) * sizeof(float);
        return b;
    }
};

// Item `k` of CTA b's walk over `items`: forth and back over the grid, so that long and short items pair up.
__device__ __forceinline__ int64_t snake(int64_t k) {
    const int64_t g = gridDim.x, b = blockIdx.x;
    return k * g + (k & 1 ? g - 1 - b : b);
}

template <int DT>
__global__ void __launch_bounds__(kGradThreads, 1) grad_rows_tc_kernel(RelParams p, int lo, int blocks, int part0, int stages) {
    using G = RowsTcGeo<DT>;
    extern __shared__ char smem_raw[];
    char* Qs = reinterpret_cast<char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);     // Q, dO
    char* KV = Qs + 2 * G::Q;                                                                // [stage][K, V]
    char* Ss = KV + stages * 2 * G::KV;                                                  // [group] dS
    RowsCtl& ctl = *reinterpret_cast<RowsCtl*>(Ss + 2 * G::S);
    float* stat = reinterpret_cast<float*>(&ctl + 1);                                        // [group][row] m, l, D
    const bool want_table = p.table && p.dtable;
    float* stage = stat + G::kStat;                                                          // [warp][8][pitch]
    float* bins = stage + (want_table ? G::kStage : 0);                                      // [group][2 reach], then [neg, pos][thread]
    float* far = bins + (want_table ? 2 * 2 * p.reach : 0);
    float* bias = far + (want_table ? G::kFar : 0);
    grid_dependency_wait();
    grid_dependency_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, h = blockIdx.y, hk = h / p.group;
    volatile int* abort_flag = &ctl.abort_flag;
    if (threadIdx.x == 0) {
        mbar_init(&ctl.q_full, 64);
        mbar_init(&ctl.q_empty, 1);
        for (int i = 0; i < stages; ++i) {
            mbar_init(&ctl.kv_full[i], 64);
            mbar_init(&ctl.kv_empty[i], 1);
        }
        for (int w = 0; w < 2; ++w) {
            mbar_init(&ctl.s_full[w], 1);
            mbar_init(&ctl.s_free[w], 4);
            mbar_init(&ctl.ds_full[w], 4);
            mbar_init(&ctl.ds_empty[w], 1);
        }
        mbar_init(&ctl.dq_full, 1);
        mbar_init(&ctl.dq_free, 8);
        mbar_init(&ctl.drain, 1);
        ctl.abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 8) tmem_alloc(&ctl.tmem, kTcTmem);
    fill_bias<kTcMargin>(p, h, bias);
    if (want_table)
        for (int i = threadIdx.x; i < 2 * 2 * p.reach; i += kGradThreads) bins[i] = 0.0f;
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *(volatile uint32_t*)&ctl.tmem, dq_col = tmem + 256;               // [group] S, dP; dQ
    const uint32_t qS = smem_u32(Qs), kvS = smem_u32(KV), sS = smem_u32(Ss);
    const int64_t items = counted(p.count_dev, p.n_seq) * blocks;
    bool ok = true;
    float far_neg = 0.0f, far_pos = 0.0f;
    // running counts over the items: score tiles (their group is the count's parity), second-pass tiles per group, items
    int64_t it0 = 0, n_items = 0;
    int64_t ds_count[2] = {0, 0};
    for (int64_t k = 0; snake(k) < items && ok; ++k) {
        const int64_t item = snake(k), sn = item / blocks;
        const int i0 = (blocks - 1 - (int)(item % blocks)) * 128;                            // the longest rows of a causal sequence first
        Seq s;
        if (!load_seq(p, sn, s) || max(s.lq, s.lk) <= lo || i0 >= s.lq) continue;
        const int nq = min(128, s.lq - i0), n = (keys_seen(p, s, i0 + nq) + kTcKeys - 1) / kTcKeys;
        if (warp >= 9) {
            // ---- loading warps
            const int tid = threadIdx.x - 288;
            if (n > 0) {
                if (n_items > 0 && !mbar_wait(&ctl.q_empty, (uint32_t)((n_items - 1) & 1), abort_flag)) ok = false;
                if (ok) {
                    load_swizzled<128, DT, 64>(p, p.q, h, s.q0 + i0, nq, qS, tid);
                    load_swizzled<128, DT, 64>(p, p.dout, h, s.q0 + i0, nq, qS + G::Q, tid);
                }
                cp_async_commit();
                // the queries (-1) and the tiles, in order, each once its copies have landed: all of them, or all but the newest group
                int handed = -2;
                const auto hand_over = [&](int upto, bool all) {
                    if (handed >= upto) return;
                    if (all) cp_async_wait<0>();
                    else cp_async_wait<1>();
                    fence_async_shared();
                    while (handed < upto) {
                        ++handed;
                        mbar_arrive(handed < 0 ? &ctl.q_full : &ctl.kv_full[(it0 + handed) % stages]);
                    }
                };
                for (int i = 0; i <= 2 * n && ok; ++i) {
                    if (i < 2 * n) {
                        const int64_t g = it0 + i;
                        const int st = (int)(g % stages), at = (i < n ? i : i - n) * kTcKeys;
                        // two stages: the tile before this one is handed over before the wait, which ends only after its scores
                        if (stages == 2) hand_over(i - 1, true);
                        if (g >= stages && !mbar_wait(&ctl.kv_empty[st], (uint32_t)((g / stages - 1) & 1), abort_flag)) {
                            ok = false;
                            break;
                        }
                        load_swizzled<kTcKeys, DT, 64>(p, p.k, hk, s.k0 + at, min(kTcKeys, s.lk - at), kvS + st * 2 * G::KV, tid);
                        load_swizzled<kTcKeys, DT, 64>(p, p.v, hk, s.k0 + at, min(kTcKeys, s.lk - at), kvS + (st * 2 + 1) * G::KV, tid);
                    }
                    cp_async_commit();
                    hand_over(i - 1, false);
                }
                cp_async_wait<0>();
            }
        } else if (warp == 8) {
            // ---- issuing warp
            constexpr uint32_t idesc_dq = umma_idesc_bf16(128, DT, false, true);
            const auto scores = [&](int i) {
                const int64_t g = it0 + i;
                const int w = (int)(g & 1), st = (int)(g % stages);
                if (!mbar_wait(&ctl.kv_full[st], (uint32_t)((g / stages) & 1), abort_flag)) return false;
                if (g >= 2 && !mbar_wait(&ctl.s_free[w], (uint32_t)((g / 2 - 1) & 1), abort_flag)) return false;
                tc_fence_after_sync();
                if (lane == 0) {
                    mma_rows<DT, 128, kTcKeys>(p, tmem + (uint32_t)(w * 128), qS, kvS + st * 2 * G::KV);
                    mma_rows<DT, 128, kTcKeys>(p, tmem + (uint32_t)(w * 128 + 64), qS + G::Q, kvS + (st * 2 + 1) * G::KV);
                    umma_commit(&ctl.s_full[w]);
                    if (i < n) umma_commit(&ctl.kv_empty[st]);
                    if (i == 2 * n - 1) umma_commit(&ctl.q_empty);
                }
                __syncwarp();
                return true;
            };
            if (n > 0) {
                ok = mbar_wait(&ctl.q_full, (uint32_t)(n_items & 1), abort_flag) && scores(0);
                // the previous item's dQ has been read
                if (ok && n_items > 0) ok = mbar_wait(&ctl.dq_free, (uint32_t)((n_items - 1) & 1), abort_flag);
                for (int i = 0; i < 2 * n && ok; ++i) {
                    if (i + 1 < 2 * n && !scores(i + 1)) {
                        ok = false;
                        break;
                    }
                    if (i < n) continue;
                    const int64_t g = it0 + i;
                    const int w = (int)(g & 1), st = (int)(g % stages);
                    if (!mbar_wait(&ctl.ds_full[w], (uint32_t)(ds_count[w] & 1), abort_flag)) {
                        ok = false;
                        break;
                    }
                    ++ds_count[w];
                    tc_fence_after_sync();
                    if (lane == 0) {
                        const uint32_t a = sS + w * G::S, b = kvS + st * 2 * G::KV;
#pragma unroll
                        for (int q = 0; q < kTcKeys / 16; ++q)
                            umma_bf16(dq_col, umma_smem_desc(a + q * 32, 16, 1024), umma_smem_desc(b + q * 2048, kTcKeys * 128, 1024), idesc_dq, (i - n) > 0 || q > 0);
                        umma_commit(&ctl.kv_empty[st]);
                        umma_commit(&ctl.ds_empty[w]);
                        if (i == 2 * n - 1) umma_commit(&ctl.dq_full);
                    }
                    __syncwarp();
                }
            }
        } else {
            // ---- score warpgroups
            const int grp = warp >> 2, r = threadIdx.x & 127, w0 = i0 + (warp & 3) * 32, i = i0 + r, shift = s.lk - s.lq;
            const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, at = tmem + lanes + (uint32_t)(grp * 128);
            const uint2 key = p.drop.thr ? instance_key(p.drop, sn) : make_uint2(0, 0);
            float m = -INFINITY, l = 0.0f, D = 0.0f, rl = 0.0f;
            bool joined = false;
            const auto join = [&]() {                        // the groups' statistics -> one
                float* mine = stat + (grp * 128 + r) * 3;
                const float* other = stat + ((grp ^ 1) * 128 + r) * 3;
                mine[0] = m;
                mine[1] = l;
                mine[2] = D;
                group_barrier(1, 256);
                const float top = fmaxf(m, other[0]), ref = top == -INFINITY ? 0.0f : top, f0 = ex2_approx(m - ref), f1 = ex2_approx(other[0] - ref);
                // added in the order of the groups: both hold the same numbers
                const float l0 = l * f0, l1 = other[1] * f1, D0 = D * f0, D1 = other[2] * f1;
                l = grp ? l1 + l0 : l0 + l1;
                D = grp ? D1 + D0 : D0 + D1;
                m = ref;
                rl = l == 0.0f ? 0.0f : 1.0f / l;
                D *= rl;
                if (grp == 0 && r < nq) p.stats[(int64_t)h * p.q_rows + s.q0 + i0 + r] = make_float4(m, rl, D, 0.0f);
                joined = true;
            };
            int64_t ds_mine = ds_count[grp];
            for (int q = 0; q < 2 * n; ++q) {
                const int64_t g = it0 + q;
                if ((int)(g & 1) != grp) continue;
                if (q >= n && !joined) join();
                const int j0 = (q < n ? q : q - n) * kTcKeys;
                if (!mbar_wait(&ctl.s_full[grp], (uint32_t)((g / 2) & 1), abort_flag)) *abort_flag = 1, ok = false;
                // (a wait that gave up: the flag ends everybody's, and barriers are met all the same)
                tc_fence_after_sync();
                __syncwarp();
                float t[64], dp[64];
                load_pair(at, t, dp);
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl.s_free[grp]);
                row_scores(p, s, bias, w0, i, j0, t);
                float sum, dsum;
                if (q < n) {
                    float top = m;
#pragma unroll
                    for (int c = 0; c < 64; ++c) top = fmaxf(top, t[c]);
                    const float ref = top == -INFINITY ? 0.0f : top, corr = ex2_approx(m - ref);
                    row_exp(p, s, key, h, i, j0, ref, t, dp, sum, dsum);
                    l = fmaf(l, corr, sum);
                    D = fmaf(D, corr, dsum);
                    m = top;
                    continue;
                }
                row_exp(p, s, key, h, i, j0, m, t, dp, sum, dsum);
                row_ds(p, rl, D, t, dp);
                if (ds_mine > 0 && !mbar_wait(&ctl.ds_empty[grp], (uint32_t)((ds_mine - 1) & 1), abort_flag)) *abort_flag = 1, ok = false;
                ++ds_mine;
                store_row(Ss + grp * G::S, r, dp);
                fence_async_shared();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl.ds_full[grp]);
                if (want_table) {
                    // the tile's distances: one side's last bucket throughout needs no diagonals
                    const bool past = j0 + 63 - (i0 + shift) <= -p.reach, ahead = j0 - (i0 + 127 + shift) >= p.reach;
                    if (past || ahead) {
                        float a = 0.0f, b = 0.0f;
#pragma unroll
                        for (int c = 0; c < 64; c += 2) {
                            a += dp[c];
                            b += dp[c + 1];
                        }
                        (past ? far_neg : far_pos) += a + b;
                    } else {
                        float* bg = bins + grp * 2 * p.reach;
#pragma unroll 1
                        for (int e = 0; e < 32 / kSkewRows; ++e) {          // these rows of every warp, along their diagonals: column c - row + 3
                            const int y0 = lane % kSkewRows;
                            float* mine = stage + (warp * kSkewRows + y0) * kSkewPitch + kSkewRows - 1 - y0;
                            if (lane / kSkewRows == e) {
#pragma unroll
                                for (int c = 0; c < 64; ++c) mine[c] = dp[c];
                            }
                            group_barrier(2 + grp, 128);
                            // a thread per diagonal of the group's 128 rows (key - row within the tile): its bin is its own
                            for (int d = r - 127; d < 64; d += 128) {
                                float a = 0.0f;
#pragma unroll
                                for (int w = 0; w < 4; ++w) {
                                    const int col = d + 32 * w + kSkewRows * e + kSkewRows - 1;
                                    if (col < 0 || col >= kSkewCols) continue;
                                    const float* st = stage + (grp * 4 + w) * kSkewRows * kSkewPitch + col;
#pragma unroll
                                    for (int y = 0; y < kSkewRows; ++y) {
                                        const float x = st[y * kSkewPitch];
                                        a += col + y >= kSkewRows - 1 && col + y < 63 + kSkewRows ? x : 0.0f;
                                    }
                                }
                                const int delta = j0 + d - (i0 + shift);
                                if (delta <= -p.reach) far_neg += a;
                                else if (delta >= p.reach || (!p.bidir && delta > 0)) far_pos += a;
                                else bg[delta + p.reach] += a;
                            }
                            group_barrier(2 + grp, 128);
                        }
                    }
                }
            }
            if (!joined) join();
            // dQ: group 0 reads the first half of the columns, group 1 the second
            uint16_t* out = r < nq ? const_cast<uint16_t*>(static_cast<const uint16_t*>(p.dq.data)) + (s.q0 + i) * p.dq.tok + (int64_t)h * p.dq.head : nullptr;
            if (n > 0) {
                if (!mbar_wait(&ctl.dq_full, (uint32_t)(n_items & 1), abort_flag)) ok = false;
                tc_fence_after_sync();
                __syncwarp();
                store_accumulator<DT / 2>(p, dq_col + lanes + (uint32_t)(grp * (DT / 2)), ok ? out : nullptr, p.scale, grp * (DT / 2));
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl.dq_free);
            } else if (out && grp == 0) {
                for (int c = 0; c < p.dim; c += 8) *reinterpret_cast<uint4*>(out + c) = make_uint4(0, 0, 0, 0);
            }
            ok = group_all(1, 256, ok);                      // and: statistics and staging are free for the next item
            // second-pass tiles of either group
            for (int w = 0; w < 2; ++w) ds_count[w] += n == 0 ? 0 : (int)((n + (((it0 + n) & 1) == w ? 1 : 0)) / 2);
        }
        if (!ok) *abort_flag = 1;
        it0 += 2 * n;
        n_items += n > 0;
    }
    if (!ok) {
        *abort_flag = 1;
        if (lane == 0) latch(p.ctl, AA_ERR_SCAN_TIMEOUT);
    }
    if (warp == 8) {
        if (lane == 0) umma_commit(&ctl.drain);
        __syncwarp();
        const long long t0 = clock64();
        while (!mbar_try_wait(&ctl.drain, 0) && clock64() - t0 < kWaitCycles) {
        }
    }
    if (want_table && warp < 8) {
        far[threadIdx.x] = far_neg;
        far[256 + threadIdx.x] = far_pos;
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == 8) tmem_dealloc(tmem, kTcTmem);
    if (want_table) {
        // the groups' bins -> one array that its far sums follow
        for (int i = threadIdx.x; i < 2 * p.reach; i += kGradThreads) bins[2 * p.reach + i] += bins[i];
        __syncthreads();
        write_table_part(p, part0 + blockIdx.x, h, bins + 2 * p.reach, 0, 1, 256);
    }
}

// ------------------------------------------------------------------------------------------------------------ keys kernel

struct KeysCtl {
    uint64_t kv_full, q_full[2], q_empty[2], s_full[2], s_free[2], ps_full[2], ps_empty[2], acc_full, drain;
    uint32_t tmem;
    int abort_flag;
};

template <int DT>
struct KeysTcGeo {
    static constexpr int KV = kTcKeys * DT * 2, Q = 128 * DT * 2, S = 128 * 128;
    static size_t smem(int pairs, int reach, bool bias) {
        return 1024 + 2 * KV + 4 * Q + (size_t)pairs * 2 * S + sizeof(KeysCtl) + (bias ? bias_floats(reach, kTcMargin) * sizeof(float) : 0);
    }
};

// grid (sequences x key blocks, key heads).  Tiles are counted over the heads of the group: tile g works on head h0 + g / per_head.
template <int DT>
__global__ void __launch_bounds__(kGradThreads, 1) grad_keys_tc_kernel(RelParams p, int lo, int blocks, int pairs) {
    // Two at least: the scores of tile g + 1 are issued before the products of tile g (below), so both tiles' q and dO are held at once; with one
    // stage the issuing warp would wait for a tile that cannot be loaded before its own next products.  (Without that look-ahead one stage gives the
    // same dk and dv under these barriers.)
    constexpr int stages = 2;
    static_assert(stages >= 2, "look-ahead of one tile");
    using G = KeysTcGeo<DT>;
    extern __shared__ char smem_raw[];
    char* KV = reinterpret_cast<char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);     // K, V
    char* Qs = KV + 2 * G::KV;                                                               // [stage][Q, dO]
    char* PS = Qs + stages * 2 * G::Q;                                                       // [P, dS], a pair for each group or one for both
    KeysCtl& ctl = *reinterpret_cast<KeysCtl*>(PS + pairs * 2 * G::S);
    float* bias = reinterpret_cast<float*>(&ctl + 1);
    grid_dependency_wait();
    grid_dependency_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, hk = blockIdx.y, h0 = hk * p.group;
    const int64_t sn = blockIdx.x / blocks;
    const int j0 = (int)(blockIdx.x % blocks) * kTcKeys;
    Seq s;
    if (!load_seq(p, sn, s) || max(s.lq, s.lk) <= lo || j0 >= s.lk) return;
    volatile int* abort_flag = &ctl.abort_flag;
    if (threadIdx.x == 0) {
        mbar_init(&ctl.kv_full, 64);
        for (int w = 0; w < 2; ++w) {
            mbar_init(&ctl.q_full[w], 64);
            mbar_init(&ctl.q_empty[w], 1);
            mbar_init(&ctl.s_full[w], 1);
            mbar_init(&ctl.s_free[w], 4);
            mbar_init(&ctl.ps_full[w], 4);
            mbar_init(&ctl.ps_empty[w], 1);
        }
        mbar_init(&ctl.acc_full, 1);
        mbar_init(&ctl.drain, 1);
        ctl.abort_flag = 0;
        mbar_fence_init();
    }
    if (warp == 8) tmem_alloc(&ctl.tmem, kTcTmem);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *(volatile uint32_t*)&ctl.tmem, dv_col = tmem + 256, dk_col = tmem + 320;      // [group] S, dP; dV^T, dK^T
    const uint32_t kvS = smem_u32(KV), qS = smem_u32(Qs), psS = smem_u32(PS);
    const int nk = min(kTcKeys, s.lk - j0);
    const int first = first_query(p, s, j0) / 128, per_head = max(0, (s.lq + 127) / 128 - first), n = per_head * p.group;
    bool ok = true;
    if (warp >= 9) {
        // ---- loading warps
        const int tid = threadIdx.x - 288;
        load_swizzled<kTcKeys, DT, 64>(p, p.k, hk, s.k0 + j0, nk, kvS, tid);
        load_swizzled<kTcKeys, DT, 64>(p, p.v, hk, s.k0 + j0, nk, kvS + G::KV, tid);
        cp_async_commit();
        int handed = -2;                                     // K and V (-1), then the query tiles
        const auto hand_over = [&](int upto, bool all) {
            if (handed >= upto) return;
            if (all) cp_async_wait<0>();
            else cp_async_wait<1>();
            fence_async_shared();
            while (handed < upto) {
                ++handed;
                mbar_arrive(handed < 0 ? &ctl.kv_full : &ctl.q_full[handed % stages]);
            }
        };
        for (int g = 0; g < n && ok; ++g) {
            const int st = g % stages, h = h0 + g / per_head, i0 = (first + g % per_head) * 128, nq = min(128, s.lq - i0);
            if (g >= stages) {
                hand_over(g - 1, true);                      // before the wait, which ends only after the next tile's scores
                if (!mbar_wait(&ctl.q_empty[st], (uint32_t)((g / stages - 1) & 1), abort_flag)) {
                    ok = false;
                    break;
                }
            }
            load_swizzled<128, DT, 64>(p, p.q, h, s.q0 + i0, nq, qS + st * 2 * G::Q, tid);
            load_swizzled<128, DT, 64>(p, p.dout, h, s.q0 + i0, nq, qS + (st * 2 + 1) * G::Q, tid);
            cp_async_commit();
            hand_over(g - 1, false);
        }
        if (ok) hand_over(n - 1, true);
        cp_async_wait<0>();
    } else if (warp == 8) {
        // ---- issuing warp
        constexpr uint32_t idesc_t = umma_idesc_bf16(128, kTcKeys, true, true);
        const auto scores = [&](int g) {
            const int w = g & 1, st = g % stages;
            if (!mbar_wait(&ctl.q_full[st], (uint32_t)((g / stages) & 1), abort_flag)) return false;
            if (g >= 2 && !mbar_wait(&ctl.s_free[w], (uint32_t)((g / 2 - 1) & 1), abort_flag)) return false;
            tc_fence_after_sync();
            if (lane == 0) {
                mma_rows<DT, 128, kTcKeys>(p, tmem + (uint32_t)(w * 128), qS + st * 2 * G::Q, kvS);
                mma_rows<DT, 128, kTcKeys>(p, tmem + (uint32_t)(w * 128 + 64), qS + (st * 2 + 1) * G::Q, kvS + G::KV);
                umma_commit(&ctl.s_full[w]);
            }
            __syncwarp();
            return true;
        };
        if (n > 0) {
            ok = mbar_wait(&ctl.kv_full, 0, abort_flag) && scores(0);
            for (int g = 0; g < n && ok; ++g) {
                // the next tile's scores before this one's products
                if (g + 1 < n && !scores(g + 1)) ok = false;
                const int w = g & 1, st = g % stages;
                if (!ok || !mbar_wait(&ctl.ps_full[w], (uint32_t)((g / 2) & 1), abort_flag)) {
                    ok = false;
                    break;
                }
                tc_fence_after_sync();
                if (lane == 0) {
                    // left operands: head elements x query rows, in two blocks of 64 elements (at a width of 64 the second half of the lanes repeats the first)
                    const uint32_t q = qS + st * 2 * G::Q, o = q + G::Q, pt = psS + (pairs == 2 ? w : 0) * 2 * G::S, ds = pt + G::S, chunk = DT > 64 ? 128 * 128 : 0;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        umma_bf16(dv_col, umma_smem_desc(o + k * 2048, chunk, 1024), umma_smem_desc(pt + k * 2048, 16, 1024), idesc_t, g > 0 || k > 0);
                        umma_bf16(dk_col, umma_smem_desc(q + k * 2048, chunk, 1024), umma_smem_desc(ds + k * 2048, 16, 1024), idesc_t, g > 0 || k > 0);
                    }
                    umma_commit(&ctl.q_empty[st]);
                    umma_commit(&ctl.ps_empty[pairs == 2 ? w : 0]);
                    if (g + 1 == n) umma_commit(&ctl.acc_full);
                }
                __syncwarp();
            }
        }
        if (lane == 0) umma_commit(&ctl.drain);
        __syncwarp();
        const long long t0 = clock64();
        while (!mbar_try_wait(&ctl.drain, 0) && clock64() - t0 < kWaitCycles) {
        }
    } else {
        // ---- score warpgroups
        const int grp = warp >> 2, r = threadIdx.x & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, at = tmem + lanes + (uint32_t)(grp * 128);
        const uint2 key = p.drop.thr ? instance_key(p.drop, sn) : make_uint2(0, 0);
        int filled = -1;
        for (int g = 0; g < n; ++g) {
            const int h = h0 + g / per_head, i0 = (first + g % per_head) * 128, i = i0 + r, w0 = i0 + (warp & 3) * 32;
            if (h != filled) {                               // both groups meet at a head's first tile
                group_barrier(1, 256);
                fill_bias<kTcMargin>(p, h, bias, 8, (int)(threadIdx.x >> 5));
                group_barrier(1, 256);
                filled = h;
            }
            if ((g & 1) != grp) continue;
            const float4 st = i < s.lq ? p.stats[(int64_t)h * p.q_rows + s.q0 + i] : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (!mbar_wait(&ctl.s_full[grp], (uint32_t)((g / 2) & 1), abort_flag)) *abort_flag = 1, ok = false;
            tc_fence_after_sync();
            __syncwarp();
            float t[64], dp[64], sum, dsum;
            load_pair(at, t, dp);
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.s_free[grp]);
            row_scores(p, s, bias, w0, i, j0, t);
            row_exp(p, s, key, h, i, j0, st.x, t, dp, sum, dsum);
            row_ds(p, st.y, st.z, t, dp);
            // the products that read this pair last: two tiles ago, or one where the groups share it
            const int pair = pairs == 2 ? grp : 0, before = pairs == 2 ? g / 2 : g;
            if (before > 0 && !mbar_wait(&ctl.ps_empty[pair], (uint32_t)((before - 1) & 1), abort_flag)) *abort_flag = 1, ok = false;
            store_row(PS + pair * 2 * G::S, r, t);
            store_row(PS + (pair * 2 + 1) * G::S, r, dp);
            fence_async_shared();
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.ps_full[grp]);
        }
        // group 0: dV, group 1: dK; a lane holds one head element of every key
        const TokArg& out = grp ? p.dk : p.dv;
        const float f = grp ? p.scale : 1.0f;
        uint16_t* base = const_cast<uint16_t*>(static_cast<const uint16_t*>(out.data)) + (s.k0 + j0) * out.tok + (int64_t)hk * out.head + r;
        const bool mine = r < p.dim && r < DT;
        if (n > 0) {
            if (!mbar_wait(&ctl.acc_full, 0, abort_flag)) ok = false;
            tc_fence_after_sync();
            __syncwarp();
            float v[64];
            load_row((grp ? dk_col : dv_col) + lanes, v);
            if (mine && ok) {
#pragma unroll
                for (int c = 0; c < 64; ++c)
                    if (c < nk) store1(base + (int64_t)c * out.tok, v[c] * f);
            }
        } else if (mine) {
            for (int c = 0; c < nk; ++c) store1(base + (int64_t)c * out.tok, 0.0f);
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

// Sequences of more than `lo` tokens on either side.
template <int DT>
aa_status backward(aa_ctx_impl* c, RelParams p, int lo, int* n_parts) {
    const void* rows = (const void*)grad_rows_tc_kernel<DT>;
    const void* keys = (const void*)grad_keys_tc_kernel<DT>;
    // a far-reaching bias leaves room for fewer stages
    int stages_r = RowsTcGeo<DT>::smem(kRowStages, p.reach, p.table, p.table && p.dtable) <= 227 * 1024 ? kRowStages : 2;
    const size_t smem_r = RowsTcGeo<DT>::smem(stages_r, p.reach, p.table, p.table && p.dtable);
    int pairs = KeysTcGeo<DT>::smem(2, p.reach, p.table) <= 227 * 1024 ? 2 : 1;       // ... or for one pair of p and dS tiles
    const size_t smem_k = KeysTcGeo<DT>::smem(pairs, p.reach, p.table);
    int blocks_q = (int)((p.max_q + 127) / 128), blocks_k = (int)((p.max_k + kTcKeys - 1) / kTcKeys);
    if (allow_smem(c, rows, smem_r) != AA_OK ||
        allow_smem(c, keys, smem_k) != AA_OK)
        return AA_ERR_CUDA;
    if (p.n_seq * blocks_k > 0x7FFFFFFFll) return AA_ERR_UNSUPPORTED;
    int64_t grid = c->sm_count / p.heads > 0 ? c->sm_count / p.heads : 1;             // one CTA an SM, one wave
    if (grid > p.n_seq * blocks_q) grid = p.n_seq * blocks_q;
    if (grid > rel_grad_parts(p.heads)) grid = rel_grad_parts(p.heads);
    if (grid > 0) {
        void* args[] = {&p, &lo, &blocks_q, n_parts, &stages_r};
        if (launch_overlapped(c, rows, dim3((unsigned)grid, p.heads), dim3(kGradThreads), args, smem_r, false) != cudaSuccess) return AA_ERR_CUDA;
        ++c->launches;
    }
    if (blocks_k > 0) {
        void* args[] = {&p, &lo, &blocks_k, &pairs};
        if (launch_overlapped(c, keys, dim3((unsigned)(p.n_seq * blocks_k), p.kv_heads), dim3(kGradThreads), args, smem_k, false) != cudaSuccess) return AA_ERR_CUDA;
        ++c->launches;
    }
    *n_parts += (int)grid;
    return AA_OK;
}

}  // namespace

aa_status launch_rel_attention_grad_tc(aa_ctx_impl* c, const RelParams& p, int lo, int* n_parts) {
    return p.dim <= 64 ? backward<64>(c, p, lo, n_parts) : backward<128>(c, p, lo, n_parts);
}

}  // namespace aa
