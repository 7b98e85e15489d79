// Backward pass of the bf16 attention with a relative position bias.
//
// keys kernel: a CTA owns a block of BK keys of one key head and walks the query tiles (64 rows) of the heads that share it; dK and dV stay
// in registers, 16 keys a warp.  WHOLE: the block holds every key of the sequence, so the row statistics come from the tile itself and the
// same pass also writes dQ and adds up the bias gradient: each operand is read once and five products are made.  Otherwise the statistics
// come from the rows kernel.
// rows kernel (sequences of more than 128 keys): a CTA owns 128 query rows of one head and streams 64-key tiles twice: first the running
// maximum, sum and D = sum p dp, from unrounded probabilities (rounded ones would cost the fp32 bias gradient its digits), then dS, its
// diagonal sums and dQ.
//
// ds = p (dp - D) and p are rounded to bf16 as operands of the products with K, Q and dO, whose results are bf16; the diagonal sums are
// taken before the rounding.
#include "rel_attention_mma.cuh"

namespace aa {

namespace {

// Row statistics of lane (g, t)'s rows g and g + 8.
struct RowStats {
    float m[2], rl[2], D[2];
};

// p, dp, D -> ds in `dp`, dropped and scaled p in `t` (both fp32).
__device__ __forceinline__ void block_ds(const RelParams& p, const RowStats& st, uint32_t dropped, float (&t)[8][4], float (&dp)[8][4]) {
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int r = e >> 1;
            const float prob = ex2_approx(t[n][e] - st.m[r]) * st.rl[r];
            dp[n][e] = prob * (dp[n][e] - st.D[r]);
            t[n][e] = (dropped >> (4 * n + e)) & 1u ? 0.0f : prob * p.drop.scale;
        }
}
// dp of dropped probabilities is 0, of kept ones scaled.
__device__ __forceinline__ void block_dp(const RelParams& p, uint32_t dropped, float (&dp)[8][4]) {
    if (!p.drop.thr) return;
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) dp[n][e] = (dropped >> (4 * n + e)) & 1u ? 0.0f : __fmul_rn(dp[n][e], p.drop.scale);
}
__device__ __forceinline__ float block_max(const float (&t)[8][4], int r, float top) {
#pragma unroll
    for (int n = 0; n < 8; ++n) top = fmaxf(top, fmaxf(t[n][2 * r], t[n][2 * r + 1]));
    return quad_max(top);
}
// sums of e = 2^(t - ref) and of e dp over row r of the block (this lane's part)
__device__ __forceinline__ void block_sums(const float (&t)[8][4], const float (&dp)[8][4], int r, float ref, float& sum, float& dsum) {
    sum = dsum = 0.0f;
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const float e = ex2_approx(t[n][2 * r + c] - ref);
            sum += e;
            dsum = fmaf(e, dp[n][2 * r + c], dsum);
        }
}
__device__ __forceinline__ float block_total(const float (&ds)[8][4]) {
    float a = 0.0f;
#pragma unroll
    for (int n = 0; n < 8; ++n) a += (ds[n][0] + ds[n][1]) + (ds[n][2] + ds[n][3]);
    return a;
}

// ------------------------------------------------------------------------------------------------------------ keys kernel

template <int DT, int BK>
struct KeysGeo {
    static constexpr int WARPS = BK / 16, THREADS = WARPS * 32, WK = BK / 64;      // 4 row groups x WK key halves of 64
    static constexpr int P = pitch_of(DT), PP = pitch_of(BK);
    static constexpr int kTileElems = 2 * BK * P + 2 * 64 * P + 2 * 64 * PP;       // K V, Q dO, P dS
    static constexpr int kStatFloats = 64 * WK * 3;
    static size_t smem(bool whole, int group, int reach, bool bias, bool table) {
        size_t b = (size_t)kTileElems * 2;
        if (whole) b += (kStatFloats + (table ? WARPS * kDiagFloats : 0)) * sizeof(float);
        if (bias) b += (size_t)(whole ? group : 1) * (2 * reach + 1) * sizeof(float);
        if (whole && table) b += (size_t)group * (2 * reach + 2 * THREADS) * sizeof(float);
        return b;
    }
};

// WHOLE: grid (parts, key heads), a CTA walks the sequences of lk_min < keys <= BK; else grid (sequences x key blocks, key heads) over the
// sequences of more than lk_min keys.
template <int DT, int BK, bool WHOLE>
__global__ void __launch_bounds__(BK * 2) grad_keys_kernel(RelParams p, int lk_min, int blocks, int part0) {
    using G = KeysGeo<DT, BK>;
    constexpr int P = G::P, PP = G::PP, THREADS = G::THREADS;
    extern __shared__ uint4 smem16[];
    uint16_t* Ks = reinterpret_cast<uint16_t*>(smem16);
    uint16_t* Vs = Ks + BK * P;
    uint16_t* Qs = Vs + BK * P;
    uint16_t* Os = Qs + 64 * P;
    uint16_t* Ps = Os + 64 * P;
    uint16_t* Ss = Ps + 64 * PP;
    float* stat = reinterpret_cast<float*>(Ss + 64 * PP);                 // [key half][row][m, l, D]
    const bool want_table = WHOLE && p.table && p.dtable;
    float* stage = stat + (WHOLE ? G::kStatFloats : 0);                   // [warp] skewed diagonals
    float* bias = stage + (want_table ? G::WARPS * kDiagFloats : 0);      // [head of the group]
    const int bias_len = p.table ? 2 * p.reach + 1 : 0;
    // per head of the group: the bins by distance, then each thread's sums of the far past and the far future
    const int bin_len = 2 * p.reach + 2 * THREADS;
    float* bins = bias + (WHOLE ? p.group : 1) * bias_len;
    grid_dependency_wait();
    grid_dependency_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wq = warp & 3, wk = warp >> 2;
    const int hk = blockIdx.y, h0 = hk * p.group;
    if (WHOLE) {
        for (int a = 0; a < p.group; ++a) fill_bias(p, h0 + a, bias + a * bias_len);
        if (want_table) {
            for (int i = threadIdx.x; i < p.group * bin_len; i += THREADS) bins[i] = 0.0f;
            for (int i = threadIdx.x; i < G::WARPS * kDiagFloats; i += THREADS) stage[i] = 0.0f;
        }
    }
    const uint32_t kS = smem_u32(Ks), vS = smem_u32(Vs), qS = smem_u32(Qs), oS = smem_u32(Os), pS = smem_u32(Ps), sS = smem_u32(Ss);
    const int64_t items = WHOLE ? counted(p.count_dev, p.n_seq) : 1;
    for (int64_t item = WHOLE ? blockIdx.x : 0; item < items; item += WHOLE ? gridDim.x : 1) {
        const int64_t sn = WHOLE ? item : blockIdx.x / blocks;
        const int j0 = WHOLE ? 0 : (int)(blockIdx.x % blocks) * BK;
        Seq s;
        if (!load_seq(p, sn, s) || s.lk <= lk_min || (WHOLE ? s.lk > BK : j0 >= s.lk)) continue;
        const uint2 key = p.drop.thr ? instance_key(p.drop, sn) : make_uint2(0, 0);
        const int nk = min(BK, s.lk - j0);
        __syncthreads();                                                  // the previous item's tiles have been read
        load_tile_async<BK, DT, THREADS>(p, p.k, hk, s.k0 + j0, nk, Ks);
        load_tile_async<BK, DT, THREADS>(p, p.v, hk, s.k0 + j0, nk, Vs);
        float gk[DT / 8][4], gv[DT / 8][4];
#pragma unroll
        for (int j = 0; j < DT / 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) gk[j][e] = gv[j][e] = 0.0f;
        for (int a = 0; a < p.group; ++a) {
            const int h = h0 + a;
            float* bias_h = bias + (WHOLE ? a * bias_len : 0);
            if (!WHOLE) {
                __syncthreads();
                fill_bias(p, h, bias_h);
            }
            // WHOLE writes dQ of every row, those before the first key's too (zeros)
            for (int i0 = WHOLE ? 0 : first_query(p, s, j0) / 64 * 64; i0 < s.lq; i0 += 64) {
                const int nq = min(64, s.lq - i0);
                __syncthreads();
                load_tile_async<64, DT, THREADS>(p, p.q, h, s.q0 + i0, nq, Qs);
                load_tile_async<64, DT, THREADS>(p, p.dout, h, s.q0 + i0, nq, Os);
                cp_async_commit();
                const Block b = {i0 + wq * 16, j0 + wk * 64};
                const int n16 = block_groups(p, s, b);
                const uint32_t dropped = p.drop.thr && n16 > 0 ? block_drops(p, s, key, h, b, lane) : 0u;
                cp_async_wait<0>();
                __syncthreads();
                float t[8][4], dp[8][4];
                {
                    uint32_t f[DT / 16][4];
                    load_frags<DT>(p, f, qS, wq * 16, lane);
                    block_dot<DT>(p, f, kS, wk * 64, n16, lane, t);
                    load_frags<DT>(p, f, oS, wq * 16, lane);
                    block_dot<DT>(p, f, vS, wk * 64, n16, lane, dp);
                }
                block_scores(p, s, bias_h, b, lane, t);
                block_dp(p, dropped, dp);
                RowStats st;
                if (WHOLE) {
                    float m[2], l[2], D[2];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        m[r] = block_max(t, r, -INFINITY);
                        block_sums(t, dp, r, m[r] == -INFINITY ? 0.0f : m[r], l[r], D[r]);
                        l[r] = quad_sum(l[r]);
                        D[r] = quad_sum(D[r]);
                    }
                    if (G::WK > 1) {                                      // join the key halves
                        if ((lane & 3) == 0)
#pragma unroll
                            for (int r = 0; r < 2; ++r) {
                                float* at = stat + (wk * 64 + wq * 16 + (lane >> 2) + 8 * r) * 3;
                                at[0] = m[r];
                                at[1] = l[r];
                                at[2] = D[r];
                            }
                        __syncthreads();
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const float* at = stat + ((1 - wk) * 64 + wq * 16 + (lane >> 2) + 8 * r) * 3;
                            const float top = fmaxf(m[r], at[0]), ref = top == -INFINITY ? 0.0f : top;
                            const float f0 = ex2_approx(m[r] - ref), f1 = ex2_approx(at[0] - ref);
                            l[r] = l[r] * f0 + at[1] * f1;
                            D[r] = D[r] * f0 + at[2] * f1;
                            m[r] = top;
                        }
                    }
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        st.m[r] = m[r] == -INFINITY ? 0.0f : m[r];
                        st.rl[r] = l[r] == 0.0f ? 0.0f : 1.0f / l[r];
                        st.D[r] = D[r] * st.rl[r];
                    }
                } else {
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int i = wq * 16 + (lane >> 2) + 8 * r;
                        const float4 x = i < nq ? __ldg(p.stats + (int64_t)h * p.q_rows + s.q0 + i0 + i) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                        st.m[r] = x.x;
                        st.rl[r] = x.y;
                        st.D[r] = x.z;
                    }
                }
                block_ds(p, st, dropped, t, dp);
                if (want_table) stage_diagonals(stage + warp * kDiagFloats, dp, lane);
                {
                    const int g = lane >> 2, q2 = 2 * (lane & 3);
                    uint16_t* prow = Ps + (wq * 16 + g) * PP + wk * 64 + q2;
                    uint16_t* srow = Ss + (wq * 16 + g) * PP + wk * 64 + q2;
#pragma unroll
                    for (int n = 0; n < 8; ++n) {
                        *reinterpret_cast<uint32_t*>(prow + 8 * n) = pack_bf16(t[n][0], t[n][1]);
                        *reinterpret_cast<uint32_t*>(prow + 8 * PP + 8 * n) = pack_bf16(t[n][2], t[n][3]);
                        *reinterpret_cast<uint32_t*>(srow + 8 * n) = pack_bf16(dp[n][0], dp[n][1]);
                        *reinterpret_cast<uint32_t*>(srow + 8 * PP + 8 * n) = pack_bf16(dp[n][2], dp[n][3]);
                    }
                }
                __syncthreads();
                // dV += P^T dO, dK += dS^T Q: this warp's 16 keys, contraction over the tile's rows
                if (warp * 16 < nk) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (k * 16 >= nq) continue;
                        uint32_t pa[4], sa[4];
                        ldsm4t(pa, frag_trans<PP>(pS, k * 16, warp * 16, lane));
                        ldsm4t(sa, frag_trans<PP>(sS, k * 16, warp * 16, lane));
#pragma unroll
                        for (int j = 0; j < DT / 16; ++j) {
                            if (DT > 64 && j * 16 >= p.dim) continue;
                            uint32_t x[4];
                            ldsm4t(x, frag_rows<P>(oS, k * 16, j * 16, lane));
                            mma16816(gv[2 * j], pa, x[0], x[1]);
                            mma16816(gv[2 * j + 1], pa, x[2], x[3]);
                            ldsm4t(x, frag_rows<P>(qS, k * 16, j * 16, lane));
                            mma16816(gk[2 * j], sa, x[0], x[1]);
                            mma16816(gk[2 * j + 1], sa, x[2], x[3]);
                        }
                    }
                }
                if (WHOLE) {
                    // dQ = dS K: this warp's 16 rows, its half (or all) of the head's columns
                    constexpr int NJ = DT / 16 / G::WK;
                    float gq[2 * NJ][4];
#pragma unroll
                    for (int j = 0; j < 2 * NJ; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) gq[j][e] = 0.0f;
                    if (wq * 16 < nq) {
#pragma unroll
                        for (int k = 0; k < BK / 16; ++k) {
                            if (k * 16 >= nk) continue;
                            uint32_t sa[4];
                            ldsm4(sa, frag_rows<PP>(sS, wq * 16, k * 16, lane));
#pragma unroll
                            for (int j = 0; j < NJ; ++j) {
                                uint32_t x[4];
                                ldsm4t(x, frag_rows<P>(kS, k * 16, (wk * NJ + j) * 16, lane));
                                mma16816(gq[2 * j], sa, x[0], x[1]);
                                mma16816(gq[2 * j + 1], sa, x[2], x[3]);
                            }
                        }
                        const int g = lane >> 2;
                        uint16_t* base = const_cast<uint16_t*>(static_cast<const uint16_t*>(p.dq.data)) + (s.q0 + i0 + wq * 16) * p.dq.tok + (int64_t)h * p.dq.head +
                                         wk * NJ * 16 + 2 * (lane & 3);
#pragma unroll
                        for (int j = 0; j < 2 * NJ; ++j) {
                            if (wk * NJ * 16 + j * 8 >= p.dim) continue;
                            if (wq * 16 + g < nq)
                                *reinterpret_cast<uint32_t*>(base + (int64_t)g * p.dq.tok + j * 8) = pack_bf16(gq[j][0] * p.scale, gq[j][1] * p.scale);
                            if (wq * 16 + g + 8 < nq)
                                *reinterpret_cast<uint32_t*>(base + (int64_t)(g + 8) * p.dq.tok + j * 8) = pack_bf16(gq[j][2] * p.scale, gq[j][3] * p.scale);
                        }
                    }
                    if (want_table) {
                        // one thread per diagonal of the tile: key - row = d in [-63, BK - 1]; its distance's bin is its own
                        for (int d = (int)threadIdx.x - 63; d < BK; d += THREADS) {
                            float sum = 0.0f;
#pragma unroll
                            for (int w = 0; w < G::WARPS; ++w) {
                                const int col = d + 16 * (w & 3) - 64 * (w >> 2) + 15;
                                if (col >= 0 && col < kDiagCols) sum += diagonal_sum(stage + w * kDiagFloats, col);
                            }
                            const int delta = d - (i0 + s.lk - s.lq);
                            float* bh = bins + a * bin_len;
                            if (delta <= -p.reach) bh[2 * p.reach + threadIdx.x] += sum;
                            else if (delta >= p.reach || (!p.bidir && delta > 0)) bh[2 * p.reach + THREADS + threadIdx.x] += sum;
                            else bh[delta + p.reach] += sum;
                        }
                    }
                }
            }
        }
        if (warp * 16 < nk) {
            store_block<DT>(p, p.dk, hk, s.k0 + j0 + warp * 16, nk - warp * 16, lane, gk, p.scale, p.scale);
            store_block<DT>(p, p.dv, hk, s.k0 + j0 + warp * 16, nk - warp * 16, lane, gv, 1.0f, 1.0f);
        }
    }
    if (want_table) {
        __syncthreads();
        for (int a = 0; a < p.group; ++a) {
            const float* bh = bins + a * bin_len;
            write_table_part(p, part0 + blockIdx.x, h0 + a, bh, bh + 2 * p.reach, bh + 2 * p.reach + THREADS, THREADS);
        }
    }
}

// ------------------------------------------------------------------------------------------------------------ rows kernel

template <int DT>
struct RowsGeo {
    static constexpr int WARPS = 8, THREADS = 256, P = pitch_of(DT);
    static size_t smem(int reach, bool bias, bool table) {
        size_t b = (size_t)(2 * 128 * P + 4 * 64 * P) * 2;                 // Q dO, K V twice
        if (bias) b += (2 * reach + 1) * sizeof(float);
        if (table) b += (WARPS * kDiagFloats + 2 * reach + 2 * THREADS) * sizeof(float);
        return b;
    }
};

template <int DT>
__global__ void __launch_bounds__(256) grad_rows_kernel(RelParams p, int lk_min, int blocks, int part0) {
    using G = RowsGeo<DT>;
    constexpr int P = G::P, THREADS = G::THREADS;
    extern __shared__ uint4 smem16[];
    uint16_t* Qs = reinterpret_cast<uint16_t*>(smem16);
    uint16_t* Os = Qs + 128 * P;
    uint16_t* KV = Os + 128 * P;                                           // K0 V0 K1 V1
    float* bias = reinterpret_cast<float*>(KV + 4 * 64 * P);
    const bool want_table = p.table && p.dtable;
    float* stage = bias + (p.table ? 2 * p.reach + 1 : 0);
    float* bins = stage + (want_table ? G::WARPS * kDiagFloats : 0);
    float* far = bins + 2 * p.reach;                                       // each thread's sums of the far past, then the far future
    grid_dependency_wait();
    grid_dependency_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, h = blockIdx.y, hk = h / p.group;
    fill_bias(p, h, bias);
    if (want_table) {
        for (int i = threadIdx.x; i < 2 * p.reach; i += THREADS) bins[i] = 0.0f;
        for (int i = threadIdx.x; i < G::WARPS * kDiagFloats; i += THREADS) stage[i] = 0.0f;
    }
    float far_neg = 0.0f, far_pos = 0.0f;
    const int64_t items = counted(p.count_dev, p.n_seq) * blocks;
    // later row blocks of a causal sequence see more keys: the longest first
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t sn = item / blocks;
        const int i0 = (blocks - 1 - (int)(item % blocks)) * 128;
        Seq s;
        if (!load_seq(p, sn, s) || s.lk <= lk_min || i0 >= s.lq) continue;
        const uint2 key = p.drop.thr ? instance_key(p.drop, sn) : make_uint2(0, 0);
        const int nq = min(128, s.lq - i0), end = keys_seen(p, s, i0 + nq), n_tiles = (end + 63) / 64;
        const auto load_kv = [&](int it) {
            const int tile = it < n_tiles ? it : it - n_tiles;             // second pass
            uint16_t* dst = KV + (it & 1) * 2 * 64 * P;
            load_tile_async<64, DT, THREADS>(p, p.k, hk, s.k0 + tile * 64, min(64, s.lk - tile * 64), dst);
            load_tile_async<64, DT, THREADS>(p, p.v, hk, s.k0 + tile * 64, min(64, s.lk - tile * 64), dst + 64 * P);
        };
        __syncthreads();                                                   // the previous item's tiles have been read
        load_tile_async<128, DT, THREADS>(p, p.q, h, s.q0 + i0, nq, Qs);
        load_tile_async<128, DT, THREADS>(p, p.dout, h, s.q0 + i0, nq, Os);
        if (n_tiles > 0) load_kv(0);
        cp_async_commit();
        uint32_t qf[DT / 16][4], of[DT / 16][4];
        float gq[DT / 8][4];
#pragma unroll
        for (int j = 0; j < DT / 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) gq[j][e] = 0.0f;
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f}, D[2] = {0.0f, 0.0f};
        RowStats st = {{0.0f, 0.0f}, {0.0f, 0.0f}, {0.0f, 0.0f}};
        const int row = warp * 16 + (lane >> 2);
        const auto finish_stats = [&]() {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float sum = quad_sum(l[r]), dsum = quad_sum(D[r]);
                st.m[r] = m[r] == -INFINITY ? 0.0f : m[r];
                st.rl[r] = sum == 0.0f ? 0.0f : 1.0f / sum;
                st.D[r] = dsum * st.rl[r];
                if ((lane & 3) == 0 && row + 8 * r < nq) p.stats[(int64_t)h * p.q_rows + s.q0 + i0 + row + 8 * r] = make_float4(st.m[r], st.rl[r], st.D[r], 0.0f);
            }
        };
        if (n_tiles == 0) {
            cp_async_wait<0>();
            finish_stats();
        }
        for (int it = 0; it < 2 * n_tiles; ++it) {
            const int j0 = (it < n_tiles ? it : it - n_tiles) * 64;
            cp_async_wait<0>();
            __syncthreads();
            if (it + 1 < 2 * n_tiles) {
                load_kv(it + 1);
                cp_async_commit();
            }
            if (it == 0) {
                load_frags<DT>(p, qf, smem_u32(Qs), warp * 16, lane);
                load_frags<DT>(p, of, smem_u32(Os), warp * 16, lane);
            }
            const uint32_t kS = smem_u32(KV + (it & 1) * 2 * 64 * P), vS = kS + 64 * P * 2;
            const Block b = {i0 + warp * 16, j0};
            const int n16 = block_groups(p, s, b);
            float t[8][4], dp[8][4];
            uint32_t dropped = 0;
            if (n16 > 0) {
                block_dot<DT>(p, qf, kS, 0, n16, lane, t);
                block_dot<DT>(p, of, vS, 0, n16, lane, dp);
                block_scores(p, s, bias, b, lane, t);
                if (p.drop.thr) dropped = block_drops(p, s, key, h, b, lane);
                block_dp(p, dropped, dp);
            }
            if (it < n_tiles) {
                if (n16 > 0) {
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float top = block_max(t, r, m[r]), ref = top == -INFINITY ? 0.0f : top, corr = ex2_approx(m[r] - ref);
                        float sum, dsum;
                        block_sums(t, dp, r, ref, sum, dsum);
                        l[r] = fmaf(l[r], corr, sum);
                        D[r] = fmaf(D[r], corr, dsum);
                        m[r] = top;
                    }
                }
                if (it == n_tiles - 1) finish_stats();
                continue;
            }
            const int shift = s.lk - s.lq;
            // distances of the whole CTA's tile: one side's last bucket throughout needs no diagonals
            const bool past = j0 + 63 - (i0 + shift) <= -p.reach, ahead = j0 - (i0 + 127 + shift) >= p.reach;
            if (n16 > 0) {
                block_ds(p, st, dropped, t, dp);
                if (want_table && past) far_neg += block_total(dp);
                if (want_table && ahead) far_pos += block_total(dp);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (k >= n16) continue;
                    const uint32_t a[4] = {pack_bf16(dp[2 * k][0], dp[2 * k][1]), pack_bf16(dp[2 * k][2], dp[2 * k][3]), pack_bf16(dp[2 * k + 1][0], dp[2 * k + 1][1]),
                                           pack_bf16(dp[2 * k + 1][2], dp[2 * k + 1][3])};
#pragma unroll
                    for (int j = 0; j < DT / 16; ++j) {
                        if (DT > 64 && j * 16 >= p.dim) continue;
                        uint32_t x[4];
                        ldsm4t(x, frag_rows<P>(kS, k * 16, j * 16, lane));
                        mma16816(gq[2 * j], a, x[0], x[1]);
                        mma16816(gq[2 * j + 1], a, x[2], x[3]);
                    }
                }
            }
            if (want_table && !past && !ahead) {
                if (n16 == 0) {
#pragma unroll
                    for (int n = 0; n < 8; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) dp[n][e] = 0.0f;
                }
                stage_diagonals(stage + warp * kDiagFloats, dp, lane);
                __syncthreads();
                if (threadIdx.x < 191) {
                    const int d = (int)threadIdx.x - 127;                  // key - row within the tile
                    float sum = 0.0f;
#pragma unroll
                    for (int w = 0; w < G::WARPS; ++w) {
                        const int col = d + 16 * w + 15;
                        if (col >= 0 && col < kDiagCols) sum += diagonal_sum(stage + w * kDiagFloats, col);
                    }
                    const int delta = j0 + d - (i0 + shift);
                    if (delta <= -p.reach) far_neg += sum;
                    else if (delta >= p.reach || (!p.bidir && delta > 0)) far_pos += sum;
                    else bins[delta + p.reach] += sum;
                }
            }
        }
        store_block<DT>(p, p.dq, h, s.q0 + i0 + warp * 16, nq - warp * 16, lane, gq, p.scale, p.scale);
    }
    if (want_table) {
        far[threadIdx.x] = far_neg;
        far[THREADS + threadIdx.x] = far_pos;
        __syncthreads();
        write_table_part(p, part0 + blockIdx.x, h, bins, far, far + THREADS, THREADS);
    }
}

aa_status prepare(aa_ctx_impl* c, const void* kernel, int threads, size_t smem, int* resident) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return AA_ERR_CUDA;
    *resident = resident_ctas(c, kernel, threads, smem);
    return *resident > 0 ? AA_OK : AA_ERR_CUDA;
}

// Sequences of lk_min < keys <= BK.
template <int DT, int BK>
aa_status whole(aa_ctx_impl* c, RelParams& p, int lk_min, int* part0) {
    using G = KeysGeo<DT, BK>;
    const void* kernel = (const void*)grad_keys_kernel<DT, BK, true>;
    const size_t smem = G::smem(true, p.group, p.reach, p.table, p.table && p.dtable);
    int cap = 0, blocks = 0;
    if (prepare(c, kernel, G::THREADS, smem, &cap) != AA_OK) return AA_ERR_CUDA;
    int64_t grid = (cap + p.kv_heads - 1) / p.kv_heads;
    if (grid > p.n_seq) grid = p.n_seq;
    if (grid > rel_grad_parts(p.heads)) grid = rel_grad_parts(p.heads);
    void* args[] = {&p, &lk_min, &blocks, part0};
    if (launch_overlapped(c, kernel, dim3((unsigned)grid, p.kv_heads), dim3(G::THREADS), args, smem, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    *part0 += (int)grid;
    return AA_OK;
}

template <int DT>
aa_status backward(aa_ctx_impl* c, RelParams p, int* n_parts) {
    using GR = RowsGeo<DT>;
    using GK = KeysGeo<DT, 128>;
    *n_parts = 0;
    // the whole-sequence kernels keep the bias and the bins of every head of a key head's group in shared memory
    const bool table = p.table && p.dtable;
    int lk_min = 0;
    const size_t extra = KeysGeo<DT, 128>::smem(true, p.group, p.reach, p.table, table);
    if (extra <= 227 * 1024) {
        aa_status st = whole<DT, 64>(c, p, -1, n_parts);
        if (st == AA_OK && p.max_k > 64) st = whole<DT, 128>(c, p, 64, n_parts);
        if (st != AA_OK) return st;
        lk_min = 128;
    } else {
        lk_min = -1;
    }
    if (p.max_k <= lk_min) return AA_OK;
    const void* rows = (const void*)grad_rows_kernel<DT>;
    const void* keys = (const void*)grad_keys_kernel<DT, 128, false>;
    const size_t smem_r = GR::smem(p.reach, p.table, table), smem_k = GK::smem(false, p.group, p.reach, p.table, false);
    int cap = 0, cap_k = 0, blocks_q = (int)((p.max_q + 127) / 128), blocks_k = (int)((p.max_k + 127) / 128);
    if (prepare(c, rows, GR::THREADS, smem_r, &cap) != AA_OK || prepare(c, keys, GK::THREADS, smem_k, &cap_k) != AA_OK) return AA_ERR_CUDA;
    if (p.n_seq * blocks_k > 0x7FFFFFFFll) return AA_ERR_UNSUPPORTED;
    int64_t grid = (cap + p.heads - 1) / p.heads;
    if (grid > p.n_seq * blocks_q) grid = p.n_seq * blocks_q;
    if (grid > rel_grad_parts(p.heads)) grid = rel_grad_parts(p.heads);
    if (grid > 0) {
        void* args[] = {&p, &lk_min, &blocks_q, n_parts};
        if (launch_overlapped(c, rows, dim3((unsigned)grid, p.heads), dim3(GR::THREADS), args, smem_r, false) != cudaSuccess) return AA_ERR_CUDA;
        ++c->launches;
    }
    int none = 0;
    if (blocks_k > 0) {
        void* args[] = {&p, &lk_min, &blocks_k, &none};
        if (launch_overlapped(c, keys, dim3((unsigned)(p.n_seq * blocks_k), p.kv_heads), dim3(GK::THREADS), args, smem_k, false) != cudaSuccess) return AA_ERR_CUDA;
        ++c->launches;
    }
    *n_parts += (int)grid;
    return AA_OK;
}

}  // namespace

aa_status launch_rel_attention_grad_mma(aa_ctx_impl* c, const RelParams& p, int* n_parts) {
    return p.dim <= 32 ? backward<32>(c, p, n_parts) : p.dim <= 64 ? backward<64>(c, p, n_parts) : backward<128>(c, p, n_parts);
}

}  // namespace aa
