// Backward pass of the bf16 attention with a relative position bias for sequences that do not fit one CTA.
//
// rows kernel: a CTA owns 128 query rows of one head and streams 64-key tiles twice: first the running maximum, sum and D = sum p dp, from
// unrounded probabilities (rounded ones would cost the fp32 bias gradient its digits), then dS, its diagonal sums and dQ.
// keys kernel: a CTA owns 128 keys of one key head and walks the query tiles (64 rows) of the heads that share it with those statistics; dK
// and dV stay in registers, 16 keys a warp.
//
// ds = p (dp - D) and p are rounded to bf16 as operands of the products with K, Q and dO, whose results are bf16; the diagonal sums are
// taken before the rounding.
#include "rel_attention_mma.cuh"

namespace aa {

namespace {

// ------------------------------------------------------------------------------------------------------------ keys kernel

template <int DT>
struct KeysGeo {
    static constexpr int BK = 128, THREADS = 256, P = pitch_of(DT), PP = pitch_of(BK);
    static size_t smem(int reach, bool bias) {
        return (size_t)(2 * BK * P + 2 * 64 * P + 2 * 64 * PP) * 2 + (bias ? bias_floats(reach, kBiasMargin) * sizeof(float) : 0);   // K V, Q dO, P dS, bias
    }
};

// grid (sequences x key blocks, key heads)
template <int DT>
__global__ void __launch_bounds__(256) grad_keys_kernel(RelParams p, int lo, int blocks) {
    using G = KeysGeo<DT>;
    constexpr int P = G::P, PP = G::PP, THREADS = G::THREADS, BK = G::BK;
    extern __shared__ uint4 smem16[];
    uint16_t* Ks = reinterpret_cast<uint16_t*>(smem16);
    uint16_t* Vs = Ks + BK * P;
    uint16_t* Qs = Vs + BK * P;
    uint16_t* Os = Qs + 64 * P;
    uint16_t* Ps = Os + 64 * P;
    uint16_t* Ss = Ps + 64 * PP;
    float* bias = reinterpret_cast<float*>(Ss + 64 * PP);
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t sn = blockIdx.x / blocks;
    const int j0 = (int)(blockIdx.x % blocks) * BK, hk = blockIdx.y;
    Seq s;
    if (!load_seq(p, sn, s) || max(s.lq, s.lk) <= lo || j0 >= s.lk) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, wq = warp & 3, wk = warp >> 2;
    const uint32_t kS = smem_u32(Ks), vS = smem_u32(Vs), qS = smem_u32(Qs), oS = smem_u32(Os), pS = smem_u32(Ps), sS = smem_u32(Ss);
    const uint2 key = p.drop.thr ? instance_key(p.drop, sn) : make_uint2(0, 0);
    const int nk = min(BK, s.lk - j0);
    load_tile_async<BK, DT, THREADS>(p, p.k, hk, s.k0 + j0, nk, Ks);
    load_tile_async<BK, DT, THREADS>(p, p.v, hk, s.k0 + j0, nk, Vs);
    cp_async_commit();
    float gk[DT / 8][4], gv[DT / 8][4];
#pragma unroll
    for (int j = 0; j < DT / 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) gk[j][e] = gv[j][e] = 0.0f;
    for (int h = hk * p.group; h < (hk + 1) * p.group; ++h) {
        __syncthreads();
        fill_bias<kBiasMargin>(p, h, bias);
        for (int i0 = first_query(p, s, j0) / 64 * 64; i0 < s.lq; i0 += 64) {
            const int nq = min(64, s.lq - i0);
            __syncthreads();
            load_tile_async<64, DT, THREADS>(p, p.q, h, s.q0 + i0, nq, Qs);
            load_tile_async<64, DT, THREADS>(p, p.dout, h, s.q0 + i0, nq, Os);
            cp_async_commit();
            const Block b = {i0 + wq * 16, j0 + wk * 64};
            const bool live = block_live(p, s, b);
            RowStats st;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int i = wq * 16 + (lane >> 2) + 8 * r;
                const float4 x = i < nq ? __ldg(p.stats + (int64_t)h * p.q_rows + s.q0 + i0 + i) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                st.m[r] = x.x;
                st.rl[r] = x.y;
                st.D[r] = x.z;
            }
            cp_async_wait<0>();
            __syncthreads();
            uint16_t* prow = Ps + (wq * 16 + (lane >> 2)) * PP + wk * 64 + 2 * (lane & 3);
            uint16_t* srow = Ss + (wq * 16 + (lane >> 2)) * PP + wk * 64 + 2 * (lane & 3);
            if (live) {
                float t[8][4], dp[8][4], unused[2] = {0.0f, 0.0f};
                uint32_t f[DT / 16][4];
                load_frags<DT>(p, f, qS, wq * 16, lane);
                block_dot<DT, 8>(p, f, kS, wk * 64, lane, t);
                load_frags<DT>(p, f, oS, wq * 16, lane);
                block_dot<DT, 8>(p, f, vS, wk * 64, lane, dp);
                block_scores(p, s, bias, b, lane, t);
                block_exp(st.m, t, unused);
                block_drop(p, s, key, h, b, lane, t, dp);
                block_ds(p, st, t, dp);
                store_scores(prow, srow, PP, t, dp);
            } else {
                const float zero[8][4] = {};
                store_scores(prow, srow, PP, zero, zero);
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
        }
    }
    cp_async_wait<0>();
    if (warp * 16 < nk) {
        store_block<DT>(p, p.dk, hk, s.k0 + j0 + warp * 16, nk - warp * 16, lane, gk, p.scale, p.scale);
        store_block<DT>(p, p.dv, hk, s.k0 + j0 + warp * 16, nk - warp * 16, lane, gv, 1.0f, 1.0f);
    }
}

// ------------------------------------------------------------------------------------------------------------ rows kernel

template <int DT>
struct RowsGeo {
    static constexpr int WARPS = 8, THREADS = 256, P = pitch_of(DT);
    static size_t smem(int reach, bool bias, bool table) {
        size_t b = (size_t)(2 * 128 * P + 4 * 64 * P) * 2;                 // Q dO, K V twice
        if (bias) b += bias_floats(reach, kBiasMargin) * sizeof(float);
        if (table) b += (WARPS * kDiagFloats + 2 * reach + 2 * THREADS) * sizeof(float);
        return b;
    }
};

template <int DT>
__global__ void __launch_bounds__(256) grad_rows_kernel(RelParams p, int lo, int blocks, int part0) {
    using G = RowsGeo<DT>;
    constexpr int P = G::P, THREADS = G::THREADS;
    extern __shared__ uint4 smem16[];
    uint16_t* Qs = reinterpret_cast<uint16_t*>(smem16);
    uint16_t* Os = Qs + 128 * P;
    uint16_t* KV = Os + 128 * P;                                           // K0 V0 K1 V1
    float* bias = reinterpret_cast<float*>(KV + 4 * 64 * P);
    const bool want_table = p.table && p.dtable;
    float* stage = bias + (p.table ? bias_floats(p.reach, kBiasMargin) : 0);
    float* bins = stage + (want_table ? G::WARPS * kDiagFloats : 0);
    float* far = bins + 2 * p.reach;                                       // each thread's sums of the far past, then the far future
    grid_dependency_wait();
    grid_dependency_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, h = blockIdx.y, hk = h / p.group;
    fill_bias<kBiasMargin>(p, h, bias);
    if (want_table) {
        for (int i = threadIdx.x; i < 2 * p.reach; i += THREADS) bins[i] = 0.0f;
    }
    float far_neg = 0.0f, far_pos = 0.0f;
    const int64_t items = counted(p.count_dev, p.n_seq) * blocks;
    // later row blocks of a causal sequence see more keys: the longest first
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t sn = item / blocks;
        const int i0 = (blocks - 1 - (int)(item % blocks)) * 128;
        Seq s;
        if (!load_seq(p, sn, s) || max(s.lq, s.lk) <= lo || i0 >= s.lq) continue;
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
            const bool live = block_live(p, s, b);
            float t[8][4], dp[8][4];
            if (live) {
                block_dot<DT, 8>(p, qf, kS, 0, lane, t);
                block_dot<DT, 8>(p, of, vS, 0, lane, dp);
                block_scores(p, s, bias, b, lane, t);
            }
            if (it < n_tiles) {
                if (live) {
                    float ref[2], sum[2] = {0.0f, 0.0f}, dsum[2] = {0.0f, 0.0f}, corr[2];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float top = quad_max(block_max(t, r, m[r]));
                        ref[r] = top == -INFINITY ? 0.0f : top;
                        corr[r] = ex2_approx(m[r] - ref[r]);
                        m[r] = top;
                    }
                    block_exp(ref, t, sum);
                    block_drop(p, s, key, h, b, lane, t, dp);
                    block_dsum(t, dp, dsum);
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        l[r] = fmaf(l[r], corr[r], sum[r]);
                        D[r] = fmaf(D[r], corr[r], dsum[r]);
                    }
                }
                if (it == n_tiles - 1) finish_stats();
                continue;
            }
            const int shift = s.lk - s.lq;
            // distances of the whole CTA's tile: one side's last bucket throughout needs no diagonals
            const bool past = j0 + 63 - (i0 + shift) <= -p.reach, ahead = j0 - (i0 + 127 + shift) >= p.reach;
            if (live) {
                float unused[2] = {0.0f, 0.0f};
                block_exp(st.m, t, unused);
                block_drop(p, s, key, h, b, lane, t, dp);
                block_ds(p, st, t, dp);
                if (want_table && past) far_neg += block_total(dp);
                if (want_table && ahead) far_pos += block_total(dp);
                block_times<DT, 8>(p, dp, kS, 0, lane, gq);
            }
            if (want_table && !past && !ahead) {
                if (!live) {
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
        write_table_part(p, part0 + blockIdx.x, h, bins, 0, 1, THREADS);
    }
}

aa_status prepare(aa_ctx_impl* c, const void* kernel, int threads, size_t smem, int* resident) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return AA_ERR_CUDA;
    *resident = resident_ctas(c, kernel, threads, smem);
    return *resident > 0 ? AA_OK : AA_ERR_CUDA;
}

// Sequences of more than `lo` tokens on either side.
template <int DT>
aa_status backward(aa_ctx_impl* c, RelParams p, int lo, int* n_parts) {
    using GR = RowsGeo<DT>;
    using GK = KeysGeo<DT>;
    const void* rows = (const void*)grad_rows_kernel<DT>;
    const void* keys = (const void*)grad_keys_kernel<DT>;
    const size_t smem_r = GR::smem(p.reach, p.table, p.table && p.dtable), smem_k = GK::smem(p.reach, p.table);
    int cap = 0, cap_k = 0, blocks_q = (int)((p.max_q + 127) / 128), blocks_k = (int)((p.max_k + 127) / 128);
    if (prepare(c, rows, GR::THREADS, smem_r, &cap) != AA_OK || prepare(c, keys, GK::THREADS, smem_k, &cap_k) != AA_OK) return AA_ERR_CUDA;
    if (p.n_seq * blocks_k > 0x7FFFFFFFll) return AA_ERR_UNSUPPORTED;
    int64_t grid = cap / p.heads > 0 ? cap / p.heads : 1;        // one wave
    if (grid > p.n_seq * blocks_q) grid = p.n_seq * blocks_q;
    if (grid > rel_grad_parts(p.heads)) grid = rel_grad_parts(p.heads);
    if (grid > 0) {
        void* args[] = {&p, &lo, &blocks_q, n_parts};
        if (launch_overlapped(c, rows, dim3((unsigned)grid, p.heads), dim3(GR::THREADS), args, smem_r, false) != cudaSuccess) return AA_ERR_CUDA;
        ++c->launches;
    }
    if (blocks_k > 0) {
        void* args[] = {&p, &lo, &blocks_k};
        if (launch_overlapped(c, keys, dim3((unsigned)(p.n_seq * blocks_k), p.kv_heads), dim3(GK::THREADS), args, smem_k, false) != cudaSuccess) return AA_ERR_CUDA;
        ++c->launches;
    }
    *n_parts += (int)grid;
    return AA_OK;
}

}  // namespace

aa_status launch_rel_attention_grad_mma(aa_ctx_impl* c, const RelParams& p, int* n_parts) {
    *n_parts = 0;
    int covered = -1;
    const aa_status st = launch_rel_sentences_grad(c, p, &covered, n_parts);
    if (st != AA_OK || (p.max_q <= covered && p.max_k <= covered)) return st;
    return p.dim <= 32 ? backward<32>(c, p, covered, n_parts) : p.dim <= 64 ? backward<64>(c, p, covered, n_parts) : backward<128>(c, p, covered, n_parts);
}

}  // namespace aa
