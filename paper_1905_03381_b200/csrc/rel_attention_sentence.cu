// bf16 attention with a relative position bias for sequences of at most LT = 64 or 128 tokens on both sides, forward and backward.
//
// A sentence's queries, keys and values of one head fit into shared memory together: persistent CTAs take one sentence after the other, and
// the bias by distance is laid out once per CTA.  A warp works on a strip of 16 query rows in steps of 16 keys.  Backward: strips leave p
// and dS in shared memory (bf16), then warps contract them for 16 keys (dV, dK) and 16 rows (dQ): five products, each operand read from
// memory once.  The bias gradient is added up along the diagonals of the unrounded dS, in a fixed order.
//
// Bound by unequal CTAs and by what a CTA waits for: sentences are dealt out by a fixed stride, whatever their length, so that the busiest SM is
// active 1.3 to 1.5 times as long as the mean one, and the forward pass fetches a sentence only after the last one; the issue slots are in use for
// 22 to 34 %, the tensor pipe for 5 to 16 %.  368 sentences of 8 to 128 tokens, 8 heads of 64: forward 56 us (1.9 TB/s), forward and every
// gradient, causal, with dropout 242 us.
#include "rel_attention_mma.cuh"

namespace aa {

namespace {

// The sentences of this class, lo < max(Lq, Lk) <= LT, in steps of the grid: a lane looks one candidate up (offsets, instance key), the warp
// takes the lanes' finds in order, so that a sentence costs a few shuffles.
struct Item {
    bool live;
    int64_t n;
    Seq s;
    uint2 key;
};
template <int LT>
struct Walk {
    const RelParams& p;
    int lo, lane;
    int64_t base, count, step;       // candidates base + lane * step
    unsigned found;
    Seq s;
    uint2 key;
    __device__ Walk(const RelParams& params, int low) : p(params), lo(low), lane(threadIdx.x & 31), base(blockIdx.x), count(counted(params.count_dev, params.n_seq)), step(gridDim.x) {
        look();
    }
    __device__ __forceinline__ void look() {
        const int64_t n = base + lane * step;
        bool ok = false;
        s = Seq{0, 0, 0, 0};
        key = make_uint2(0, 0);
        if (n < count && load_seq(p, n, s)) {
            const int len = max(s.lq, s.lk);
            ok = len > lo && len <= LT;
            if (ok && p.drop.thr) key = instance_key(p.drop, n);
        }
        found = __ballot_sync(0xFFFFFFFFu, ok);
    }
    __device__ __forceinline__ Item next() {
        Item it;
        while (!found && base + 32 * step < count) {
            base += 32 * step;
            look();
        }
        it.live = found != 0;
        const int from = it.live ? __ffs(found) - 1 : 0;
        found &= found - 1;
        it.n = base + from * step;
        it.s.q0 = __shfl_sync(0xFFFFFFFFu, (int)s.q0, from);
        it.s.k0 = __shfl_sync(0xFFFFFFFFu, (int)s.k0, from);
        it.s.lq = __shfl_sync(0xFFFFFFFFu, s.lq, from);
        it.s.lk = __shfl_sync(0xFFFFFFFFu, s.lk, from);
        it.key.x = __shfl_sync(0xFFFFFFFFu, key.x, from);
        it.key.y = __shfl_sync(0xFFFFFFFFu, key.y, from);
        return it;
    }
};

// ---------------------------------------------------------------------------------------------------------------- forward

template <int DT, int LT>
__global__ void __launch_bounds__(128, DT == 128 ? 2 : 4) sentence_forward_kernel(RelParams p, int lo) {
    constexpr int THREADS = 128, P = pitch_of(DT), TILE = LT * P;
    extern __shared__ uint4 smem16[];
    uint16_t* tiles = reinterpret_cast<uint16_t*>(smem16);                 // Q, K, V
    float* bias = reinterpret_cast<float*>(tiles + 3 * TILE);
    grid_dependency_wait();
    grid_dependency_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, h = blockIdx.y, hk = h / p.group;
    const uint32_t qS = smem_u32(tiles), kS = qS + TILE * 2, vS = kS + TILE * 2;
    Walk<LT> walk(p, lo);
    Item it = walk.next();
    if (!it.live) return;
    const auto load = [&](const Item& x) {
        load_tile_async<LT, DT, THREADS, 16>(p, p.q, h, x.s.q0, x.s.lq, tiles);
        load_tile_async<LT, DT, THREADS, 32>(p, p.k, hk, x.s.k0, x.s.lk, tiles + TILE);
        load_tile_async<LT, DT, THREADS, 32>(p, p.v, hk, x.s.k0, x.s.lk, tiles + 2 * TILE);
        cp_async_commit();
    };
    load(it);
    fill_bias<kBiasMargin>(p, h, bias);
    while (it.live) {
        const Seq& s = it.s;
        cp_async_wait<0>();
        __syncthreads();
        // strips: the last (under a causal mask longest) four first, then the rest in the opposite order: long ones pair with short ones
        const int strips = (s.lq + 15) >> 4;
#pragma unroll 1
        for (int round = 0; round < LT / 64; ++round) {
            const int strip = round == 0 ? strips - 1 - warp : strips - 8 + warp;
            if (strip < 0 || (round == 1 && strip > strips - 5)) continue;
            const int i0 = strip * 16;
            float o[DT / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
#pragma unroll
            for (int j = 0; j < DT / 8; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[j][e] = 0.0f;
            uint32_t qf[DT / 16][4];
            load_frags<DT>(p, qf, qS, i0, lane);
            const int end = keys_seen(p, s, min(i0 + 16, s.lq));
#pragma unroll 1
            for (int j0 = 0; j0 < end; j0 += 32) {
                const Block b = {i0, j0};
                float t[4][4];
                block_dot<DT, 4>(p, qf, kS, j0, lane, t);
                block_scores(p, s, bias, b, lane, t);
                block_softmax<DT, 4>(t, m, l, o);
                if (p.drop.thr) block_drops<4>(p, s, it.key, h, b, lane, [&](int n, int e, bool d) { t[n][e] = d ? 0.0f : t[n][e]; });
                block_times<DT, 4>(p, t, vS, j0, lane, o);
            }
            float f[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float sum = quad_sum(l[r]);
                f[r] = sum == 0.0f ? 0.0f : p.drop.scale / sum;
            }
            store_block<DT>(p, p.out, h, s.q0 + i0, s.lq - i0, lane, o, f[0], f[1]);
        }
        it = walk.next();
        __syncthreads();                                                   // the tiles are free
        if (it.live) load(it);
    }
}

// --------------------------------------------------------------------------------------------------------------- backward

template <int DT, int LT>
struct BackGeo {
    static constexpr int HALVES = LT / 64, WARPS = LT / 16 * HALVES, THREADS = WARPS * 32;
    static constexpr int P = pitch_of(DT), TILE = LT * P, PP = 2 * LT + 8;  // a row of the second area: p, dS, an odd number of chunks
    static constexpr int SLOTS = LT == 128 ? 6 : 4;                         // K Q V dO, and a second K and Q
    static_assert(16 * PP * 2 >= HALVES * kDiagFloats * 4, "a strip's rows hold its staged diagonals");
    static constexpr int BIN_FAR = 2 * THREADS;
    static size_t smem(int group, int reach, bool bias, bool table) {
        size_t b = (size_t)(SLOTS * TILE + LT * PP) * 2 + LT * HALVES * 3 * sizeof(float);
        if (bias) b += (size_t)group * bias_floats(reach, kBiasMargin) * sizeof(float);
        if (table) b += (size_t)group * (WARPS * kDiagAccFloats + 2 * reach + BIN_FAR) * sizeof(float);
        return b + 16;
    }
};

// A half of a strip that sees no key: what it adds to the row statistics.
template <int LT>
__device__ __forceinline__ void join_nothing(const Block b, int lane, float* stat) {
    if (LT == 64) return;
    float* mine = stat + (b.j0 / 64 * LT + b.i0 + (lane >> 2)) * 3;
    if ((lane & 3) == 0)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            mine[24 * r] = -INFINITY;
            mine[24 * r + 1] = mine[24 * r + 2] = 0.0f;
        }
    asm volatile("bar.sync %0, 64;" ::"r"(1 + (b.i0 >> 4)) : "memory");
}

// p and dS of a warp's block, from scores to shared memory, with the strip's row statistics.
template <int DT, int LT, int NT>
__device__ __forceinline__ void strip_scores(const RelParams& p, const Seq& s, uint2 key, int h, const Block b, int lane, uint32_t qS, uint32_t kS, uint32_t oS, uint32_t vS,
                                             const float* bias, float* stat, uint16_t* PS, float* dacc) {
    constexpr int HALVES = LT / 64, PP = BackGeo<DT, LT>::PP;
    float t[NT][4], dp[NT][4];
    RowStats st;
    float m[2], l[2] = {0.0f, 0.0f}, D[2] = {0.0f, 0.0f};
    {
        uint32_t f[DT / 16][4];
        load_frags<DT>(p, f, qS, b.i0, lane);
        block_dot<DT, NT>(p, f, kS, b.j0, lane, t);
    }
    block_scores(p, s, bias, b, lane, t);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        m[r] = quad_max(block_max(t, r, -INFINITY));
        st.m[r] = m[r] == -INFINITY ? 0.0f : m[r];
    }
    block_exp(st.m, t, l);
    {
        uint32_t f[DT / 16][4];
        load_frags<DT>(p, f, oS, b.i0, lane);
        block_dot<DT, NT>(p, f, vS, b.j0, lane, dp);
    }
    block_drop(p, s, key, h, b, lane, t, dp);
    block_dsum(t, dp, D);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        l[r] = quad_sum(l[r]);
        D[r] = quad_sum(D[r]);
    }
    float own[2] = {1.0f, 1.0f};
    if (HALVES > 1) {                                                      // join with the strip's other keys
        const int half = b.j0 / 64;
        float* mine = stat + (half * LT + b.i0 + (lane >> 2)) * 3;
        const float* other = stat + ((half ^ 1) * LT + b.i0 + (lane >> 2)) * 3;
        if ((lane & 3) == 0)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                mine[24 * r] = m[r];
                mine[24 * r + 1] = l[r];
                mine[24 * r + 2] = D[r];
            }
        asm volatile("bar.sync %0, 64;" ::"r"(1 + (b.i0 >> 4)) : "memory");
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const float mo = other[24 * r], top = fmaxf(m[r], mo), ref = top == -INFINITY ? 0.0f : top, fo = ex2_approx(mo - ref);
            own[r] = ex2_approx(m[r] - ref);
            l[r] = l[r] * own[r] + other[24 * r + 1] * fo;
            D[r] = D[r] * own[r] + other[24 * r + 2] * fo;
        }
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const float rl = l[r] == 0.0f ? 0.0f : 1.0f / l[r];
        st.D[r] = D[r] * rl;
        st.rl[r] = rl * own[r];
    }
    block_ds(p, st, t, dp);
    if (dacc) add_diagonals(dacc, dp, lane);
    uint16_t* row = PS + (b.i0 + (lane >> 2)) * PP + b.j0 + 2 * (lane & 3);
    store_scores(row, row + LT, PP, t, dp);
}

// A strip's rows belong to HALVES warps, one per 64 keys, which join their row statistics.  SHARED: several query heads per key head.
// Dropping LT = 64 to four warps keeps three CTAs on an SM; LT = 128 fills it with 16 warps and fetches the next sentence's K and Q meanwhile,
// its V as soon as this one's is used up, its dO last.
template <int DT, int LT, bool SHARED>
__global__ void __launch_bounds__(LT * 2 * (LT / 64), LT == 64 && DT <= 64 ? (SHARED ? 2 : 3) : 1) sentence_backward_kernel(RelParams p, int lo, int part0) {
    using G = BackGeo<DT, LT>;
    constexpr int THREADS = G::THREADS, P = G::P, PP = G::PP, TILE = G::TILE, WARPS = G::WARPS, HALVES = G::HALVES;
    constexpr bool AHEAD = G::SLOTS == 6 && !SHARED;
    extern __shared__ uint4 smem16[];
    uint16_t* tiles = reinterpret_cast<uint16_t*>(smem16);                 // K, Q, V, dO, K', Q'
    uint16_t* PS = tiles + G::SLOTS * TILE;
    const int group = SHARED ? p.group : 1;
    const bool want_table = p.table && p.dtable;
    float* dacc = reinterpret_cast<float*>(PS + LT * PP);                  // [head of the group][warp] diagonals of blocks at one distance
    float* stat = dacc + (want_table ? group * WARPS * kDiagAccFloats : 0);  // [half][row][m, l, D]
    float* bias = stat + LT * HALVES * 3;                                  // [head of the group]
    const int bias_len = p.table ? bias_floats(p.reach, kBiasMargin) : 0, bin_len = 2 * p.reach + G::BIN_FAR;
    float* bins = bias + group * bias_len;                                 // [head of the group]: by distance, then each thread's far past, far future
    grid_dependency_wait();
    grid_dependency_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, hk = blockIdx.y, h0 = hk * group;
    const int strip = warp & (LT / 16 - 1), half = warp / (LT / 16), i0 = strip * 16, j0 = half * 64;
    Walk<LT> walk(p, lo);
    Item it = walk.next();
    int slot = 0;                                                          // 0 or 4: where this sentence's K and Q are
    const auto load = [&](const TokArg& t, int head, int64_t row0, int n, int at) { load_tile_async<LT, DT, THREADS, 32>(p, t, head, row0, n, tiles + at * TILE); };
    if (it.live) {
        load(p.k, hk, it.s.k0, it.s.lk, 0);
        load(p.q, h0, it.s.q0, it.s.lq, 1);
        cp_async_commit();
        load(p.v, hk, it.s.k0, it.s.lk, 2);
        load(p.dout, h0, it.s.q0, it.s.lq, 3);
        cp_async_commit();
    }
    for (int a = 0; a < group; ++a) fill_bias<kBiasMargin>(p, h0 + a, bias + a * bias_len);
    if (want_table) {
        for (int i = threadIdx.x; i < group * bin_len; i += THREADS) bins[i] = 0.0f;
        for (int i = threadIdx.x; i < group * WARPS * kDiagAccFloats; i += THREADS) dacc[i] = 0.0f;
    }
    const uint32_t tS = smem_u32(tiles), vS = tS + 2 * TILE * 2, oS = tS + 3 * TILE * 2, psS = smem_u32(PS);
    // The accumulated diagonals belong to one shift Lk - Lq (0 throughout for self-attention); another one folds them into the bins:
    // a thread per diagonal key - row = d adds up the warps' staged columns.  p and dS are not in use; ends with a barrier.
    const auto fold = [&](int shift) {
        for (int a = 0; a < group; ++a) {
            __syncthreads();
            stage_accumulated(reinterpret_cast<float*>(PS + i0 * PP) + half * kDiagFloats, dacc + (a * WARPS + warp) * kDiagAccFloats, lane);
            __syncthreads();
            float* bh = bins + a * bin_len;
            for (int d = (int)threadIdx.x - (LT - 1); d < LT; d += THREADS) {
                float sum = 0.0f;
#pragma unroll 4
                for (int w = 0; w < WARPS; ++w) {
                    const int st = w & (LT / 16 - 1), ha = w / (LT / 16), col = d + 16 * st - 64 * ha + 15;
                    if (col >= 0 && col < kDiagCols) sum += diagonal_sum(reinterpret_cast<const float*>(PS + st * 16 * PP) + ha * kDiagFloats, col);
                }
                const int delta = d - shift;
                if (delta <= -p.reach) bh[2 * p.reach + threadIdx.x] += sum;
                else if (delta >= p.reach || (!p.bidir && delta > 0)) bh[2 * p.reach + THREADS + threadIdx.x] += sum;
                else bh[delta + p.reach] += sum;
            }
        }
        __syncthreads();
    };
    int acc_shift = it.s.lk - it.s.lq;
    while (it.live) {
        const Item nx = walk.next();
        const Seq& s = it.s;
        const uint32_t kS = tS + slot * TILE * 2, qS = kS + TILE * 2;
        const int shift = s.lk - s.lq;
        if (want_table && shift != acc_shift) {
            fold(acc_shift);
            acc_shift = shift;
        }
        float ga[DT / 8][4], gb[HALVES == 1 ? DT / 8 : 1][4];              // dV and dK of 16 keys; with two halves one of them
#pragma unroll
        for (int j = 0; j < DT / 8; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                ga[j][e] = 0.0f;
                if (HALVES == 1) gb[j][e] = 0.0f;
            }
#pragma unroll 1
        for (int a = 0; a < group; ++a) {
            const int h = h0 + a;
            if (AHEAD) {
                if (nx.live) {                                             // K' and Q': one group, empty at the end of the walk
                    load(p.k, hk, nx.s.k0, nx.s.lk, slot ^ 4);
                    load(p.q, h0, nx.s.q0, nx.s.lq, (slot ^ 4) + 1);
                }
                cp_async_commit();
                cp_async_wait<1>();
            } else {
                cp_async_wait<0>();
            }
            __syncthreads();
            const int end = i0 < s.lq ? keys_seen(p, s, min(i0 + 16, s.lq)) : 0;      // keys this strip sees
            if (i0 < s.lq) {
                if (end <= j0) join_nothing<LT>(Block{i0, j0}, lane, stat);
                else if (end - j0 > 32) strip_scores<DT, LT, 8>(p, s, it.key, h, Block{i0, j0}, lane, qS, kS, oS, vS, bias + a * bias_len, stat, PS, want_table ? dacc + (a * WARPS + warp) * kDiagAccFloats : nullptr);
                else strip_scores<DT, LT, 4>(p, s, it.key, h, Block{i0, j0}, lane, qS, kS, oS, vS, bias + a * bias_len, stat, PS, want_table ? dacc + (a * WARPS + warp) * kDiagAccFloats : nullptr);
            }
            __syncthreads();
            if (AHEAD && nx.live) load(p.v, hk, nx.s.k0, nx.s.lk, 2);
            // dV += P^T dO, dK += dS^T Q for 16 keys: the strips that see the first of them, in order
            if (i0 < s.lk) {
#pragma unroll
                for (int k = 0; k < LT / 16; ++k) {
                    if (k * 16 >= s.lq || (p.causal && min(k * 16 + 16, s.lq) + shift <= i0)) continue;
                    uint32_t x[4], y[4];
                    ldsm4t(x, frag_trans<PP>(psS, k * 16, i0 + (HALVES > 1 && half ? LT : 0), lane));
                    if (HALVES == 1) ldsm4t(y, frag_trans<PP>(psS, k * 16, i0 + LT, lane));
                    const uint32_t right = HALVES > 1 && half ? qS : oS;
#pragma unroll
                    for (int j = 0; j < DT / 16; ++j) {
                        if (DT > 64 && j * 16 >= p.dim) continue;
                        uint32_t z[4];
                        ldsm4t(z, frag_rows<P>(right, k * 16, j * 16, lane));
                        mma16816(ga[2 * j], x, z[0], z[1]);
                        mma16816(ga[2 * j + 1], x, z[2], z[3]);
                        if (HALVES == 1) {
                            ldsm4t(z, frag_rows<P>(qS, k * 16, j * 16, lane));
                            mma16816(gb[2 * j], y, z[0], z[1]);
                            mma16816(gb[2 * j + 1], y, z[2], z[3]);
                        }
                    }
                }
            }
            if (i0 < s.lq) {                                               // dQ = dS K: this strip, the half's columns
                constexpr int NJ = DT / 16 / HALVES;
                float gq[2 * NJ][4];
#pragma unroll
                for (int j = 0; j < 2 * NJ; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) gq[j][e] = 0.0f;
                const int c0 = half * NJ * 16;
#pragma unroll
                for (int k = 0; k < LT / 16; ++k) {
                    if (k * 16 >= end) continue;
                    uint32_t x[4];
                    ldsm4(x, frag_rows<PP>(psS, i0, LT + k * 16, lane));
#pragma unroll
                    for (int j = 0; j < NJ; ++j) {
                        if (DT > 64 && j * 16 >= p.dim) continue;
                        uint32_t z[4];
                        ldsm4t(z, frag_rows<P>(kS, k * 16, c0 + j * 16, lane));
                        mma16816(gq[2 * j], x, z[0], z[1]);
                        mma16816(gq[2 * j + 1], x, z[2], z[3]);
                    }
                }
                store_block<2 * NJ * 8>(p, p.dq, h, s.q0 + i0, s.lq - i0, lane, gq, p.scale, p.scale, c0);
            }
            __syncthreads();                                               // tiles, p and dS are free
            if (SHARED && a + 1 < group) {
                load(p.q, h + 1, s.q0, s.lq, slot + 1);
                load(p.dout, h + 1, s.q0, s.lq, 3);
                cp_async_commit();
            }
        }
        if (AHEAD) {
            if (nx.live) load(p.dout, h0, nx.s.q0, nx.s.lq, 3);
            cp_async_commit();                                             // V' and dO'
            slot ^= 4;
        } else if (nx.live) {
            load(p.k, hk, nx.s.k0, nx.s.lk, 0);
            load(p.q, h0, nx.s.q0, nx.s.lq, 1);
            load(p.v, hk, nx.s.k0, nx.s.lk, 2);
            load(p.dout, h0, nx.s.q0, nx.s.lq, 3);
            cp_async_commit();
        }
        if (i0 < s.lk) {
            if (HALVES == 1) {
                store_block<DT>(p, p.dv, hk, s.k0 + i0, s.lk - i0, lane, ga, 1.0f, 1.0f, 0);
                store_block<HALVES == 1 ? DT : 8>(p, p.dk, hk, s.k0 + i0, s.lk - i0, lane, gb, p.scale, p.scale, 0);
            } else {
                const float f = half ? p.scale : 1.0f;
                store_block<DT>(p, half ? p.dk : p.dv, hk, s.k0 + i0, s.lk - i0, lane, ga, f, f, 0);
            }
        }
        it = nx;
    }
    cp_async_wait<0>();
    if (want_table) {
        fold(acc_shift);
        for (int a = 0; a < group; ++a) write_table_part(p, part0 + blockIdx.x, h0 + a, bins + a * bin_len, 0, 1, THREADS);
    }
}

aa_status prepare(aa_ctx_impl* c, const void* kernel, int threads, size_t smem, int* resident) {
    if (allow_smem(c, kernel, smem) != AA_OK) return AA_ERR_CUDA;
    *resident = resident_ctas(c, kernel, threads, smem);
    return *resident > 0 ? AA_OK : AA_ERR_CUDA;
}

template <int DT, int LT>
aa_status forward(aa_ctx_impl* c, RelParams p, int lo) {
    const void* kernel = (const void*)sentence_forward_kernel<DT, LT>;
    int cap = 0;
    const size_t smem = (size_t)3 * LT * pitch_of(DT) * 2 + (p.table ? bias_floats(p.reach, kBiasMargin) : 0) * sizeof(float);
    if (prepare(c, kernel, 128, smem, &cap) != AA_OK) return AA_ERR_CUDA;
    int64_t grid = cap / p.heads > 0 ? cap / p.heads : 1;
    if (grid > p.n_seq) grid = p.n_seq;
    void* args[] = {&p, &lo};
    if (launch_overlapped(c, kernel, dim3((unsigned)grid, p.heads), dim3(128), args, smem, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

template <int DT, int LT, bool SHARED>
aa_status backward(aa_ctx_impl* c, RelParams p, int lo, int* part0) {
    using G = BackGeo<DT, LT>;
    const void* kernel = (const void*)sentence_backward_kernel<DT, LT, SHARED>;
    int cap = 0;
    const size_t smem = G::smem(p.group, p.reach, p.table, p.table && p.dtable);
    if (prepare(c, kernel, G::THREADS, smem, &cap) != AA_OK) return AA_ERR_CUDA;
    int64_t grid = cap / p.kv_heads > 0 ? cap / p.kv_heads : 1;
    if (grid > p.n_seq) grid = p.n_seq;
    if (grid > rel_grad_parts(p.heads)) grid = rel_grad_parts(p.heads);
    void* args[] = {&p, &lo, part0};
    if (launch_overlapped(c, kernel, dim3((unsigned)grid, p.kv_heads), dim3(G::THREADS), args, smem, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    *part0 += (int)grid;
    return AA_OK;
}

template <int DT, int LT>
aa_status backward(aa_ctx_impl* c, const RelParams& p, int lo, int* part0) {
    return p.group > 1 ? backward<DT, LT, true>(c, p, lo, part0) : backward<DT, LT, false>(c, p, lo, part0);
}

template <int DT>
aa_status forward_classes(aa_ctx_impl* c, const RelParams& p, int* covered) {
    *covered = p.max_q > 64 || p.max_k > 64 ? 128 : 64;
    return *covered == 128 ? forward<DT, 128>(c, p, -1) : forward<DT, 64>(c, p, -1);
}

template <int DT>
aa_status backward_classes(aa_ctx_impl* c, const RelParams& p, int* covered, int* n_parts) {
    const bool table = p.table && p.dtable;
    *covered = -1;
    // the bias and the bins of every head of a group are in shared memory: a large group or reach leaves the sentences to the long kernels
    if (BackGeo<DT, 64>::smem(p.group, p.reach, p.table, table) > 227 * 1024) return AA_OK;
    aa_status st = backward<DT, 64>(c, p, -1, n_parts);
    *covered = 64;
    if constexpr (DT <= 64) {       // at a width of 128 two key blocks of scores and 16 keys' gradients do not fit the registers
        if (st == AA_OK && (p.max_q > 64 || p.max_k > 64) && BackGeo<DT, 128>::smem(p.group, p.reach, p.table, table) <= 227 * 1024) {
            st = backward<DT, 128>(c, p, 64, n_parts);
            *covered = 128;
        }
    }
    return st;
}

}  // namespace

aa_status launch_rel_sentences(aa_ctx_impl* c, const RelParams& p, int* covered) {
    return p.dim <= 32 ? forward_classes<32>(c, p, covered) : p.dim <= 64 ? forward_classes<64>(c, p, covered) : forward_classes<128>(c, p, covered);
}
aa_status launch_rel_sentences_grad(aa_ctx_impl* c, const RelParams& p, int* covered, int* n_parts) {
    return p.dim <= 32   ? backward_classes<32>(c, p, covered, n_parts)
           : p.dim <= 64 ? backward_classes<64>(c, p, covered, n_parts)
                         : backward_classes<128>(c, p, covered, n_parts);
}

}  // namespace aa
