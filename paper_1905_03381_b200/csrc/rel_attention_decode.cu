// bf16 attention of a few new tokens over long contexts.  The queries that share a key head (up to 16 per pass: query heads of the group x
// new tokens) are the rows of one matrix instruction, so every key and value is read once per 16 rows; the context is split over CTAs so
// that a single sequence fills the GPU, and the parts (maximum, sum, unnormalised output) are joined by a second small kernel.
//
// Four warps share a 64-key tile, 16 keys each, with running statistics of their own; three tiles of K and V are in flight per CTA.
//
// Bound by latency: launch, first tiles, the warps' and the splits' joins.  Four sequences of 4,001 tokens, 16 heads of 128 on 4 key heads:
// 23.7 us for 33 MB (34 us while every part kept 16 rows and the context's partial sums held 4 splits of a sequence).
#include "rel_attention_mma.cuh"

namespace aa {

namespace {

constexpr int kStages = 3;

struct DecodeParams {
    RelParams p;
    int splits, row_tiles, part_rows;   // rows kept of a pass: 16, or all there can be
    float* part;             // [sequence][key head][row tile][split][part_rows][dim + 2]: o, m, l
};

// Row r of the pass: query head h0 + r / lq, new token r % lq.
template <int DT>
__global__ void __launch_bounds__(128) decode_kernel(DecodeParams d) {
    constexpr int P = pitch_of(DT);
    const RelParams& p = d.p;
    extern __shared__ uint4 smem16[];
    uint16_t* Qs = reinterpret_cast<uint16_t*>(smem16);                    // 16 rows
    uint16_t* KV = Qs + 16 * P;                                            // [stage][K, V]
    float* join = reinterpret_cast<float*>(KV);                            // after the last tile: [warp][16][DT + 2]
    float* bias = reinterpret_cast<float*>(KV + kStages * 2 * 64 * P);     // [head of the group]
    grid_dependency_wait();
    grid_dependency_release();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int split = blockIdx.x, hk = blockIdx.y % p.kv_heads, rt = blockIdx.y / p.kv_heads;
    const int64_t sn = blockIdx.z;
    Seq s;
    if (!load_seq(p, sn, s)) return;
    const int rows = p.group * s.lq, r0 = rt * 16;
    if (r0 >= rows) return;
    const int tiles = (s.lk + 63) >> 6, per = (tiles + d.splits - 1) / d.splits, first = split * per, n_tiles = max(0, min(per, tiles - first));
    const int h0 = hk * p.group;
    const auto load_kv = [&](int i) {
        uint16_t* dst = KV + (i % kStages) * 2 * 64 * P;
        const int at = (first + i) * 64;
        load_tile_async<64, DT, 128>(p, p.k, hk, s.k0 + at, min(64, s.lk - at), dst);
        load_tile_async<64, DT, 128>(p, p.v, hk, s.k0 + at, min(64, s.lk - at), dst + 64 * P);
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) {
        if (i < n_tiles) load_kv(i);
        cp_async_commit();
    }
    for (int i = threadIdx.x; i < 16 * (DT / 8); i += 128) {               // the pass's queries, 8 elements at a time
        const int r = i / (DT / 8), c = i % (DT / 8) * 8, q = r0 + r;
        uint4 x = make_uint4(0, 0, 0, 0);
        if (q < rows && c < p.dim)
            x = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p.q.data) + (s.q0 + q % s.lq) * p.q.tok + (int64_t)(h0 + q / s.lq) * p.q.head + c);
        *reinterpret_cast<uint4*>(Qs + r * P + c) = x;
    }
    const int bias_len = p.table ? bias_floats(p.reach, 0) : 0;
    // the warps share out the heads: one trip to the table, where all warps on one head after the other would make `group` of them
    const int share = max(1, 4 / p.group);
    for (int a = warp / share; a < p.group; a += 4 / share) fill_bias<0>(p, h0 + a, bias + a * bias_len, share, warp % share);
    const uint2 key = p.drop.thr ? instance_key(p.drop, sn) : make_uint2(0, 0);
    // this lane's two rows
    int qi[2], pos[2], lim[2], head[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int q = r0 + g + 8 * r;
        head[r] = q < rows ? q / s.lq : 0;
        qi[r] = q - head[r] * s.lq;
        pos[r] = qi[r] + s.lk - s.lq;
        lim[r] = q < rows ? (p.causal ? min(s.lk, pos[r] + 1) : s.lk) : 0;
    }
    uint32_t qf[DT / 16][4];
    float o[DT / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < DT / 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] = 0.0f;
    for (int i = 0; i < n_tiles; ++i) {
        cp_async_wait<kStages - 2>();
        __syncthreads();
        if (i + kStages - 1 < n_tiles) load_kv(i + kStages - 1);
        cp_async_commit();
        if (i == 0) load_frags<DT>(p, qf, smem_u32(Qs), 0, lane);
        const uint32_t Ks = smem_u32(KV + (i % kStages) * 2 * 64 * P), Vs = Ks + 64 * P * 2;
        const int j0 = (first + i) * 64 + warp * 16;
        if (j0 >= s.lk) continue;
        float x[2][4];
        block_dot<DT, 2>(p, qf, Ks, warp * 16, lane, x);
        const bool near = p.table && (j0 + 15 > (s.lk - s.lq) - p.reach);   // some key within the reach of some query
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = e >> 1, j = j0 + 8 * n + 2 * t + (e & 1);
                float b = 0.0f;
                if (p.table) b = bias[head[r] * bias_len + (near ? min(max(j - pos[r], -p.reach), p.reach) + p.reach : 0)];
                x[n][e] = j < lim[r] ? fmaf(x[n][e], p.scale2, b) : -INFINITY;
            }
        block_softmax<DT, 2>(x, m, l, o);
        if (p.drop.thr) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const Words4 w = draw_block(p.drop, key, draw_row(s, h0 + head[r], qi[r]) + (uint64_t)((j0 >> 5) * 4 + t));
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const uint32_t y = j0 & 16 ? w.w[2 + n] : w.w[n];       // keys 16 (j0 / 16 % 2) + 8 n of the chunk of 32
                    if ((y & 0xFFFFu) < p.drop.thr) x[n][2 * r] = 0.0f;
                    if ((y >> 16) < p.drop.thr) x[n][2 * r + 1] = 0.0f;
                }
            }
        }
        block_times<DT, 2>(p, x, Vs, warp * 16, lane, o);
    }
    cp_async_wait<0>();
    __syncthreads();
    // the warps' parts -> one
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        float* at = join + (warp * 16 + g + 8 * r) * (DT + 2);
#pragma unroll
        for (int j = 0; j < DT / 8; ++j) {
            at[8 * j + 2 * t] = o[j][2 * r];
            at[8 * j + 2 * t + 1] = o[j][2 * r + 1];
        }
        const float sum = quad_sum(l[r]);
        if (t == 0) {
            at[DT] = m[r];
            at[DT + 1] = sum;
        }
    }
    __syncthreads();
    float* part = d.part + (((sn * p.kv_heads + hk) * d.row_tiles + rt) * d.splits + split) * d.part_rows * (p.dim + 2);
    for (int r = warp; r < 16 && r0 + r < rows; r += 4) {
        float mw[4], top = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            mw[w] = join[(w * 16 + r) * (DT + 2) + DT];
            top = fmaxf(top, mw[w]);
        }
        const float ref = top == -INFINITY ? 0.0f : top;
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            mw[w] = ex2_approx(mw[w] - ref);
            sum = fmaf(join[(w * 16 + r) * (DT + 2) + DT + 1], mw[w], sum);
        }
        const int q = r0 + r;
        uint16_t* out = const_cast<uint16_t*>(static_cast<const uint16_t*>(p.out.data)) + (s.q0 + q % s.lq) * p.out.tok + (int64_t)(h0 + q / s.lq) * p.out.head;
        const float f = sum == 0.0f ? 0.0f : p.drop.scale / sum;
        for (int e = lane; e < p.dim; e += 32) {
            float v = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w) v = fmaf(join[(w * 16 + r) * (DT + 2) + e], mw[w], v);
            if (d.splits == 1) store1(out + e, v * f);
            else part[r * (p.dim + 2) + e] = v;
        }
        if (d.splits > 1 && lane == 0) {
            part[r * (p.dim + 2) + p.dim] = top;
            part[r * (p.dim + 2) + p.dim + 1] = sum;
        }
    }
}

// One warp per row adds up the splits.
__global__ void __launch_bounds__(128) decode_join_kernel(DecodeParams d) {
    const RelParams& p = d.p;
    grid_dependency_wait();
    grid_dependency_release();
    const int lane = threadIdx.x & 31, row = blockIdx.x * 4 + (threadIdx.x >> 5), hk = blockIdx.y;
    const int64_t sn = blockIdx.z;
    Seq s;
    if (!load_seq(p, sn, s) || row >= p.group * s.lq) return;
    const int pitch = p.dim + 2;
    const float* part = d.part + ((sn * p.kv_heads + hk) * d.row_tiles + row / 16) * d.splits * d.part_rows * pitch + row % 16 * pitch;
    float top = -INFINITY;
    for (int i = lane; i < d.splits; i += 32) top = fmaxf(top, part[(int64_t)i * d.part_rows * pitch + p.dim]);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    const float ref = top == -INFINITY ? 0.0f : top;
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f}, sum = 0.0f;
#pragma unroll 4
    for (int i = 0; i < d.splits; ++i) {
        const float* at = part + (int64_t)i * d.part_rows * pitch;
        const float w = ex2_approx(at[p.dim] - ref);
        sum = fmaf(at[p.dim + 1], w, sum);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (lane + 32 * k < p.dim) acc[k] = fmaf(at[lane + 32 * k], w, acc[k]);
    }
    const float f = sum == 0.0f ? 0.0f : p.drop.scale / sum;
    uint16_t* out = const_cast<uint16_t*>(static_cast<const uint16_t*>(p.out.data)) + (s.q0 + row % s.lq) * p.out.tok + (int64_t)(hk * p.group + row / s.lq) * p.out.head;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (lane + 32 * k < p.dim) store1(out + lane + 32 * k, acc[k] * f);
}

template <int DT>
aa_status decode(aa_ctx_impl* c, const RelParams& p) {
    DecodeParams d;
    d.p = p;
    const void* kernel = (const void*)decode_kernel<DT>;
    const size_t smem = (size_t)(16 + kStages * 2 * 64) * pitch_of(DT) * 2 + (p.table ? (size_t)p.group * bias_floats(p.reach, 0) : 0) * sizeof(float);
    if (allow_smem(c, kernel, smem) != AA_OK) return AA_ERR_CUDA;
    const int cap = resident_ctas(c, kernel, 128, smem);
    if (cap <= 0) return AA_ERR_CUDA;
    d.row_tiles = (int)((p.group * p.max_q + 15) / 16);
    d.part_rows = p.group * p.max_q < 16 ? (int)(p.group * p.max_q) : 16;
    // one wave of CTAs, at least two tiles each, and as many parts as the context's partial sums hold
    const int64_t units = p.n_seq * p.kv_heads * d.row_tiles, tiles = (p.max_k + 63) / 64;
    int64_t splits = cap / units;
    if (splits > (tiles + 1) / 2) splits = (tiles + 1) / 2;
    const int64_t room = c->partial_floats / (units * d.part_rows * (p.dim + 2));
    if (splits > room) splits = room;
    d.splits = splits > 1 ? (int)splits : 1;
    d.part = c->partials;
    void* args[] = {&d};
    if (launch_overlapped(c, kernel, dim3(d.splits, p.kv_heads * d.row_tiles, (unsigned)p.n_seq), dim3(128), args, smem, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    if (d.splits == 1) return AA_OK;
    if (launch_overlapped(c, (const void*)decode_join_kernel, dim3((unsigned)((p.group * p.max_q + 3) / 4), p.kv_heads, (unsigned)p.n_seq), dim3(128), args, 0, false) !=
        cudaSuccess)
        return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

}  // namespace

// Few rows: the passes of 16 rows over a context cost less than tiles of 64 rows that are mostly empty, and the split keeps the GPU busy.
bool rel_decode_fits(const RelParams& p) {
    return p.max_q * p.group <= 32 && p.max_q <= 16 && p.max_k > 128 && p.n_seq <= 65535 && p.kv_heads * ((p.max_q * p.group + 15) / 16) <= 65535 &&
           (size_t)p.group * bias_floats(p.reach, 0) * sizeof(float) <= 96 * 1024;
}

aa_status launch_rel_decode(aa_ctx_impl* c, const RelParams& p) {
    return p.dim <= 32 ? decode<32>(c, p) : p.dim <= 64 ? decode<64>(c, p) : decode<128>(c, p);
}

}  // namespace aa
