// Forward pass of the bf16 attention with a relative position bias: a CTA owns NW * 16 query rows of one head and streams 64-key tiles
// of K and V through two shared-memory stages; each warp keeps its 16 rows' queries, running maximum, sum and output in registers.
#include "rel_attention_mma.cuh"

namespace aa {

namespace {

template <int DT>
struct FwdTile {
    static constexpr int P = pitch_of(DT);
    static constexpr int kKv = 64 * P;                     // elements of one K or V stage
};

template <int DT, int NW>
__global__ void __launch_bounds__(NW * 32) forward_mma_kernel(RelParams p, int tiles) {
    constexpr int THREADS = NW * 32, ROWS = NW * 16, P = pitch_of(DT);
    extern __shared__ uint4 smem16[];
    uint16_t* Qs = reinterpret_cast<uint16_t*>(smem16);
    uint16_t* KV = Qs + ROWS * P;                          // K0 V0 K1 V1
    float* bias = reinterpret_cast<float*>(KV + 4 * 64 * P);
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t sn = blockIdx.x / tiles;
    const int i0 = (int)(blockIdx.x % tiles) * ROWS, h = blockIdx.y, hk = h / p.group;
    Seq s;
    if (!load_seq(p, sn, s) || i0 >= s.lq) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int nq = min(ROWS, s.lq - i0), end = keys_seen(p, s, i0 + nq), n_tiles = (end + 63) / 64;
    const auto load_kv = [&](int tile) {
        uint16_t* dst = KV + (tile & 1) * 2 * 64 * P;
        load_tile_async<64, DT, THREADS>(p, p.k, hk, s.k0 + tile * 64, min(64, s.lk - tile * 64), dst);
        load_tile_async<64, DT, THREADS>(p, p.v, hk, s.k0 + tile * 64, min(64, s.lk - tile * 64), dst + 64 * P);
    };
    load_tile_async<ROWS, DT, THREADS>(p, p.q, h, s.q0 + i0, nq, Qs);
    if (n_tiles > 0) load_kv(0);
    cp_async_commit();
    const uint2 key = p.drop.thr ? instance_key(p.drop, sn) : make_uint2(0, 0);
    fill_bias(p, h, bias);
    uint32_t qf[DT / 16][4];
    float o[DT / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < DT / 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[j][e] = 0.0f;
    for (int tile = 0; tile < n_tiles; ++tile) {
        cp_async_wait<0>();
        __syncthreads();                                   // this tile is there, the other stage's readers are done
        if (tile + 1 < n_tiles) {
            load_kv(tile + 1);
            cp_async_commit();
        }
        if (tile == 0) load_frags<DT>(p, qf, smem_u32(Qs), warp * 16, lane);
        const Block b = {i0 + warp * 16, tile * 64};
        const int n16 = block_groups(p, s, b);
        if (n16 == 0) continue;
        const uint32_t Ks = smem_u32(KV + (tile & 1) * 2 * 64 * P), Vs = Ks + 64 * P * 2;
        float t[8][4];
        block_dot<DT>(p, qf, Ks, 0, n16, lane, t);
        block_scores(p, s, bias, b, lane, t);
        const uint32_t dropped = p.drop.thr ? block_drops(p, s, key, h, b, lane) : 0u;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float top = m[r];
#pragma unroll
            for (int n = 0; n < 8; ++n) top = fmaxf(top, fmaxf(t[n][2 * r], t[n][2 * r + 1]));
            top = quad_max(top);
            const float ref = top == -INFINITY ? 0.0f : top, corr = ex2_approx(m[r] - ref);
            float sum = 0.0f;
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const float e = ex2_approx(t[n][2 * r + c] - ref);
                    sum += e;
                    t[n][2 * r + c] = (dropped >> (4 * n + 2 * r + c)) & 1u ? 0.0f : e;
                }
            l[r] = fmaf(l[r], corr, sum);                  // this lane's part of the row
            m[r] = top;
#pragma unroll
            for (int j = 0; j < DT / 8; ++j) {
                o[j][2 * r] *= corr;
                o[j][2 * r + 1] *= corr;
            }
        }
        // probabilities (at most 1) rounded to bf16 as the left operand: relative 2^-9 per term of the output, which is bf16 itself
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (k >= n16) continue;
            const uint32_t a[4] = {pack_bf16(t[2 * k][0], t[2 * k][1]), pack_bf16(t[2 * k][2], t[2 * k][3]), pack_bf16(t[2 * k + 1][0], t[2 * k + 1][1]),
                                   pack_bf16(t[2 * k + 1][2], t[2 * k + 1][3])};
#pragma unroll
            for (int j = 0; j < DT / 16; ++j) {
                if (DT > 64 && j * 16 >= p.dim) continue;
                uint32_t v[4];
                ldsm4t(v, frag_rows<P>(Vs, k * 16, j * 16, lane));
                mma16816(o[2 * j], a, v[0], v[1]);
                mma16816(o[2 * j + 1], a, v[2], v[3]);
            }
        }
    }
    cp_async_wait<0>();                                    // a tile that sees no key has loaded its queries all the same
    float f[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const float sum = quad_sum(l[r]);
        f[r] = sum == 0.0f ? 0.0f : p.drop.scale / sum;
    }
    store_block<DT>(p, p.out, h, s.q0 + i0 + warp * 16, nq - warp * 16, lane, o, f[0], f[1]);
}

template <int DT, int NW>
aa_status forward(aa_ctx_impl* c, RelParams p) {
    const void* kernel = (const void*)forward_mma_kernel<DT, NW>;
    const size_t smem = (size_t)(NW * 16 + 4 * 64) * pitch_of(DT) * 2 + (p.table ? 2 * p.reach + 1 : 0) * sizeof(float);
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return AA_ERR_CUDA;
    int tiles = (int)((p.max_q + NW * 16 - 1) / (NW * 16));
    if (p.n_seq * tiles > 0x7FFFFFFFll) return AA_ERR_UNSUPPORTED;
    void* args[] = {&p, &tiles};
    if (launch_overlapped(c, kernel, dim3((unsigned)(p.n_seq * tiles), p.heads), dim3(NW * 32), args, smem, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

template <int DT>
aa_status forward_rows(aa_ctx_impl* c, const RelParams& p) {
    return p.max_q > 128 ? forward<DT, 8>(c, p) : forward<DT, 4>(c, p);
}

}  // namespace

bool rel_mma_fits(const RelParams& p) {
    const auto ok = [&](const TokArg& a) { return !a.data || ((uintptr_t)a.data % 16 == 0 && a.tok % 8 == 0 && a.head % 8 == 0); };
    return p.dim % 8 == 0 && p.dim <= 128 && ok(p.q) && ok(p.k) && ok(p.v) && ok(p.out) && ok(p.dout) && ok(p.dq) && ok(p.dk) && ok(p.dv);
}

aa_status launch_rel_attention_mma(aa_ctx_impl* c, const RelParams& p) {
    return p.dim <= 32 ? forward_rows<32>(c, p) : p.dim <= 64 ? forward_rows<64>(c, p) : forward_rows<128>(c, p);
}

}  // namespace aa
