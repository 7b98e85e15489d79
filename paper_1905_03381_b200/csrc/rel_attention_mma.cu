// Forward pass of the bf16 attention with a relative position bias: a CTA owns NW * 16 query rows of one head and streams 64-key tiles
// of K and V through two shared-memory stages; each warp keeps its 16 rows' queries, running maximum, sum and output in registers.
#include "rel_attention_mma.cuh"

namespace aa {

namespace {

template <int DT, int NW>
__global__ void __launch_bounds__(NW * 32) forward_mma_kernel(RelParams p, int lo, int tiles) {
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
    if (!load_seq(p, sn, s) || max(s.lq, s.lk) <= lo || i0 >= s.lq) return;
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
    fill_bias<kBiasMargin>(p, h, bias);
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
        if (!block_live(p, s, b)) continue;
        const uint32_t Ks = smem_u32(KV + (tile & 1) * 2 * 64 * P), Vs = Ks + 64 * P * 2;
        float t[8][4];
        block_dot<DT, 8>(p, qf, Ks, 0, lane, t);
        block_scores(p, s, bias, b, lane, t);
        block_softmax<DT, 8>(t, m, l, o);
        if (p.drop.thr) block_drops<8>(p, s, key, h, b, lane, [&](int n, int e, bool d) { t[n][e] = d ? 0.0f : t[n][e]; });
        block_times<DT, 8>(p, t, Vs, 0, lane, o);
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
aa_status forward(aa_ctx_impl* c, RelParams p, int lo) {
    const void* kernel = (const void*)forward_mma_kernel<DT, NW>;
    const size_t smem = (size_t)(NW * 16 + 4 * 64) * pitch_of(DT) * 2 + (p.table ? bias_floats(p.reach, kBiasMargin) : 0) * sizeof(float);
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return AA_ERR_CUDA;
    int tiles = (int)((p.max_q + NW * 16 - 1) / (NW * 16));
    if (p.n_seq * tiles > 0x7FFFFFFFll) return AA_ERR_UNSUPPORTED;
    void* args[] = {&p, &lo, &tiles};
    if (launch_overlapped(c, kernel, dim3((unsigned)(p.n_seq * tiles), p.heads), dim3(NW * 32), args, smem, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

template <int DT>
aa_status forward_rows(aa_ctx_impl* c, const RelParams& p, int lo) {
    return p.max_q > 128 ? forward<DT, 8>(c, p, lo) : forward<DT, 4>(c, p, lo);
}

}  // namespace

bool rel_mma_fits(const RelParams& p) {
    const auto ok = [&](const TokArg& a) { return !a.data || ((uintptr_t)a.data % 16 == 0 && a.tok % 8 == 0 && a.head % 8 == 0 && a.tok < (1 << 30)); };
    return p.dim % 8 == 0 && p.dim <= 128 && ok(p.q) && ok(p.k) && ok(p.v) && ok(p.out) && ok(p.dout) && ok(p.dq) && ok(p.dk) && ok(p.dv);
}

aa_status launch_rel_attention_mma(aa_ctx_impl* c, const RelParams& p) {
    if (rel_decode_fits(p)) return launch_rel_decode(c, p);
    int covered = -1;
    const aa_status st = launch_rel_sentences(c, p, &covered);
    if (st != AA_OK || (p.max_q <= covered && p.max_k <= covered)) return st;
    return launch_rel_attention_tc(c, p, covered);
}

}  // namespace aa
