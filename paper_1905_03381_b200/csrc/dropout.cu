// Dropout whose mask is a function of (seed, step, instance id, site, element): out = residual + mask * scale * x.
//
// One Philox block decides eight elements (16 bits each).  Work is handed out in units of one row's chunk of kGroups * LPR groups of
// eight: a sub-warp of LPR lanes takes a contiguous run of units, so that the segment search and the instance's key are paid once per
// run and again only where a new instance begins.
#include "boss_common.cuh"

namespace aa {

namespace {

constexpr int kThreads = 256;
constexpr int kGroups = 2;    // groups of eight per lane and unit

template <typename T, int LPR, bool VEC>
__global__ void __launch_bounds__(kThreads) dropout_kernel(DropParams p, int64_t chunks, int64_t units_per_sub) {
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t n_inst = counted(p.count_dev, p.n_inst);
    if (p.offsets && blockIdx.x == 0) check_offsets(p.ctl, p.offsets, n_inst, p.rows);
    if (n_inst == 0) return;
    const int sl = threadIdx.x % LPR;
    const unsigned sub_mask = LPR == 32 ? 0xFFFFFFFFu : ((1u << LPR) - 1u) << ((threadIdx.x & 31) / LPR * LPR);
    const int64_t sub = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / LPR;
    int64_t u = sub * units_per_sub;
    const int64_t rows = p.offsets ? p.rows : n_inst;      // rows past the counted instances: skipped below where there are offsets
    const int64_t u_end = min(u + units_per_sub, rows * chunks);
    if (u >= u_end) return;
    int64_t row = u / chunks;
    int chunk = (int)(u - row * chunks);
    const int groups = (int)((p.cols + 7) >> 3);
    // the instance that holds `row`: rows [first, last)
    int64_t inst = -1, first = 0, last = 0;
    uint2 key = make_uint2(0, 0);
    for (; u < u_end; ++u) {
        if (row >= last) {
            if (p.offsets) {
                inst = inst < 0 ? find_segment(p.offsets, n_inst, row) : inst + 1;
                while (inst < n_inst && __ldg(p.offsets + inst + 1) <= row) ++inst;     // empty segments
                if (inst >= n_inst) return;                                            // rows behind the last counted instance
                first = __ldg(p.offsets + inst);
                last = __ldg(p.offsets + inst + 1);
            } else {
                inst = first = row;
                last = row + 1;
            }
            key = instance_key(p.rule, inst);
        }
        if (row >= first) {
            const T* x = static_cast<const T*>(p.x.data) + row * p.x.stride;
            const T* res = p.res.data ? static_cast<const T*>(p.res.data) + row * p.res.stride : nullptr;
            T* out = const_cast<T*>(static_cast<const T*>(p.out.data)) + row * p.out.stride;
            const uint64_t block0 = (uint64_t)(row - first) * (uint64_t)groups;
            const int g0 = chunk * (LPR * kGroups);
            if constexpr (VEC) {
                float v[kGroups][8], r[kGroups][8];
#pragma unroll
                for (int k = 0; k < kGroups; ++k) {
                    const int c = (g0 + k * LPR + sl) * 8;
                    if (c + 8 <= p.cols) {
                        load8(x + c, v[k]);
                        if (res) load8(res + c, r[k]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            v[k][e] = c + e < p.cols ? load1(x + c + e) : 0.0f;
                            if (res) r[k][e] = c + e < p.cols ? load1(res + c + e) : 0.0f;
                        }
                    }
                }
#pragma unroll
                for (int k = 0; k < kGroups; ++k) {
                    const int g = g0 + k * LPR + sl, c = g * 8;
                    if (p.rule.thr) {
                        const Words4 w = draw_block(p.rule, key, block0 + (uint64_t)g);
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[k][e] = draw_half(w, e) < p.rule.thr ? 0.0f : v[k][e] * p.rule.scale;
                    }
                    if (res) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[k][e] += r[k][e];
                    }
                    if (c + 8 <= p.cols) {
                        store8(out + c, v[k]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (c + e < p.cols) store1(out + c + e, v[k][e]);
                    }
                }
            } else {
                // rows that start at any element: a lane draws for its own group of eight, then the sub-warp walks the elements
                // in memory order (coalesced) and takes each element's bit from the lane that drew it
#pragma unroll
                for (int k = 0; k < kGroups; ++k) {
                    const int gb = g0 + k * LPR;
                    if (gb >= groups) break;
                    float v[8], r[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int c = gb * 8 + e * LPR + sl;
                        v[e] = c < p.cols ? load1(x + c) : 0.0f;
                        r[e] = res && c < p.cols ? load1(res + c) : 0.0f;
                    }
                    uint32_t dropped = 0;
                    if (p.rule.thr) {
                        const Words4 w = draw_block(p.rule, key, block0 + (uint64_t)(gb + sl));
#pragma unroll
                        for (int e = 0; e < 8; ++e) dropped |= (draw_half(w, e) < p.rule.thr ? 1u : 0u) << e;
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int at = e * LPR + sl;                       // element within the LPR * 8 of this pass
                        const uint32_t d = __shfl_sync(sub_mask, dropped, at >> 3, LPR);
                        float y = (d >> (at & 7)) & 1u ? 0.0f : (p.rule.thr ? v[e] * p.rule.scale : v[e]);
                        if (res) y += r[e];
                        const int c = gb * 8 + at;
                        if (c < p.cols) store1(out + c, y);
                    }
                }
            }
        }
        if (++chunk == chunks) {
            chunk = 0;
            ++row;
        }
    }
}

template <typename T, int LPR>
aa_status launch(aa_ctx_impl* c, const DropParams& p, bool vec) {
    const void* kernel = vec ? (const void*)dropout_kernel<T, LPR, true> : (const void*)dropout_kernel<T, LPR, false>;
    const int64_t groups = (p.cols + 7) / 8;
    int64_t chunks = (groups + LPR * kGroups - 1) / (LPR * kGroups);
    const int64_t units = p.rows * chunks;
    const int cap = resident_ctas(c, kernel, kThreads, 0);
    if (cap <= 0) return AA_ERR_CUDA;
    const int64_t subs_per_cta = kThreads / LPR;
    const int64_t subs = (int64_t)cap * subs_per_cta;
    int64_t per_sub = (units + subs - 1) / subs;
    const int64_t used = (units + per_sub - 1) / per_sub;
    const int64_t grid = (used + subs_per_cta - 1) / subs_per_cta;
    DropParams q = p;
    void* args[] = {&q, &chunks, &per_sub};
    if (launch_overlapped(c, kernel, dim3((unsigned)grid), dim3(kThreads), args, 0, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

template <typename T>
aa_status launch_t(aa_ctx_impl* c, const DropParams& p) {
    const auto aligned = [](const RowsArg& a) { return !a.data || ((uintptr_t)a.data % 16 == 0 && (a.stride * (int64_t)sizeof(T)) % 16 == 0); };
    const bool vec = aligned(p.x) && aligned(p.res) && aligned(p.out);
    // lanes per row: enough for the row's groups of eight, at most a warp
    const int64_t groups = (p.cols + 7) / 8;
    if (groups > 16) return launch<T, 32>(c, p, vec);
    if (groups > 4) return launch<T, 8>(c, p, vec);
    return launch<T, 2>(c, p, vec);
}

}  // namespace

bool make_drop_rule(const aa_dropout_rule* r, DropRule& out) {
    out = DropRule{};
    out.scale = 1.0f;
    if (!r) return true;
    if (!(r->p >= 0.0f && r->p < 1.0f)) return false;
    double t = (double)r->p * 65536.0 + 0.5;
    out.thr = t >= 65535.0 ? 65535u : (uint32_t)t;
    out.scale = (float)(65536.0 / (65536.0 - (double)out.thr));
    out.seed_lo = (uint32_t)r->seed;
    out.seed_hi = (uint32_t)(r->seed >> 32);
    out.step_lo = (uint32_t)r->step;
    out.step_hi = (uint32_t)(r->step >> 32);
    out.site = r->site;
    out.row_idx = r->row_idx;
    out.id_base = r->id_base;
    return true;
}

aa_status launch_dropout(aa_ctx_impl* c, const DropParams& p, int dtype) {
    return dtype == AA_BF16 ? launch_t<uint16_t>(c, p) : launch_t<float>(c, p);
}

}  // namespace aa
