// Dropout whose mask is a function of (seed, step, instance id, site, element): out = residual + mask * scale * x.
//
// One Philox block decides eight elements (16 bits each): about 8 of the 29 instructions an element costs, so the kernel stays near memory's
// time only if the next unit's loads are under way while this one's draws are made.  Work is handed out in units of one row's chunk of kGroups *
// LPR groups of eight: a sub-warp of LPR lanes takes a contiguous run of units, so that the segment search and the instance's key are paid
// once per run and again only where a new instance begins.  Bound by instructions (44 and 56 % of the issue slots) together with loads that 24
// warps an SM do not hide: 25,000 x 512 bf16 with residual 21 us (78 MB, 3.7 TB/s), 30,011 x 1,001 fp32, whose rows are not aligned, 52 us (240 MB,
// 4.6 TB/s), one sentence 7 us (launch).
#include "boss_common.cuh"

namespace aa {

namespace {

constexpr int kThreads = 256;
// Groups of eight per lane and unit.  Two where their operands fit the registers of three CTAs on an SM without spilling (fp32 vectors with
// their successors do not); one and more CTAs instead is slower where both fit (25,000 x 512 bf16, at the time: 21.4 against 20.8 us).
template <typename T, bool VEC>
constexpr int kGroupsOf = VEC == (sizeof(T) == 2) ? 2 : 1;

// Eight elements as they are stored.
template <typename T>
struct Raw8 {
    uint4 q[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) q[i] = reinterpret_cast<const uint4*>(p)[i];
    }
    __device__ __forceinline__ void unpack(float (&x)[8]) const {
        if constexpr (sizeof(T) == 2) {
            Vec<uint16_t>::unpack(q[0], x);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                x[4 * i] = __uint_as_float(q[i].x);
                x[4 * i + 1] = __uint_as_float(q[i].y);
                x[4 * i + 2] = __uint_as_float(q[i].z);
                x[4 * i + 3] = __uint_as_float(q[i].w);
            }
        }
    }
};

// x -> scaled or 0: the high half of a word compares in place, the low half shifted up.
__device__ __forceinline__ void drop8(const Words4& w, uint32_t top, float scale, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = (w.w[i] << 16) < top ? 0.0f : x[2 * i] * scale;
        x[2 * i + 1] = w.w[i] < top ? 0.0f : x[2 * i + 1] * scale;
    }
}

// A run of units: where it stands, and the instance that holds the row in hand.
struct Run {
    int64_t u, u_end, row;
    int chunk, chunks;
    int64_t inst, first, last;             // rows [first, last)
    int32_t next_last, next_row;           // what the next instance will need of the lists, on its way
    uint2 key;
    __device__ __forceinline__ void next() {
        ++u;
        if (++chunk == chunks) {
            chunk = 0;
            ++row;
        }
    }
    // The instance of `row`; false: behind the last counted one.
    template <int LPR>
    __device__ __forceinline__ bool locate(const DropParams& p, int64_t n_inst, int sl, unsigned mask) {
        if (row < last) return true;
        int64_t stored;
        if (inst >= 0) {
            ++inst;
            first = last;
            last = p.offsets ? next_last : row + 1;
            stored = p.rule.row_idx ? (int64_t)next_row : inst;
        } else {
            inst = p.offsets ? find_segment_lanes<LPR>(p.offsets, n_inst, row, sl, mask) : row;
            first = p.offsets ? (int64_t)p.offsets[inst] : row;
            last = p.offsets ? (int64_t)p.offsets[inst + 1] : row + 1;
            stored = instance_row(p.rule, inst);
        }
        if (inst >= n_inst) return false;
        while (last <= row) {              // empty segments
            if (++inst >= n_inst) return false;
            first = last;
            last = p.offsets[inst + 1];
            stored = instance_row(p.rule, inst);
        }
        key = id_key(p.rule, p.rule.id_base + stored);
        if (inst + 1 < n_inst) {
            if (p.offsets) next_last = p.offsets[inst + 2];
            if (p.rule.row_idx) next_row = p.rule.row_idx[inst + 1];
        }
        return true;
    }
};

template <typename T, int LPR, bool VEC>
__global__ void __launch_bounds__(kThreads, 3) dropout_kernel(DropParams p, int chunks, int64_t units_per_sub) {
    constexpr int kGroups = kGroupsOf<T, VEC>;
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t n_inst = counted(p.count_dev, p.n_inst);
    if (p.offsets && blockIdx.x == 0) check_offsets(p.ctl, p.offsets, n_inst, p.rows);
    if (n_inst == 0) return;
    const int sl = threadIdx.x % LPR;
    const unsigned mask = LPR == 32 ? 0xFFFFFFFFu : ((1u << LPR) - 1u) << ((threadIdx.x & 31) / LPR * LPR);
    Run run;
    run.u = ((int64_t)blockIdx.x * kThreads + threadIdx.x) / LPR * units_per_sub;
    const int64_t rows = p.offsets ? p.rows : n_inst;      // with offsets, rows behind the counted instances end the run
    run.u_end = min(run.u + units_per_sub, rows * chunks);
    if (run.u >= run.u_end) return;
    run.row = run.u / chunks;
    run.chunk = (int)(run.u - run.row * chunks);
    run.chunks = chunks;
    run.inst = -1;
    run.first = run.last = 0;
    run.next_last = run.next_row = 0;
    run.key = make_uint2(0, 0);
    const int cols = (int)p.cols, groups = (cols + 7) >> 3;
    const uint32_t top = p.rule.thr << 16;
    const auto x_row = [&](int64_t r) { return static_cast<const T*>(p.x.data) + r * p.x.stride; };
    const auto res_row = [&](int64_t r) { return static_cast<const T*>(p.res.data) + r * p.res.stride; };
    const auto out_row = [&](int64_t r) { return const_cast<T*>(static_cast<const T*>(p.out.data)) + r * p.out.stride; };
    if constexpr (VEC) {
        Raw8<T> x[kGroups], res[kGroups];
        const auto fetch = [&](const Run& at) {
#pragma unroll
            for (int k = 0; k < kGroups; ++k) {
                const int c = (at.chunk * (LPR * kGroups) + k * LPR + sl) * 8;
                if (c + 8 <= cols) {
                    x[k].load(x_row(at.row) + c);
                    if (p.res.data) res[k].load(res_row(at.row) + c);
                }
            }
        };
        fetch(run);
        while (true) {
            if (!run.locate<LPR>(p, n_inst, sl, mask)) return;
            const Run here = run;
            Raw8<T> x0[kGroups], res0[kGroups];
#pragma unroll
            for (int k = 0; k < kGroups; ++k) {
                x0[k] = x[k];
                res0[k] = res[k];
            }
            run.next();
            if (run.u < run.u_end) fetch(run);
            if (here.row >= here.first) {
                T* out = out_row(here.row);
                const uint64_t block0 = (uint64_t)(here.row - here.first) * (uint64_t)groups;
#pragma unroll
                for (int k = 0; k < kGroups; ++k) {
                    const int g = here.chunk * (LPR * kGroups) + k * LPR + sl, c = g * 8;
                    if (c >= cols) continue;
                    float v[8], r[8];
                    if (c + 8 <= cols) {
                        x0[k].unpack(v);
                        if (p.res.data) res0[k].unpack(r);
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            v[e] = c + e < cols ? load1(x_row(here.row) + c + e) : 0.0f;
                            if (p.res.data) r[e] = c + e < cols ? load1(res_row(here.row) + c + e) : 0.0f;
                        }
                    }
                    if (p.rule.thr) drop8(draw_block(p.rule, here.key, block0 + (uint64_t)g), top, p.rule.scale, v);
                    if (p.res.data) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] += r[e];
                    }
                    if (c + 8 <= cols) {
                        store8(out + c, v);
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (c + e < cols) store1(out + c + e, v[e]);
                    }
                }
            }
            if (run.u >= run.u_end) return;
        }
    } else {
        // rows that start at any element: a lane draws for its own group of eight, then the sub-warp walks the elements in memory order
        // (coalesced) and takes each element's bit from the lane that drew it
        for (; run.u < run.u_end; run.next()) {
            if (!run.locate<LPR>(p, n_inst, sl, mask)) return;
            if (run.row < run.first) continue;
            const T* x = x_row(run.row);
            const T* res = p.res.data ? res_row(run.row) : nullptr;
            T* out = out_row(run.row);
            const uint64_t block0 = (uint64_t)(run.row - run.first) * (uint64_t)groups;
            const int c0 = run.chunk * (LPR * kGroups) * 8 + sl;
            float v[kGroups][8], r[kGroups][8];
#pragma unroll
            for (int k = 0; k < kGroups; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int c = c0 + (k * 8 + e) * LPR;
                    v[k][e] = c < cols ? load1(x + c) : 0.0f;
                    if (res) r[k][e] = c < cols ? load1(res + c) : 0.0f;
                }
#pragma unroll
            for (int k = 0; k < kGroups; ++k) {
                uint32_t dropped = 0;
                if (p.rule.thr) {
                    const Words4 w = draw_block(p.rule, run.key, block0 + (uint64_t)(run.chunk * (LPR * kGroups) + k * LPR + sl));
#pragma unroll
                    for (int i = 0; i < 4; ++i) dropped |= ((w.w[i] << 16) < top ? 1u << (2 * i) : 0u) | (w.w[i] < top ? 2u << (2 * i) : 0u);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int at = e * LPR + sl;                       // element within the LPR * 8 of this pass
                    const uint32_t d = __shfl_sync(mask, dropped, at >> 3, LPR);
                    float y = (d >> (at & 7)) & 1u ? 0.0f : v[k][e] * p.rule.scale;
                    if (res) y += r[k][e];
                    const int c = c0 + (k * 8 + e) * LPR;
                    if (c < cols) store1(out + c, y);
                }
            }
        }
    }
}

template <typename T, int LPR>
aa_status launch(aa_ctx_impl* c, const DropParams& p, bool vec) {
    const int kGroups = vec ? kGroupsOf<T, true> : kGroupsOf<T, false>;
    static_assert(LPR * 2 * 8 + 8 <= 1024, "kMaxDropoutCols leaves room for a unit behind the last column");
    const void* kernel = vec ? (const void*)dropout_kernel<T, LPR, true> : (const void*)dropout_kernel<T, LPR, false>;
    const int64_t groups = (p.cols + 7) / 8;
    int chunks = (int)((groups + LPR * kGroups - 1) / (LPR * kGroups));
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
