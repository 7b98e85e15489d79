// Gradient of the weighted instance losses with respect to the logits:  G_rc = g_r (softmax(x_r)_c - [c = y_r]).
//
// One read and one write of the logits: a row stays on chip between its sum and its gradient.  Rows of up to 4 KB sit in the registers of up to
// a warp, rows of up to 16 KB in those of a small CTA, rows of up to 64 KB in a stage of a shared-memory ring (bulk copies in and out, in place).
// Longer rows, and gradients that are not aligned like the logits, are swept twice, the second time out of L2.  Measured: 39,000 x 100 fp32 8 us
// (31 MB), of which 6 are the launch; about 25,000 rows x 32,000 bf16 (ring) 3.26 GB in 0.63 ms, 5.2 TB/s: the maximum and the sum of a row are
// two barriers that the copies have to bridge; 4,096 rows x 131,071 bf16 (two sweeps) 2.15 GB in 0.51 ms, 4.2 TB/s, the second sweep out of L2.
#include "async_copy.cuh"
#include "boss_common.cuh"
#include "loss_common.cuh"

namespace aa {

namespace {

struct GradParams {
    LossParams loss;         // logits, rows, cols, labels; out = row losses (nullable); count_dev unused
    const int32_t* offsets;
    int64_t n_inst;
    const int32_t* count_dev;
    const float* weight;
    float scale;
    int mean;
    void* grad;
    int64_t grad_stride;
};

// The factor g_r of row r, or false where no counted instance holds the row.
__device__ __forceinline__ bool row_factor(const GradParams& p, int64_t n_inst, int64_t r, float& g) {
    int64_t inst = r;
    if (p.offsets) {
        if (n_inst == 0) return false;
        inst = find_segment(p.offsets, n_inst, r);
        // empty segments share their start with the next one; the search ends at the last of them
        if (r < p.offsets[inst] || r >= p.offsets[inst + 1]) return false;
    } else if (r >= n_inst) {
        return false;
    }
    g = p.scale;
    if (p.mean) g = g / (float)n_inst;
    if (p.weight) g *= p.weight[inst];
    return true;
}

// First sweep: elements rank, rank + nthreads, ... in 16-byte vectors between the row's 16-byte boundaries.
template <typename T>
__device__ __forceinline__ void scan_row_nat(NatState& st, const T* row, int64_t cols, int rank, int nthreads) {
    constexpr int VE = Vec<T>::kElems;
    int64_t head = ((16 - ((uintptr_t)row & 15)) & 15) / sizeof(T);
    if (head > cols) head = cols;
    const int64_t nvec = (cols - head) / VE;
    int64_t v = rank;
    for (; v + 3 * (int64_t)nthreads < nvec; v += 4 * (int64_t)nthreads) {
        float x[4 * VE];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float y[VE];
            Vec<T>::unpack(*reinterpret_cast<const uint4*>(row + head + (v + k * (int64_t)nthreads) * VE), y);
#pragma unroll
            for (int e = 0; e < VE; ++e) x[k * VE + e] = y[e];
        }
        absorb_nat(st, x);
    }
    for (; v < nvec; v += nthreads) {
        float x[VE];
        Vec<T>::unpack(*reinterpret_cast<const uint4*>(row + head + v * VE), x);
        absorb_nat(st, x);
    }
    for (int64_t c = rank; c < head; c += nthreads) {
        const float x[1] = {load1(row + c)};
        absorb_nat(st, x);
    }
    for (int64_t c = head + nvec * VE + rank; c < cols; c += nthreads) {
        const float x[1] = {load1(row + c)};
        absorb_nat(st, x);
    }
}

// Second sweep, a = g / sum: elements rank, rank + nthreads, ... in 16-byte vectors where both rows are aligned alike.
template <typename T>
__device__ __forceinline__ void write_row(const T* row, T* out, int64_t cols, float m, float a, float g, int y, int rank, int nthreads) {
    constexpr int VE = Vec<T>::kElems;
    const auto at = [&](float x, int64_t c) { return fmaf(a, exp_from(x, m), c == y ? -g : 0.0f); };
    int64_t head = cols, nvec = 0;
    if ((((uintptr_t)row ^ (uintptr_t)out) & 15) == 0) {
        head = ((16 - ((uintptr_t)row & 15)) & 15) / sizeof(T);
        if (head > cols) head = cols;
        nvec = (cols - head) / VE;
    }
    const auto put = [&](const uint4& q, int64_t v) {
        const int64_t c = head + v * VE;
        float x[VE];
        Vec<T>::unpack(q, x);
#pragma unroll
        for (int e = 0; e < VE; ++e) x[e] = a * exp_from(x[e], m);
        if ((uint64_t)(y - c) < (uint64_t)VE) {
#pragma unroll
            for (int e = 0; e < VE; ++e) x[e] -= c + e == y ? g : 0.0f;
        }
        if constexpr (VE == 8) store8(out + c, x);
        else *reinterpret_cast<float4*>(out + c) = make_float4(x[0], x[1], x[2], x[3]);
    };
    int64_t v = rank;
    for (; v + 3 * (int64_t)nthreads < nvec; v += 4 * (int64_t)nthreads) {
        uint4 q[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) q[k] = *reinterpret_cast<const uint4*>(row + head + (v + k * (int64_t)nthreads) * VE);
#pragma unroll
        for (int k = 0; k < 4; ++k) put(q[k], v + k * (int64_t)nthreads);
    }
    for (; v < nvec; v += nthreads) put(*reinterpret_cast<const uint4*>(row + head + v * VE), v);
    for (int64_t c = rank; c < head; c += nthreads) store1(out + c, at(load1(row + c), c));
    for (int64_t c = head + nvec * VE + rank; c < cols; c += nthreads) store1(out + c, at(load1(row + c), c));
}

template <typename T>
__device__ __forceinline__ void zero_row(T* out, int64_t cols, int rank, int nthreads) {
    for (int64_t c = rank; c < cols; c += nthreads) store1(out + c, 0.0f);
}

// ------------------------------------------------------------------------------------------- rows in registers

// Below this size of m, 2^(x log2 e - fl(m log2 e)) may stand for it: the rounding of m log2 e is at most 2^-4 (half an ulp below 2^21) and a
// factor close to one takes it out of sums and gradients.  It doubles with every doubling of m and passes the exponent's range at a few 1e9.
constexpr float kFusedLimit = 1048576.0f;

// Where a row's 16-byte vectors lie: `head` elements before them, nvec vectors, the rest behind.
template <typename T>
struct RowSpan {
    int head, nvec, tail0;
    __device__ __forceinline__ RowSpan(const T* row, int cols) {
        constexpr int VE = Vec<T>::kElems;
        head = min((int)(((16 - ((uintptr_t)row & 15)) & 15) / sizeof(T)), cols);
        nvec = (cols - head) / VE;
        tail0 = head + nvec * VE;
    }
};

// A thread's share of a row: V vectors (rank, rank + n, ...) and at most one element of the head and of the tail.
template <typename T, int V>
struct RowPart {
    static constexpr int VE = Vec<T>::kElems;
    float e[V][VE], eh, et;    // logits, then exponentials against the thread's own maximum
    float m, s, undo;          // s and what they stand for include the factor `undo`
    __device__ __forceinline__ void load_ends(const T* row, const RowSpan<T>& sp, int cols, int rank) {
        eh = rank < sp.head ? load1(row + rank) : -INFINITY;
        et = sp.tail0 + rank < cols ? load1(row + sp.tail0 + rank) : -INFINITY;
    }
    // vectors rank + k n < nv of `body` (memory or shared); what is missing reads as -inf
    __device__ __forceinline__ void load_body(const T* body, int nv, int rank, int n) {
        constexpr uint32_t kNegInf = VE == 8 ? 0xFF80FF80u : 0xFF800000u;
        uint4 w[V];
#pragma unroll
        for (int k = 0; k < V; ++k) {
            w[k] = make_uint4(kNegInf, kNegInf, kNegInf, kNegInf);
            if (rank + k * n < nv) w[k] = *reinterpret_cast<const uint4*>(body + (int64_t)(rank + k * n) * VE);
        }
#pragma unroll
        for (int k = 0; k < V; ++k) Vec<T>::unpack(w[k], e[k]);
    }
    __device__ __forceinline__ void exponentials() {
        m = fmaxf(eh, et);
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int i = 0; i < VE; ++i) m = fmaxf(m, e[k][i]);
        const float ref = m == -INFINITY ? 0.0f : m;
        float s0, s1;
        if (fabsf(ref) < kFusedLimit) {
            // 2^(x log2 e - fl(m log2 e)): one multiply-add; the rounding of the product is common to all and taken out of the sum and the factor
            const float shift = -ref * kLog2e;
            undo = ex2_approx(-fmaf(ref, kLog2e, shift));
            eh = ex2_approx(fmaf(eh, kLog2e, shift));
            et = ex2_approx(fmaf(et, kLog2e, shift));
            s0 = eh;
            s1 = et;
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < VE; ++i) {
                    e[k][i] = ex2_approx(fmaf(e[k][i], kLog2e, shift));
                    (i & 1 ? s1 : s0) += e[k][i];
                }
        } else {
            undo = 1.0f;
            eh = exp_from(eh, ref);
            et = exp_from(et, ref);
            s0 = eh;
            s1 = et;
#pragma unroll
            for (int k = 0; k < V; ++k)
#pragma unroll
                for (int i = 0; i < VE; ++i) {
                    e[k][i] = exp_from(e[k][i], ref);
                    (i & 1 ? s1 : s0) += e[k][i];
                }
        }
        s = (s0 + s1) * undo;
    }
    // What turns this thread's exponentials into g p.  A thread that saw only -inf holds zeros; a row of nothing else is NaN, as its loss is.
    __device__ __forceinline__ float factor(const NatState& all, float g) const {
        return (m == -INFINITY && all.m != -INFINITY ? 0.0f : exp_from(m, all.m)) * undo * (g / all.s);
    }
    __device__ __forceinline__ void store_ends(T* out, const RowSpan<T>& sp, int cols, int rank, float f, float g, int y) {
        if (rank < sp.head) store1(out + rank, fmaf(eh, f, rank == y ? -g : 0.0f));
        if (sp.tail0 + rank < cols) store1(out + sp.tail0 + rank, fmaf(et, f, sp.tail0 + rank == y ? -g : 0.0f));
    }
    // at_y: element of `body` that is the label's (negative: none here), fy: its gradient.  The thread that owns it writes it again: an index into
    // the exponentials would put them into local memory.
    __device__ __forceinline__ void store_body(T* body, int nv, int rank, int n, float f, int at_y, float fy) {
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const int v = rank + k * n;
            if (v >= nv) continue;
            float x[VE];
#pragma unroll
            for (int i = 0; i < VE; ++i) x[i] = e[k][i] * f;
            if constexpr (VE == 8) store8(body + (int64_t)v * VE, x);
            else *reinterpret_cast<float4*>(body + (int64_t)v * VE) = make_float4(x[0], x[1], x[2], x[3]);
        }
        if (at_y >= 0 && (at_y / VE) % n == rank) store1(body + at_y, fy);
    }
};

// Gradient of the label's logit.
__device__ __forceinline__ float label_grad(const NatState& all, float label_logit, float g) { return fmaf(exp_from(label_logit, all.m), g / all.s, -g); }

// LPR lanes per row (LPR * V vectors at least; at least 16 / sizeof(T) - 1 lanes for the ends).
template <typename T, int LPR, int V>
__global__ void __launch_bounds__(256) row_grad_lanes_kernel(GradParams p) {
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t n_inst = counted(p.count_dev, p.n_inst);
    if (p.offsets && blockIdx.x == 0) check_offsets(p.loss.ctl, p.offsets, n_inst, p.loss.rows);
    const int gl = threadIdx.x % LPR, cols = (int)p.loss.cols;
    const int64_t groups_per_grid = (int64_t)gridDim.x * (256 / LPR), group0 = (int64_t)blockIdx.x * (256 / LPR) + threadIdx.x / LPR;
    const int64_t rounds = (p.loss.rows + groups_per_grid - 1) / groups_per_grid;   // whole warps iterate together (shuffles)
    for (int64_t it = 0; it < rounds; ++it) {
        const int64_t r = group0 + it * groups_per_grid;
        float g = 0.0f;
        const bool live = r < p.loss.rows && row_factor(p, n_inst, r, g);
        const T* row = static_cast<const T*>(p.loss.logits) + (live ? r : 0) * p.loss.row_stride;
        const RowSpan<T> sp(row, cols);
        RowPart<T, V> part;
        part.load_ends(row, sp, live ? cols : 0, live ? gl : cols);
        part.load_body(row + sp.head, live ? sp.nvec : 0, gl, LPR);
        const int y = live ? checked_label(p.loss, r) : -1;
        const float label_logit = y >= 0 ? load1(row + y) : 0.0f;
        part.exponentials();
        const NatState all = group_merge_nat<LPR>(NatState{part.m, part.s});       // and: every lane has read the row
        __syncwarp();
        if (live) {
            T* out = static_cast<T*>(p.grad) + r * p.grad_stride;
            if (y >= 0) {
                const float f = part.factor(all, g);
                part.store_ends(out, sp, cols, gl, f, g, y);
                part.store_body(out + sp.head, sp.nvec, gl, LPR, f, y >= sp.head && y < sp.tail0 ? y - sp.head : -1, label_grad(all, label_logit, g));
            } else {
                zero_row<T>(out, cols, gl, LPR);
            }
            if (p.loss.out && gl == 0) p.loss.out[r] = y >= 0 ? row_loss(all, label_logit) : 0.0f;
        }
    }
}

// A CTA of 128 threads per row: up to 128 * V vectors.
template <typename T, int V>
__global__ void __launch_bounds__(128) row_grad_block_kernel(GradParams p) {
    __shared__ NatState warp_state[2][4];
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t n_inst = counted(p.count_dev, p.n_inst);
    if (p.offsets && blockIdx.x == 0) check_offsets(p.loss.ctl, p.offsets, n_inst, p.loss.rows);
    const int cols = (int)p.loss.cols;
    int turn = 0;
    for (int64_t r = blockIdx.x; r < p.loss.rows; r += gridDim.x, turn ^= 1) {
        const T* row = static_cast<const T*>(p.loss.logits) + r * p.loss.row_stride;
        const RowSpan<T> sp(row, cols);
        RowPart<T, V> part;
        part.load_ends(row, sp, cols, threadIdx.x);
        part.load_body(row + sp.head, sp.nvec, threadIdx.x, 128);
        float g = 0.0f;
        const bool live = row_factor(p, n_inst, r, g);                // uniform over the CTA
        const int y = live ? checked_label(p.loss, r) : -1;
        const float label_logit = y >= 0 ? load1(row + y) : 0.0f;
        part.exponentials();
        const NatState mine = group_merge_nat<32>(NatState{part.m, part.s});
        if ((threadIdx.x & 31) == 0) warp_state[turn][threadIdx.x >> 5] = mine;
        __syncthreads();                                              // and: every thread has read the row
        if (!live) continue;
        T* out = static_cast<T*>(p.grad) + r * p.grad_stride;
        if (y >= 0) {
            const NatState all = merge(merge(warp_state[turn][0], warp_state[turn][1]), merge(warp_state[turn][2], warp_state[turn][3]));
            const float f = part.factor(all, g);
            part.store_ends(out, sp, cols, threadIdx.x, f, g, y);
            part.store_body(out + sp.head, sp.nvec, threadIdx.x, 128, f, y >= sp.head && y < sp.tail0 ? y - sp.head : -1, label_grad(all, label_logit, g));
            if (p.loss.out && threadIdx.x == 0) p.loss.out[r] = row_loss(all, label_logit);
        } else {
            zero_row<T>(out, cols, threadIdx.x, 128);
            if (p.loss.out && threadIdx.x == 0) p.loss.out[r] = 0.0f;
        }
    }
}

// --------------------------------------------------------------------------------------------- ring of long rows

constexpr int kRingThreads = 512;          // consumers; a producer warp and a storing warp come on top
constexpr int kRingVecs = 8;                // vectors per consumer: rows of up to 64 KB
constexpr int kRingMaxStages = 6;

// What the producer hands over with a row.
struct RingRow {
    int64_t row;               // -1: no more rows
    float g, label_logit;
    int y;
    float ends[16];            // head elements, then tail elements
};
struct RingControl {
    uint64_t full[kRingMaxStages], done[kRingMaxStages], empty[kRingMaxStages];
    RingRow rows[kRingMaxStages];
    NatState warp_state[2][kRingThreads / 32];
    int abort_flag;
};

// All consumers: true iff `ok` in every one of them.
__device__ __forceinline__ bool consumers_all(bool ok) {
    int r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %1, 0;\n\tbarrier.red.and.pred q, 1, %2, p;\n\tselp.s32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"((int)ok), "n"(kRingThreads) : "memory");
    return r != 0;
}
__device__ __forceinline__ void bulk_s2g(void* dst, const void* src_smem, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(smem_u32(src_smem)), "r"(bytes) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }

// 2^((x - m) log2 e) / undo: one multiply-add and the exponential; `undo` takes the rounding of m log2 e out of sums and factors.  Where that
// rounding is no longer small the difference is taken first.
struct ExpAt {
    float ref, shift, undo;
    bool plain;
    __device__ __forceinline__ explicit ExpAt(float m) {
        ref = m == -INFINITY ? 0.0f : m;
        plain = !(fabsf(ref) < kFusedLimit);
        shift = plain ? 0.0f : -ref * kLog2e;
        undo = plain ? 1.0f : ex2_approx(-fmaf(ref, kLog2e, shift));
    }
    __device__ __forceinline__ float fast(float x) const { return ex2_approx(fmaf(x, kLog2e, shift)); }
    __device__ __forceinline__ float operator()(float x) const { return plain ? exp_from(x, ref) : fast(x); }
};

__device__ __forceinline__ float vec_max(const uint4& w, const float*) {
    return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
}
__device__ __forceinline__ float vec_max(const uint4& w, const uint16_t*) {
    float x[8];
    Vec<uint16_t>::unpack(w, x);
    return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
}
template <typename T>
__device__ __forceinline__ float slice_max(const T* body, int nv, int tid) {
    const uint4* w = reinterpret_cast<const uint4*>(body);
    float m = -INFINITY;
#pragma unroll 4
    for (int v = tid; v < nv; v += kRingThreads) {
        const uint4 q = w[v];              // one 16-byte load
        m = fmaxf(m, vec_max(q, body));
    }
    return m;
}
// The thread's exponentials of the row in `body`, and their sum.
template <typename T>
__device__ __forceinline__ float row_exponentials(const T* body, int nv, int tid, const ExpAt& at, float (&e)[kRingVecs][Vec<T>::kElems]) {
    constexpr int VE = Vec<T>::kElems;
    const uint4* w = reinterpret_cast<const uint4*>(body);
    float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
    for (int k = 0; k < kRingVecs; ++k) {
        if (tid + k * kRingThreads < nv) {
            const uint4 q = w[tid + k * kRingThreads];
            Vec<T>::unpack(q, e[k]);
            if (at.plain) {
#pragma unroll
                for (int i = 0; i < VE; ++i) e[k][i] = exp_from(e[k][i], at.ref);
            } else {
#pragma unroll
                for (int i = 0; i < VE; ++i) e[k][i] = at.fast(e[k][i]);
            }
#pragma unroll
            for (int i = 0; i < VE; ++i) (i & 1 ? s1 : s0) += e[k][i];
        }
    }
    return s0 + s1;
}
template <typename T>
__device__ __forceinline__ void row_gradient(T* body, int nv, int tid, float f, const float (&e)[kRingVecs][Vec<T>::kElems]) {
    constexpr int VE = Vec<T>::kElems;
#pragma unroll
    for (int k = 0; k < kRingVecs; ++k) {
        const int v = tid + k * kRingThreads;
        if (v < nv) {
            float x[VE];
#pragma unroll
            for (int i = 0; i < VE; ++i) x[i] = e[k][i] * f;
            if constexpr (VE == 8) store8(body + (int64_t)v * VE, x);
            else *reinterpret_cast<float4*>(body + (int64_t)v * VE) = make_float4(x[0], x[1], x[2], x[3]);
        }
    }
}

// One persistent CTA per SM, rows handed out in turn, one ring stage each: fetched once, read for the maximum and again for the exponentials,
// which stay in registers until the sum is known, overwritten by the gradient and copied out.
template <typename T>
__global__ void __launch_bounds__(kRingThreads + 64, 1) row_grad_ring_kernel(GradParams p, int stages, int stage_vecs) {
    constexpr int VE = Vec<T>::kElems;
    extern __shared__ uint4 smem16[];
    __shared__ RingControl ctl;
    grid_dependency_wait();
    grid_dependency_release();
    const int cols = (int)p.loss.cols;
    const int64_t n_inst = counted(p.count_dev, p.n_inst), step = gridDim.x;
    uint4* ring = smem16;
    volatile int* abort_flag = &ctl.abort_flag;
    if (threadIdx.x == 0) {
        for (int i = 0; i < stages; ++i) {
            mbar_init(&ctl.full[i], 1);
            mbar_init(&ctl.done[i], kRingThreads / 32);
            mbar_init(&ctl.empty[i], 1);
        }
        ctl.abort_flag = 0;
        mbar_fence_init();
    }
    __syncthreads();
    const int lane = threadIdx.x & 31;
    if (threadIdx.x >= kRingThreads + 32) {
        // ---- storing warp: a finished row goes out, and its stage is free as soon as the copies have read it
        for (int64_t j = 0;; ++j) {
            const int stage = (int)(j % stages);
            if (!mbar_wait(&ctl.done[stage], (uint32_t)((j / stages) & 1), abort_flag) || *abort_flag) break;
            const int64_t r = ctl.rows[stage].row;
            if (r < 0) break;
            T* out = static_cast<T*>(p.grad) + r * p.grad_stride;
            const RowSpan<T> sp(static_cast<const T*>(p.loss.logits) + r * p.loss.row_stride, cols);
            const int piece = (sp.nvec + 31) >> 5, v0 = lane * piece, n = min(piece, sp.nvec - v0);
            if (n > 0) bulk_s2g(out + sp.head + (int64_t)v0 * VE, ring + (size_t)stage * stage_vecs + v0, (uint32_t)n * 16u);
            bulk_wait_read();
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.empty[stage]);
        }
    } else if (threadIdx.x >= kRingThreads) {
        // ---- producer warp
        if (p.offsets && blockIdx.x == 0) {
            bool bad = false;
            for (int64_t s = lane; s < n_inst; s += 32) {
                const int a = p.offsets[s], b = p.offsets[s + 1];
                bad |= a < 0 || b < a || b > p.loss.rows;
            }
            if (bad) latch(p.loss.ctl, AA_ERR_BAD_INDEX);
        }
        int64_t j = 0;
        bool ok = true, more = true;
        for (int64_t r0 = blockIdx.x; ok && more; r0 += 32 * step) {
            // a lane per row: 32 rows' searches, labels and label logits cost one chain of loads
            const int64_t mine = r0 + lane * step;
            float my_g = 0.0f, my_logit = 0.0f;
            int my_y = -2;                 // not counted
            if (mine < p.loss.rows && row_factor(p, n_inst, mine, my_g)) {
                my_y = checked_label(p.loss, mine);
                if (my_y >= 0) my_logit = load1(static_cast<const T*>(p.loss.logits) + mine * p.loss.row_stride + my_y);
            }
            for (int i = 0; more && i < 32; ++i) {
                const int64_t r = r0 + i * step;
                more = r < p.loss.rows;
                const int y = __shfl_sync(0xFFFFFFFFu, my_y, i);
                const float g = __shfl_sync(0xFFFFFFFFu, my_g, i), label_logit = __shfl_sync(0xFFFFFFFFu, my_logit, i);
                if (more && y == -2) continue;
                const int stage = (int)(j % stages);
                if (j >= stages && !mbar_wait(&ctl.empty[stage], (uint32_t)((j / stages - 1) & 1), abort_flag)) {
                    ok = false;
                    break;
                }
                const T* row = static_cast<const T*>(p.loss.logits) + (more ? r : 0) * p.loss.row_stride;
                const RowSpan<T> sp(row, cols);
                const bool load = more && y >= 0;                     // padding rows are only written
                const int nv = load ? sp.nvec : 0;
                RingRow* c = &ctl.rows[stage];
                if (lane == 0) {
                    c->row = more ? r : -1;
                    c->g = g;
                    c->y = y;
                    c->label_logit = label_logit;
                    mbar_expect_tx(&ctl.full[stage], (uint32_t)nv * 16u);
                }
                __syncwarp();
                // one copy per lane: many in flight at once (the phase cannot complete before lane 0's arrival below)
                const int piece = (nv + 31) >> 5, v0 = lane * piece, n = min(piece, nv - v0);
                if (n > 0) bulk_g2s(ring + (size_t)stage * stage_vecs + v0, row + sp.head + (int64_t)v0 * VE, (uint32_t)n * 16u, &ctl.full[stage]);
                float end = 0.0f;          // lanes 0..7: head, 8..15: tail
                if (load && lane < sp.head) end = load1(row + lane);
                if (load && lane >= 8 && lane < 16 && sp.tail0 + lane - 8 < cols) end = load1(row + sp.tail0 + lane - 8);
                if (lane < 16) c->ends[lane] = end;
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl.full[stage]);
                ++j;
            }
        }
        if (!ok) {                         // the copies in flight still write to this CTA's memory
            ctl.abort_flag = 1;
            for (int64_t i = j > stages ? j - stages : 0; i < j; ++i) {
                const long long t0 = clock64();
                while (!mbar_try_wait(&ctl.full[i % stages], (uint32_t)((i / stages) & 1)) && clock64() - t0 < kWaitCycles) {
                }
            }
        }
    } else {
        // ---- consumers
        const int tid = threadIdx.x, warp = tid >> 5;
        bool ok = true;
        for (int64_t j = 0;; ++j) {
            const int stage = (int)(j % stages), turn = (int)(j & 1);
            ok = mbar_wait(&ctl.full[stage], (uint32_t)((j / stages) & 1), abort_flag);
            const RingRow* c = &ctl.rows[stage];
            const int64_t r = ok ? c->row : 0;
            const int y = ok && r >= 0 ? c->y : -1;
            const RowSpan<T> sp(static_cast<const T*>(p.loss.logits) + (r < 0 ? 0 : r) * p.loss.row_stride, cols);
            T* body = reinterpret_cast<T*>(ring + (size_t)stage * stage_vecs);
            const int nh = sp.head, nt = cols - sp.tail0;
            float e[kRingVecs][VE];
            float eh = -INFINITY, et = -INFINITY;
            NatState mine = {-INFINITY, 0.0f};
            float undo = 1.0f;
            if (y >= 0) {
                if (tid < nh) eh = c->ends[tid];
                if (tid < nt) et = c->ends[8 + tid];
                mine.m = fmaxf(fmaxf(eh, et), slice_max(body, sp.nvec, tid));
                const ExpAt at(mine.m);
                undo = at.undo;
                eh = at(eh);
                et = at(et);
                mine.s = (eh + et + row_exponentials(body, sp.nvec, tid, at, e)) * undo;
                const NatState w = group_merge_nat<32>(mine);
                if (lane == 0) ctl.warp_state[turn][warp] = w;
            }
            if (!consumers_all(ok)) {      // a wait that gave up: all leave here
                ok = false;
                break;
            }
            if (r < 0) {
                if (lane == 0) mbar_arrive(&ctl.done[stage]);
                break;
            }
            T* out = static_cast<T*>(p.grad) + r * p.grad_stride;
            if (y >= 0) {
                const NatState all = group_merge_nat<16>(ctl.warp_state[turn][lane & 15]);
                const float g = c->g, label_logit = c->label_logit;
                // this thread's exponentials -> g p; one that saw only -inf holds zeros, a row of nothing else is NaN as its loss is
                const float f = (mine.m == -INFINITY && all.m != -INFINITY ? 0.0f : exp_from(mine.m, all.m)) * undo * (g / all.s);
                row_gradient(body, sp.nvec, tid, f, e);
                const int idx = y - sp.head;
                if (idx >= 0 && y < sp.tail0 && (idx / VE) % kRingThreads == tid) store1(body + idx, label_grad(all, label_logit, g));
                if (tid < nh) store1(out + tid, fmaf(eh, f, tid == y ? -g : 0.0f));
                if (tid < nt) store1(out + sp.tail0 + tid, fmaf(et, f, sp.tail0 + tid == y ? -g : 0.0f));
                if (p.loss.out && tid == 0) p.loss.out[r] = row_loss(all, label_logit);
            } else {
                for (int v = tid; v < sp.nvec; v += kRingThreads) reinterpret_cast<uint4*>(body)[v] = make_uint4(0, 0, 0, 0);
                if (tid < nh) store1(out + tid, 0.0f);
                if (tid < nt) store1(out + sp.tail0 + tid, 0.0f);
                if (p.loss.out && tid == 0) p.loss.out[r] = 0.0f;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl.done[stage]);
        }
        if (!ok) {
            ctl.abort_flag = 1;
            if (tid == 0) latch(p.loss.ctl, AA_ERR_SCAN_TIMEOUT);
        }
    }
}

// ------------------------------------------------------------------------------------------- two sweeps

template <typename T>
__global__ void __launch_bounds__(256) row_grad_group_kernel(GradParams p) {
    constexpr int LPR = 32;
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t n_inst = counted(p.count_dev, p.n_inst);
    if (p.offsets && blockIdx.x == 0) check_offsets(p.loss.ctl, p.offsets, n_inst, p.loss.rows);
    const int gl = threadIdx.x % LPR;
    const int64_t groups_per_grid = (int64_t)gridDim.x * (blockDim.x / LPR);
    const int64_t group0 = (int64_t)blockIdx.x * (blockDim.x / LPR) + threadIdx.x / LPR;
    const int64_t rounds = (p.loss.rows + groups_per_grid - 1) / groups_per_grid;   // whole warps iterate together (shuffles)
    for (int64_t it = 0; it < rounds; ++it) {
        const int64_t r = group0 + it * groups_per_grid;
        float g = 0.0f;
        const bool live = r < p.loss.rows && row_factor(p, n_inst, r, g);
        const int y = live ? checked_label(p.loss, r) : -1;
        const T* row = static_cast<const T*>(p.loss.logits) + (live ? r : 0) * p.loss.row_stride;
        NatState st = {-INFINITY, 0.0f};
        float label_logit = 0.0f;
        if (y >= 0) {
            label_logit = load1(row + y);
            scan_row_nat<T>(st, row, p.loss.cols, gl, LPR);
        }
        st = group_merge_nat<LPR>(st);          // also: every lane has read the row before any lane writes over it
        __syncwarp();
        if (live) {
            T* out = static_cast<T*>(p.grad) + r * p.grad_stride;
            if (y >= 0) write_row<T>(row, out, p.loss.cols, st.m, g / st.s, g, y, gl, LPR);
            else zero_row<T>(out, p.loss.cols, gl, LPR);
            if (p.loss.out && gl == 0) p.loss.out[r] = y >= 0 ? row_loss(st, label_logit) : 0.0f;
        }
    }
}

// A CTA of 512 threads per row, two on an SM: the rows in flight (296) fit L2 up to 400 KB each.
constexpr int kSweepThreads = 512;

template <typename T>
__global__ void __launch_bounds__(kSweepThreads, 2) row_grad_cta_kernel(GradParams p) {
    __shared__ NatState warp_state[kSweepThreads / 32];
    grid_dependency_wait();
    grid_dependency_release();
    const int64_t n_inst = counted(p.count_dev, p.n_inst);
    if (p.offsets && blockIdx.x == 0) check_offsets(p.loss.ctl, p.offsets, n_inst, p.loss.rows);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int64_t r = blockIdx.x; r < p.loss.rows; r += gridDim.x) {
        float g = 0.0f;
        if (!row_factor(p, n_inst, r, g)) continue;     // uniform over the CTA
        const int y = checked_label(p.loss, r);
        const T* row = static_cast<const T*>(p.loss.logits) + r * p.loss.row_stride;
        T* out = static_cast<T*>(p.grad) + r * p.grad_stride;
        if (y < 0) {
            zero_row<T>(out, p.loss.cols, threadIdx.x, kSweepThreads);
            if (p.loss.out && threadIdx.x == 0) p.loss.out[r] = 0.0f;
            continue;
        }
        const float label_logit = load1(row + y);
        NatState st = {-INFINITY, 0.0f};
        scan_row_nat<T>(st, row, p.loss.cols, threadIdx.x, kSweepThreads);
        st = group_merge_nat<32>(st);
        __syncthreads();                                 // the previous row's states have been read
        if (lane == 0) warp_state[warp] = st;
        __syncthreads();
        st = group_merge_nat<32>(lane < kSweepThreads / 32 ? warp_state[lane] : NatState{-INFINITY, 0.0f});
        write_row<T>(row, out, p.loss.cols, st.m, g / st.s, g, y, threadIdx.x, kSweepThreads);
        if (p.loss.out && threadIdx.x == 0) p.loss.out[r] = row_loss(st, label_logit);
    }
}

template <typename T>
aa_status launch_ring(aa_ctx_impl* c, GradParams& p) {
    const void* kernel = (const void*)row_grad_ring_kernel<T>;
    const int64_t vecs = p.loss.cols * (int64_t)sizeof(T) / 16;
    int stage_vecs = (int)((vecs + 7) / 8 * 8);
    int stages = 208 * 1024 / (stage_vecs * 16);                      // three of 64 KB
    if (stages > kRingMaxStages) stages = kRingMaxStages;
    const size_t smem = (size_t)stages * stage_vecs * 16;
    if (allow_smem(c, kernel, smem) != AA_OK) return AA_ERR_CUDA;
    const int cap = resident_ctas(c, kernel, kRingThreads + 64, smem);
    if (cap <= 0) return AA_ERR_CUDA;
    void* args[] = {&p, &stages, &stage_vecs};
    const unsigned grid = (unsigned)(p.loss.rows < cap ? p.loss.rows : cap);
    if (launch_overlapped(c, kernel, dim3(grid), dim3(kRingThreads + 64), args, smem, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

template <typename T>
aa_status launch_rows(aa_ctx_impl* c, GradParams& p) {
    const int64_t row_bytes = p.loss.cols * (int64_t)sizeof(T), vecs = (row_bytes + 15) / 16;
    // the gradient's rows start at the logits' offsets from a 16-byte boundary
    const bool alike = (((uintptr_t)p.loss.logits ^ (uintptr_t)p.grad) & 15) == 0 && ((p.loss.row_stride - p.grad_stride) * (int64_t)sizeof(T)) % 16 == 0;
    void* args[] = {&p};
    const void* kernel;
    int64_t want;
    int threads = 256;
    if (alike && vecs <= 256) {
        if (sizeof(T) == 4 && vecs <= 16) {
            kernel = (const void*)row_grad_lanes_kernel<T, sizeof(T) == 4 ? 4 : 8, 4>;
            want = (p.loss.rows + 63) / 64;
        } else if (vecs <= 32) {
            kernel = (const void*)row_grad_lanes_kernel<T, 8, 4>;
            want = (p.loss.rows + 31) / 32;
        } else if (vecs <= 64) {
            kernel = (const void*)row_grad_lanes_kernel<T, 16, 4>;
            want = (p.loss.rows + 15) / 16;
        } else if (vecs <= 128) {
            kernel = (const void*)row_grad_lanes_kernel<T, 32, 4>;
            want = (p.loss.rows + 7) / 8;
        } else {
            kernel = (const void*)row_grad_lanes_kernel<T, 32, 8>;
            want = (p.loss.rows + 7) / 8;
        }
    } else if (alike && vecs <= 1024) {
        kernel = (const void*)row_grad_block_kernel<T, 8>;
        want = p.loss.rows;
        threads = 128;
    } else if (alike && vecs <= kRingThreads * kRingVecs) {
        return launch_ring<T>(c, p);
    } else if (row_bytes > 8 * 1024) {
        kernel = (const void*)row_grad_cta_kernel<T>;
        want = p.loss.rows;
        threads = kSweepThreads;
    } else {
        kernel = (const void*)row_grad_group_kernel<T>;
        want = (p.loss.rows + 7) / 8;
    }
    const int cap = resident_ctas(c, kernel, threads, 0);
    if (cap <= 0) return AA_ERR_CUDA;
    const unsigned grid = (unsigned)(want < cap ? want : cap);
    if (launch_overlapped(c, kernel, dim3(grid), dim3(threads), args, 0, false) != cudaSuccess) return AA_ERR_CUDA;
    ++c->launches;
    return AA_OK;
}

}  // namespace

aa_status launch_instance_loss_grad(aa_ctx_impl* c, const aa_logits& lg, const int32_t* labels, const int32_t* offsets, int64_t n_seg,
                                    const int32_t* count_dev, const float* weight, float scale, int mean, float* out_loss, const aa_rows& grad) {
    GradParams p = {};
    p.loss.logits = lg.data;
    p.loss.rows = p.loss.n_stored = lg.rows;
    p.loss.cols = lg.cols;
    p.loss.row_stride = lg.row_stride;
    p.loss.labels = labels;
    p.loss.ctl = c->ctl;
    p.loss.out = out_loss && offsets ? c->row_scratch : out_loss;
    p.offsets = offsets;
    p.n_inst = offsets ? n_seg : lg.rows;
    p.count_dev = count_dev;
    p.weight = weight;
    p.scale = scale;
    p.mean = mean;
    p.grad = grad.data;
    p.grad_stride = grad.row_stride;
    if (lg.rows > 0) {
        const aa_status st = lg.dtype == AA_BF16 ? launch_rows<uint16_t>(c, p) : launch_rows<float>(c, p);
        if (st != AA_OK) return st;
    }
    if (offsets && out_loss && n_seg > 0) return launch_segment_sum(c, c->row_scratch, offsets, n_seg, count_dev, lg.rows, out_loss);
    return AA_OK;
}

}  // namespace aa
