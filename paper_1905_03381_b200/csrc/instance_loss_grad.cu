// Gradient of the weighted instance losses with respect to the logits:  G_rc = g_r (softmax(x_r)_c - [c = y_r]).
//
// One read and one write of the logits: a row stays on chip between its sum and its gradient.  Rows of up to 4 KB sit in the registers of up to
// a warp, rows of up to 16 KB in those of a small CTA; longer ones stream through a ring of shared-memory stages (bulk copies in and out,
// in place), split over a cluster of CTAs where a slice would pass 64 KB.  Every exponential is evaluated once, against the thread's own
// maximum, and rescaled by one factor per thread.  What is left (rows past 512 KB, gradients that are not aligned like the logits) is swept
// twice through L2.
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
        if (r < __ldg(p.offsets + inst) || r >= __ldg(p.offsets + inst + 1)) return false;
    } else if (r >= n_inst) {
        return false;
    }
    g = p.scale;
    if (p.mean) g = g / (float)n_inst;
    if (p.weight) g *= __ldg(p.weight + inst);
    return true;
}

// Running maximum and sum of a row in the logits' own scale: exponents are 2^((x - m) log2 e), so that logits near the type's limits do not
// overflow in a change of base (one subtraction more per element than the loss kernels' fused form; these kernels have the room).
struct NatState {
    float m, s;
};
__device__ __forceinline__ float exp_from(float x, float m) { return ex2_approx((x - m) * kLog2e); }
template <int N>
__device__ __forceinline__ void absorb_nat(NatState& st, const float (&x)[N]) {
    float top = x[0];
#pragma unroll
    for (int e = 1; e < N; ++e) top = fmaxf(top, x[e]);
    if (top > st.m) {
        st.s *= exp_from(st.m, top);       // st.m = -inf gives 0 * 0
        st.m = top;
    }
    const float ref = st.m == -INFINITY ? 0.0f : st.m;      // only -inf so far: every term is 0
    float a = 0.0f, b = 0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) (e & 1 ? b : a) += exp_from(x[e], ref);
    st.s += a + b;
}
__device__ __forceinline__ NatState merge(const NatState& a, const NatState& b) {
    const float m = fmaxf(a.m, b.m), ref = m == -INFINITY ? 0.0f : m;
    return NatState{m, a.s * exp_from(a.m, ref) + b.s * exp_from(b.m, ref)};
}
template <int WIDTH>
__device__ __forceinline__ NatState group_merge_nat(NatState st) {
#pragma unroll
    for (int o = WIDTH / 2; o > 0; o >>= 1)
        st = merge(st, NatState{__shfl_xor_sync(0xFFFFFFFFu, st.m, o), __shfl_xor_sync(0xFFFFFFFFu, st.s, o)});
    return st;
}
__device__ __forceinline__ float row_loss(const NatState& st, float label_logit) { return (st.m - label_logit) + lg2_approx(st.s) * kLn2; }

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
    for (int64_t v = rank; v < nvec; v += nthreads) {
        const int64_t c = head + v * VE;
        float x[VE];
        Vec<T>::unpack(*reinterpret_cast<const uint4*>(row + c), x);
#pragma unroll
        for (int e = 0; e < VE; ++e) x[e] = at(x[e], c + e);
        if constexpr (VE == 8) store8(out + c, x);
        else *reinterpret_cast<float4*>(out + c) = make_float4(x[0], x[1], x[2], x[3]);
    }
    for (int64_t c = rank; c < head; c += nthreads) store1(out + c, at(load1(row + c), c));
    for (int64_t c = head + nvec * VE + rank; c < cols; c += nthreads) store1(out + c, at(load1(row + c), c));
}

template <typename T>
__device__ __forceinline__ void zero_row(T* out, int64_t cols, int rank, int nthreads) {
    for (int64_t c = rank; c < cols; c += nthreads) store1(out + c, 0.0f);
}

// ------------------------------------------------------------------------------------------- rows in registers

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
    float m, s;
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
        eh = exp_from(eh, ref);
        et = exp_from(et, ref);
        float s0 = eh, s1 = et;
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                e[k][i] = exp_from(e[k][i], ref);
                (i & 1 ? s1 : s0) += e[k][i];
            }
        s = s0 + s1;
    }
    // What turns this thread's exponentials into g p.  A thread that saw only -inf holds zeros; a row of nothing else is NaN, as its loss is.
    __device__ __forceinline__ float factor(const NatState& all, float g) const {
        return (m == -INFINITY && all.m != -INFINITY ? 0.0f : exp_from(m, all.m)) * (g / all.s);
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

constexpr int kRingThreads = 480;          // consumers; with the producer warp 16 warps, 128 registers a thread
constexpr int kRingVecs = 9;               // vectors per consumer: slices of up to 67.5 KB
constexpr int kRingSliceVecs = 4096;       // ... of which 64 KB are used: three stages
constexpr int kRingMaxStages = 6;
constexpr int kMaxCluster = 8;

// What the producer hands over with a row.
struct RingRow {
    int64_t row;               // -1: no more rows
    float g, label_logit;
    int y;
    float ends[16];            // head elements, then tail elements
};
struct RingControl {
    uint64_t full[kRingMaxStages], empty[kRingMaxStages], joined[2];
    RingRow meta[kRingMaxStages];
    NatState warp_state[2][kRingThreads / 32];
    NatState peer[2][kMaxCluster];
    int abort_flag;
};

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
// All consumers: true iff `ok` in every one of them.
__device__ __forceinline__ bool consumers_all(bool ok) {
    int r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 p, %1, 0;\n\tbarrier.red.and.pred q, 1, %2, p;\n\tselp.s32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"((int)ok), "n"(kRingThreads) : "memory");
    return r != 0;
}
// This CTA's row state into every CTA of the cluster; completes one arrival on their barriers.
__device__ __forceinline__ void send_state(NatState* slot, uint64_t* bar, int rank, const NatState& st) {
    uint32_t a, b;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(slot)), "r"(rank));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(b) : "r"(smem_u32(bar)), "r"(rank));
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(a), "f"(st.m), "f"(st.s) : "memory");
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(b) : "memory");
}
__device__ __forceinline__ bool wait_states(uint64_t* bar, uint32_t parity, volatile int* abort_flag) {
    const long long t0 = clock64();
    while (true) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(smem_u32(bar)), "r"(parity)
            : "memory");
        if (ok) return true;
        if (*abort_flag || clock64() - t0 > kWaitCycles) return false;
    }
}
__device__ __forceinline__ void bulk_s2g(void* dst, const void* src_smem, uint32_t bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(dst), "r"(smem_u32(src_smem)), "r"(bytes) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
template <int N>
__device__ __forceinline__ void bulk_wait_read() {
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory");
}

// A cluster of `C` CTAs per row, rows handed out in turn; CTA `rank` owns the vectors [rank * per, rank * per + nv) of a row.
template <typename T>
__global__ void __launch_bounds__(kRingThreads + 32) row_grad_ring_kernel(GradParams p, int C, int stages, int stage_bytes) {
    constexpr int VE = Vec<T>::kElems;
    extern __shared__ uint4 smem16[];
    __shared__ RingControl ctl;
    grid_dependency_wait();
    grid_dependency_release();
    const int rank = (int)(blockIdx.x % C), cols = (int)p.loss.cols;
    const int64_t first = blockIdx.x / C, step = gridDim.x / C;
    const int64_t n_inst = counted(p.count_dev, p.n_inst);
    char* ring = reinterpret_cast<char*>(smem16);
    volatile int* abort_flag = &ctl.abort_flag;
    if (threadIdx.x == 0) {
        for (int i = 0; i < stages; ++i) {
            mbar_init(&ctl.full[i], 1);
            mbar_init(&ctl.empty[i], 1);
        }
        mbar_init(&ctl.joined[0], C);
        mbar_init(&ctl.joined[1], C);
        ctl.abort_flag = 0;
        mbar_fence_init();
    }
    __syncthreads();
    cluster_sync();                        // nobody sends before every barrier stands
    if (threadIdx.x >= kRingThreads) {
        // ---- producer warp: looks a row's factor and label up, fetches its ends and its slice
        const int lane = threadIdx.x & 31;
        if (p.offsets && blockIdx.x == 0) {
            bool bad = false;
            for (int64_t s = lane; s < n_inst; s += 32) {
                const int a = __ldg(p.offsets + s), b = __ldg(p.offsets + s + 1);
                bad |= a < 0 || b < a || b > p.loss.rows;
            }
            if (bad) latch(p.loss.ctl, AA_ERR_BAD_INDEX);
        }
        int64_t j = 0;
        bool ok = true, more = true;
        for (int64_t r0 = first; ok && more; r0 += 32 * step) {
            // a lane per row: 32 rows' searches, labels and label logits cost one chain of loads
            const int64_t mine = r0 + lane * step;
            float my_g = 0.0f, my_logit = 0.0f;
            int my_y = -2;                 // not counted
            if (mine < p.loss.rows && row_factor(p, n_inst, mine, my_g)) {
                my_y = checked_label(p.loss, mine);
                if (my_y >= 0) my_logit = load1(static_cast<const T*>(p.loss.logits) + mine * p.loss.row_stride + my_y);
            }
            for (int i = 0; i < 32; ++i) {
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
                const int per = (sp.nvec + C - 1) / C, nv = more && y >= 0 ? max(0, min(per, sp.nvec - rank * per)) : 0;
                // one copy per lane: many in flight at once (the barrier's phase cannot complete before lane 0's arrival below)
                const int piece = (nv + 31) >> 5, v0 = lane * piece, n = min(piece, nv - v0);
                if (lane == 0) mbar_expect_tx(&ctl.full[stage], (uint32_t)nv * 16u);
                __syncwarp();
                if (n > 0) bulk_g2s(ring + (size_t)stage * stage_bytes + v0 * 16, row + sp.head + ((int64_t)rank * per + v0) * VE, (uint32_t)n * 16u, &ctl.full[stage]);
                float end = 0.0f;          // lanes 0..7: head, 8..15: tail
                if (more && y >= 0 && lane < sp.head) end = load1(row + lane);
                if (more && y >= 0 && lane >= 8 && lane < 16 && sp.tail0 + lane - 8 < cols) end = load1(row + sp.tail0 + lane - 8);
                RingRow* meta = &ctl.meta[stage];
                if (lane < 16) meta->ends[lane] = end;
                __syncwarp();
                if (lane == 0) {
                    meta->row = more ? r : -1;
                    meta->g = g;
                    meta->y = y;
                    meta->label_logit = label_logit;
                    mbar_arrive(&ctl.full[stage]);
                }
                ++j;
                if (!more) break;
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
        const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
        bool ok = true;
        int64_t joins = 0;
        for (int64_t j = 0;; ++j) {
            const int stage = (int)(j % stages), turn = (int)(j & 1);
            ok = mbar_wait(&ctl.full[stage], (uint32_t)((j / stages) & 1), abort_flag);
            const RingRow* meta = &ctl.meta[stage];
            const int64_t r = ok ? meta->row : 0;
            const int y = ok ? meta->y : -1;
            const T* row = static_cast<const T*>(p.loss.logits) + (r < 0 ? 0 : r) * p.loss.row_stride;
            T* out = static_cast<T*>(p.grad) + (r < 0 ? 0 : r) * p.grad_stride;
            const RowSpan<T> sp(row, cols);
            const int per = (sp.nvec + C - 1) / C, nv = max(0, min(per, sp.nvec - rank * per));
            T* body = reinterpret_cast<T*>(ring + (size_t)stage * stage_bytes);
            // the row's ends: rank 0 has the head, the last rank the tail
            const int nh = rank == 0 ? sp.head : 0, nt = rank == C - 1 ? cols - sp.tail0 : 0;
            RowPart<T, kRingVecs> part;
            if (y >= 0) {
                part.eh = tid < nh ? meta->ends[tid] : -INFINITY;
                part.et = tid < nt ? meta->ends[8 + tid] : -INFINITY;
                part.load_body(body, nv, tid, kRingThreads);
                part.exponentials();
                const NatState mine = group_merge_nat<32>(NatState{part.m, part.s});
                if (lane == 0) ctl.warp_state[turn][warp] = mine;
            }
            const float g = ok ? meta->g : 0.0f, label_logit = ok ? meta->label_logit : 0.0f;
            if (!consumers_all(ok)) {
                ok = false;
                break;
            }
            if (r < 0) break;              // every consumer has seen the same hand-over
            float f = 0.0f;
            if (y >= 0) {
                NatState all = group_merge_nat<16>((lane & 15) < kRingThreads / 32 ? ctl.warp_state[turn][lane & 15] : NatState{-INFINITY, 0.0f});
                if (C > 1) {
                    const int slot = (int)(joins & 1);
                    if (tid < C) send_state(&ctl.peer[slot][rank], &ctl.joined[slot], tid, all);
                    ok = wait_states(&ctl.joined[slot], (uint32_t)((joins >> 1) & 1), abort_flag);
                    ++joins;
                    all = ctl.peer[slot][0];
                    for (int c = 1; c < C; ++c) all = merge(all, ctl.peer[slot][c]);
                }
                f = part.factor(all, g);
                const int at = y - sp.head - rank * per * VE;
                part.store_body(body, nv, tid, kRingThreads, f, y >= sp.head && y < sp.tail0 && at >= 0 && at < nv * VE ? at : -1, label_grad(all, label_logit, g));
                if (p.loss.out && rank == 0 && tid == 0) p.loss.out[r] = row_loss(all, label_logit);
            } else {
                for (int v = tid; v < nv; v += kRingThreads) reinterpret_cast<uint4*>(body)[v] = make_uint4(0, 0, 0, 0);
                if (p.loss.out && rank == 0 && tid == 0) p.loss.out[r] = 0.0f;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            if (tid < nh) store1(out + tid, y >= 0 ? fmaf(part.eh, f, tid == y ? -g : 0.0f) : 0.0f);
            if (tid < nt) store1(out + sp.tail0 + tid, y >= 0 ? fmaf(part.et, f, sp.tail0 + tid == y ? -g : 0.0f) : 0.0f);
            if (!consumers_all(ok)) {
                ok = false;
                break;
            }
            if (warp == 0) {
                const int piece = (nv + 31) >> 5, v0 = lane * piece, n = min(piece, nv - v0);
                if (n > 0) bulk_s2g(out + sp.head + ((int64_t)rank * per + v0) * VE, body + (int64_t)v0 * VE, (uint32_t)n * 16u);
                else asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                // the previous row's copies have been read out of their stage once only these are pending
                bulk_wait_read<1>();
                __syncwarp();
                if (lane == 0 && j > 0) mbar_arrive(&ctl.empty[(j - 1) % stages]);
            }
        }
        if (!ok) {
            ctl.abort_flag = 1;
            if (tid == 0) latch(p.loss.ctl, AA_ERR_SCAN_TIMEOUT);
        }
        if (warp == 0) bulk_wait_read<0>();
    }
    __syncthreads();
    cluster_sync();                        // peers may still send here until they are done
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

template <typename T>
__global__ void __launch_bounds__(256) row_grad_cta_kernel(GradParams p) {
    __shared__ NatState warp_state[8];
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
            zero_row<T>(out, p.loss.cols, threadIdx.x, 256);
            if (p.loss.out && threadIdx.x == 0) p.loss.out[r] = 0.0f;
            continue;
        }
        const float label_logit = load1(row + y);
        NatState st = {-INFINITY, 0.0f};
        scan_row_nat<T>(st, row, p.loss.cols, threadIdx.x, 256);
        st = group_merge_nat<32>(st);
        __syncthreads();                                 // the previous row's states have been read
        if (lane == 0) warp_state[warp] = st;
        __syncthreads();
        st = group_merge_nat<32>(lane < 8 ? warp_state[lane] : NatState{-INFINITY, 0.0f});
        write_row<T>(row, out, p.loss.cols, st.m, g / st.s, g, y, threadIdx.x, 256);
        if (p.loss.out && threadIdx.x == 0) p.loss.out[r] = row_loss(st, label_logit);
    }
}

template <typename T>
aa_status launch_ring(aa_ctx_impl* c, GradParams& p, int C) {
    const void* kernel = (const void*)row_grad_ring_kernel<T>;
    const int64_t vecs = p.loss.cols * (int64_t)sizeof(T) / 16;
    int stage_bytes = (int)((vecs + C - 1) / C * 16 + 127) / 128 * 128;
    int stages = 210 * 1024 / stage_bytes;
    if (stages > kRingMaxStages) stages = kRingMaxStages;
    const size_t smem = (size_t)stages * stage_bytes;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return AA_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kRingThreads + 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = c->stream;
    cudaLaunchAttribute attrs[2];
    attrs[0].id = cudaLaunchAttributeClusterDimension;
    attrs[0].val.clusterDim.x = (unsigned)C;
    attrs[0].val.clusterDim.y = attrs[0].val.clusterDim.z = 1;
    attrs[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attrs[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attrs;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3((unsigned)(c->sm_count / C * C));
    int clusters = resident_clusters(c, kernel, &cfg, C);
    if (clusters < 1) return AA_ERR_CUDA;
    if (clusters > p.loss.rows) clusters = (int)p.loss.rows;
    cfg.gridDim = dim3((unsigned)(clusters * C));
    cfg.numAttrs = 2;
    void* args[] = {&p, &C, &stages, &stage_bytes};
    if (cudaLaunchKernelExC(&cfg, kernel, args) != cudaSuccess) return AA_ERR_CUDA;
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
    } else if (alike && vecs <= (int64_t)kRingSliceVecs * kMaxCluster) {
        int C = 1;
        while ((vecs + C - 1) / C > kRingSliceVecs) C *= 2;
        return launch_ring<T>(c, p, C);
    } else if (row_bytes > 8 * 1024) {
        kernel = (const void*)row_grad_cta_kernel<T>;
        want = p.loss.rows;
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
