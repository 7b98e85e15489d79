// Pieces shared by the operators that train the Boss on a generated batch: the counter-based draws of dropout, keyed by instance,
// and the ragged-batch bookkeeping (segment of a row, checks of the offsets).
#pragma once

#include "aa_internal.cuh"

namespace aa {

// Dropout rule as a kernel takes it.  thr == 0: nothing is dropped.
struct DropRule {
    uint32_t thr;            // an element is dropped iff its 16-bit draw is below
    float scale;             // 65536 / (65536 - thr)
    uint32_t seed_lo, seed_hi, step_lo, step_hi, site;
    const int32_t* row_idx;
    int64_t id_base;
};

struct RowsArg {             // one matrix operand
    const void* data;
    int64_t stride;          // elements
};

// Column numbers are 32 bits and those of the last unit's idle lanes pass the row's end, by less than 1,024.
constexpr int64_t kMaxDropoutCols = 0x7FFFFFFFll - 1023;

struct DropParams {
    RowsArg x, res, out;     // res.data nullable
    int64_t rows, cols;
    const int32_t* offsets;  // nullable
    int64_t n_inst;          // rows, or segments with offsets
    const int32_t* count_dev;
    DropRule rule;
    Control* ctl;
};

bool make_drop_rule(const aa_dropout_rule* r, DropRule& out);   // false: malformed
aa_status launch_dropout(aa_ctx_impl* c, const DropParams& p, int dtype);
aa_status launch_instance_loss_grad(aa_ctx_impl* c, const aa_logits& lg, const int32_t* labels, const int32_t* offsets, int64_t n_seg,
                                    const int32_t* count_dev, const float* weight, float scale, int mean, float* out_loss, const aa_rows& grad);
// Sums of row losses per segment; only the first min(*count_dev, n_seg) segments are written.
aa_status launch_segment_sum(aa_ctx_impl* c, const float* row_loss, const int32_t* offsets, int64_t n_seg, const int32_t* count_dev,
                             int64_t rows, float* out);

#ifdef __CUDACC__

// The kernels that include this may start while the launch before theirs still runs (grid_dependency_wait).  What that launch may have written - lists,
// counts, offsets, weights, row statistics - is read by ordinary loads: those of the read-only path need memory that nothing writes meanwhile.

struct Words4 {
    uint32_t w[4];
};

// Philox4x32-10 (Salmon et al., SC'11), all four output words.
__device__ __forceinline__ Words4 philox4x32_10(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return Words4{{c0, c1, c2, c3}};
}

// Key of the draws of the instance with this id: words 2 and 3 of the block whose word 0 is the screen's draw.
__device__ __forceinline__ uint2 id_key(const DropRule& r, int64_t id) {
    const Words4 w = philox4x32_10((uint32_t)id, (uint32_t)((uint64_t)id >> 32), r.step_lo, r.step_hi, r.seed_lo, r.seed_hi);
    return make_uint2(w.w[2], w.w[3]);
}

__device__ __forceinline__ int64_t instance_row(const DropRule& r, int64_t instance) { return r.row_idx ? (int64_t)r.row_idx[instance] : instance; }
__device__ __forceinline__ uint2 instance_key(const DropRule& r, int64_t instance) { return id_key(r, r.id_base + instance_row(r, instance)); }

__device__ __forceinline__ Words4 draw_block(const DropRule& r, uint2 key, uint64_t block) {
    return philox4x32_10((uint32_t)block, (uint32_t)(block >> 32), r.site, 0u, key.x, key.y);
}

// min(*count_dev, n), or n.
__device__ __forceinline__ int64_t counted(const int32_t* count_dev, int64_t n) {
    if (!count_dev) return n;
    const int64_t c = *count_dev;
    return c < 0 ? 0 : (c < n ? c : n);
}

// The last segment s in [0, n) with offsets[s] <= r (0 if there is none); reads offsets[0..n-1] only, whatever they hold.
__device__ __forceinline__ int64_t find_segment(const int32_t* offsets, int64_t n, int64_t r) {
    int64_t lo = 0, hi = n;          // offsets[lo] <= r (or lo = 0), offsets[hi] > r (or hi = n)
    while (hi - lo > 1) {
        const int64_t mid = (lo + hi) >> 1;
        if ((int64_t)offsets[mid] <= r) lo = mid; else hi = mid;
    }
    return lo;
}

// The same by WIDTH lanes together (lane `l` of them, `mask` theirs): WIDTH probes a round instead of one.
template <int WIDTH>
__device__ __forceinline__ int64_t find_segment_lanes(const int32_t* offsets, int64_t n, int64_t r, int l, unsigned mask) {
    int64_t lo = 0, hi = n;
    while (hi - lo > 1) {
        const int64_t step = (hi - lo + WIDTH) / (WIDTH + 1);      // probes lo + step, lo + 2 step, ...
        const int64_t at = lo + (int64_t)(l + 1) * step;
        const bool below = at < hi && (int64_t)offsets[at] <= r;
        const int count = __popc(__ballot_sync(mask, below) & mask);  // offsets ascend: the probes that hold are the first ones
        const int64_t next = lo + (int64_t)(count + 1) * step;
        lo += (int64_t)count * step;
        hi = next < hi ? next : hi;
    }
    return lo;
}

// One CTA looks every counted segment's offsets over.
__device__ __forceinline__ void check_offsets(Control* ctl, const int32_t* offsets, int64_t n, int64_t rows) {
    bool bad = false;
    for (int64_t s = threadIdx.x; s < n; s += blockDim.x) {
        const int a = offsets[s], b = offsets[s + 1];
        bad |= a < 0 || b < a || b > rows;
    }
    if (bad) latch(ctl, AA_ERR_BAD_INDEX);
}

// Two floats as packed bf16, `lo` in the low half.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Eight consecutive elements, rounded once (to nearest even).  Pointers 16-byte aligned.
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
    *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&x)[8]) {
    *reinterpret_cast<uint4*>(p) =
        make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
}
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ void store1(float* p, float x) { *p = x; }
__device__ __forceinline__ void store1(uint16_t* p, float x) { *p = (uint16_t)pack_bf16(x, 0.0f); }

#endif  // __CUDACC__

}  // namespace aa
