// Checks of the matrices that the Boss operators take: element types, alignment, and operands that a call may not write into.
#pragma once

#include "aa_internal.cuh"

namespace aa {

inline bool elem_size(int32_t dtype, int64_t& es) {
    es = dtype == AA_BF16 ? 2 : 4;
    return dtype == AA_F32 || dtype == AA_BF16;
}

inline aa_status check_rows(const aa_rows* m) {
    int64_t es;
    if (!m || !elem_size(m->dtype, es) || m->rows < 0 || m->cols <= 0 || m->cols > 0x7FFFFFF0ll || m->row_stride < m->cols) return AA_ERR_INVALID_ARG;
    if (m->rows > 0 && !m->data) return AA_ERR_INVALID_ARG;
    return (uintptr_t)m->data % (uintptr_t)es ? AA_ERR_INVALID_ARG : AA_OK;
}

// Elements of an operand: data + r * row_step + h * head_step + [0, width), r < rows, h < heads.
struct Extent {
    const void* data;
    int64_t rows, row_step, heads, head_step, width;
};

// No element in common.  Operands whose address ranges interleave are told apart exactly if they have the same steps (views of one packed array);
// interleaving ranges of different steps count as an overlap.
inline bool apart(Extent a, Extent b, int64_t es) {
    if (a.rows <= 0 || b.rows <= 0) return true;
    const auto span = [](const Extent& x) { return (x.rows - 1) * x.row_step + (x.heads - 1) * x.head_step + x.width; };
    const int64_t d = ((int64_t)(uintptr_t)b.data - (int64_t)(uintptr_t)a.data) / es;
    if (d >= span(a) || -d >= span(b)) return true;
    // an axis of length one has no step
    if (a.rows == 1) a.row_step = b.row_step;
    if (b.rows == 1) b.row_step = a.row_step;
    if (a.heads == 1) a.head_step = b.head_step;
    if (b.heads == 1) b.head_step = a.head_step;
    if (a.row_step != b.row_step || a.head_step != b.head_step) return false;
    // element (r1, h1, e1) of a is (r2, h2, e2) of b:  e1 - e2 = d - (r1 - r2) row_step - (h1 - h2) head_step
    const int64_t lo = 1 - b.width, hi = a.width - 1, step = a.row_step;
    for (int64_t h = 1 - b.heads; h < a.heads; ++h) {
        const int64_t left = d - h * a.head_step;
        if (step == 0) {
            if (left >= lo && left <= hi) return false;
            continue;
        }
        int64_t r = (left - hi) / step;                     // the smallest r with left - r step <= hi
        if (r * step < left - hi) ++r;
        if (r < 1 - b.rows) r = 1 - b.rows;
        if (r < a.rows && left - r * step >= lo) return false;
    }
    return true;
}

// `out` written while `in` is read: the same matrix, or nothing in common.
inline bool same_or_apart(const void* in, int64_t in_stride, const void* out, int64_t out_stride, int64_t rows, int64_t cols, int64_t es) {
    if (in == out) return in_stride == out_stride || rows <= 1;
    return apart(Extent{in, rows, in_stride, 1, 0, cols}, Extent{out, rows, out_stride, 1, 0, cols}, es);
}

inline bool same_shape(const aa_rows& a, const aa_rows& b) { return a.dtype == b.dtype && a.rows == b.rows && a.cols == b.cols; }

}  // namespace aa
