// One AdamW step over a list of tensors (see the header for the formulas and the 8-bit states).
//
// Bound by memory: with fp32 moments 24 bytes an element are read and written for the moments and parameters and 2 to 6 for gradient and copy; with e4m3
// moments 12 and 2 to 6.  The list travels in the kernel's parameters, so that a step is one launch for up to 256 tensors and nothing is
// copied to the device; a CTA finds its tensor by bisection over the running number of chunks.  A warp owns 256 consecutive elements, which is
// one block of the 8-bit states: two runs of 128, four elements a lane in each, so that every access is contiguous over the warp, a lane's
// four elements share one block of random words and the block's largest magnitude is a warp reduction.
// 51.7 M parameters, bf16 gradients and copies: fp32 moments 219 us (1.44 GB, 6.5 TB/s: the copy rate); e4m3 moments 258 us (0.83 GB, 3.2 TB/s), bound by
// 111 instructions an element, of which the draws, the decoding and the rounding to codes are most (64 % of the issue slots in use).
// What is rounded to a code comes of products, sums and roots that are each rounded by themselves: the code depends on its last bits.
#include <math.h>

#include "boss_common.cuh"

namespace aa {

namespace {

constexpr int kWarpsPerCta = 8, kPerCta = kWarpsPerCta * 256 * 4;      // a warp takes four blocks, one after the other

struct Entry {
    float* param;
    const void* grad;
    void *m, *v;
    uint8_t *m_scale, *v_scale;
    uint16_t* copy;
    int64_t n;
    float keep;              // 1 - lr weight_decay
    uint32_t first;          // chunks of the entries before
    uint32_t index;          // in the caller's list
    uint32_t flags;          // 1: bf16 gradient, 2: arrays aligned for vectors
};

template <int N>
struct Table {
    Entry e[N];
    int n;
    float b1, c1, b2, c2;    // betas and 1 - beta
    float rate, root, eps;   // lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
    uint32_t t_lo, t_hi, keys[20];   // round keys of the draws
    const float* grad_scale;
};

// Philox4x32-10 of counter (c0, c1, t) under keys that the host has laid out round by round.
template <int N>
__device__ __forceinline__ Words4 draw(const Table<N>& tab, uint32_t c0, uint32_t c1) {
    uint32_t c2 = tab.t_lo, c3 = tab.t_hi;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ tab.keys[2 * r];
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ tab.keys[2 * r + 1];
        c3 = (uint32_t)a;
    }
    return Words4{{c0, c1, c2, c3}};
}

__device__ __forceinline__ void decode4(uint32_t w, float unit, float (&x)[4]) {
    uint32_t a, b;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}" : "=r"(a), "=r"(b) : "r"(w));
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, h;\n\t}" : "=f"(x[0]), "=f"(x[1]) : "r"(a));
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.f32.f16 %0, l;\n\tcvt.f32.f16 %1, h;\n\t}" : "=f"(x[2]), "=f"(x[3]) : "r"(b));
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __fmul_rn(x[i], unit);
}
__device__ __forceinline__ uint32_t encode4(const float (&y)[4]) {
    uint32_t w;
    asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
        : "=r"(w)
        : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]));
    return w;
}

// x in units, |x| < 256 -> a neighbouring e4m3 number, by the low 16 bits of w.  Below 2^-6 the steps are those of [2^-6, 2^-5).
__device__ __forceinline__ float to_e4m3(float x, uint32_t w) {
    const float lift = fabsf(x) < 0.015625f ? 0.015625f : 0.0f;
    const float y = __uint_as_float((__float_as_uint(__fadd_rn(fabsf(x), lift)) + ((w & 0xFFFFu) << 4)) & 0xFFF00000u);
    return copysignf(__fadd_rn(y, -lift), x);
}
// The same for a root x >= 0 whose square is to keep its mean, by the high 16 bits of w.  (z - y)(z + y) of two neighbours has few bits and is exact in any
// order.  LOW: x may be below 2^-6.
template <bool LOW>
__device__ __forceinline__ float root_to_e4m3(float x, uint32_t w) {
    const float lift = LOW && x < 0.015625f ? 0.015625f : 0.0f;
    const uint32_t bits = __float_as_uint(LOW ? __fadd_rn(x, lift) : x) & 0xFFF00000u;
    float y = __uint_as_float(bits), z = __uint_as_float(bits + 0x100000u);
    if (LOW) {
        y = __fadd_rn(y, -lift);
        z = __fadd_rn(z, -lift);
    }
    const float u = __fadd_rn(__uint_as_float((w >> 9 & 0x7FFF80u) | 0x3F800000u), -1.0f);      // the 16 bits over 65,536
    y = __fmul_rn(__fadd_rn(x, -y), __fadd_rn(x, y)) > __fmul_rn(u, __fmaf_rn(z, z, -__fmul_rn(y, y))) ? z : y;
    return LOW && x > 0.0f ? fmaxf(y, 0.001953125f) : y;   // 2^-9 at least
}

__device__ __forceinline__ float sqrt_approx(float x) {
    float y;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Scale of a block from the bits of its largest magnitude (those of an infinity or NaN are larger than any number's).
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) { return top ? (uint32_t)max((int)(top >> 23) - 7, 1) : 0u; }

template <bool VEC>
__device__ __forceinline__ void load4(const float* p, int64_t left, float (&x)[4]) {
    if (VEC && left >= 4) {
        const float4 v = *reinterpret_cast<const float4*>(p);
        x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = i < left ? p[i] : 0.0f;
    }
}
template <bool VEC>
__device__ __forceinline__ void store4(float* p, int64_t left, const float (&x)[4]) {
    if (VEC && left >= 4) {
        *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) p[i] = x[i];
    }
}
template <bool VEC>
__device__ __forceinline__ void store4(uint16_t* p, int64_t left, const float (&x)[4]) {
    if (VEC && left >= 4) {
        *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) store1(p + i, x[i]);
    }
}
template <bool VEC>
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int64_t left) {
    if (VEC && left >= 4) return *reinterpret_cast<const uint32_t*>(p);
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left) w |= (uint32_t)p[i] << (8 * i);
    return w;
}
template <bool VEC>
__device__ __forceinline__ void store_codes(uint8_t* p, int64_t left, uint32_t w) {
    if (VEC && left >= 4) {
        *reinterpret_cast<uint32_t*>(p) = w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < left) p[i] = (uint8_t)(w >> (8 * i));
    }
}

// A lane's eight elements of a block as they lie in memory.
template <int BITS>
struct Fetched {
    float p[2][4], g[2][4];                  // g: the words of a bf16 gradient until `widen`
    float m[2][4], v[2][4];                  // BITS 32
    uint32_t mc[2], vc[2], mb, vb;           // BITS 8
};

template <int BITS, bool VEC>
__device__ __forceinline__ void fetch(const Entry& e, int64_t block, Fetched<BITS>& f) {
    const int lane = threadIdx.x & 31;
    if (BITS == 8) {
        f.mb = e.m_scale[block];
        f.vb = e.v_scale[block];
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t at = block * 256 + h * 128 + lane * 4, left = e.n - at;
        load4<VEC>(e.param + at, left, f.p[h]);
        if (!(e.flags & 1)) {
            load4<VEC>(static_cast<const float*>(e.grad) + at, left, f.g[h]);
        } else if (VEC && left >= 4) {
            const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(e.grad) + at);
            f.g[h][0] = __uint_as_float(w.x);
            f.g[h][1] = __uint_as_float(w.y);
        } else {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = i < left ? static_cast<const uint16_t*>(e.grad)[at + i] : 0u;
            f.g[h][0] = __uint_as_float(w[0] | w[1] << 16);
            f.g[h][1] = __uint_as_float(w[2] | w[3] << 16);
        }
        if (BITS == 32) {
            load4<VEC>(static_cast<const float*>(e.m) + at, left, f.m[h]);
            load4<VEC>(static_cast<const float*>(e.v) + at, left, f.v[h]);
        } else {
            f.mc[h] = load_codes<VEC>(static_cast<const uint8_t*>(e.m) + at, left);
            f.vc[h] = load_codes<VEC>(static_cast<const uint8_t*>(e.v) + at, left);
        }
    }
}

template <int N, int BITS, bool VEC>
__device__ __forceinline__ void update(const Table<N>& tab, const Entry& e, int64_t block, float gs, Fetched<BITS>& f) {
    const int lane = threadIdx.x & 31;
    uint32_t m_top = 0, v_top = 0;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (BITS == 8) {
            decode4(f.mc[h], __uint_as_float(f.mb << 23), f.m[h]);
            decode4(f.vc[h], __uint_as_float(f.vb << 23), f.v[h]);
        }
        if (e.flags & 1) {
            const uint32_t a = __float_as_uint(f.g[h][0]), b = __float_as_uint(f.g[h][1]);
            f.g[h][0] = bf16_lo(a), f.g[h][1] = bf16_hi(a), f.g[h][2] = bf16_lo(b), f.g[h][3] = bf16_hi(b);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float &p = f.p[h][i], &m = f.m[h][i], &v = f.v[h][i];
            const float x = tab.grad_scale ? __fmul_rn(f.g[h][i], gs) : f.g[h][i];
            if (BITS == 8) v = __fmul_rn(v, v);
            m = __fadd_rn(__fmul_rn(m, tab.b1), __fmul_rn(x, tab.c1));
            v = __fadd_rn(__fmul_rn(v, tab.b2), __fmul_rn(__fmul_rn(x, x), tab.c2));
            // the step itself is nobody's border: quotient and root to two units of the last place
            float den;
            if (BITS == 8) {
                v = __fsqrt_rn(v);
                m_top = max(m_top, __float_as_uint(m) & 0x7FFFFFFFu);
                v_top = max(v_top, __float_as_uint(v) & 0x7FFFFFFFu);
                den = fmaf(v, tab.root, tab.eps);
            } else {
                den = fmaf(sqrt_approx(v), tab.root, tab.eps);
            }
            p = fmaf(-tab.rate, __fdividef(m, den), __fmul_rn(p, e.keep));
        }
        const int64_t at = block * 256 + h * 128 + lane * 4, left = e.n - at;
        store4<VEC>(e.param + at, left, f.p[h]);
        if (e.copy) store4<VEC>(e.copy + at, left, f.p[h]);
        if (BITS == 32) {
            store4<VEC>(static_cast<float*>(e.m) + at, left, f.m[h]);
            store4<VEC>(static_cast<float*>(e.v) + at, left, f.v[h]);
        }
    }
    if (BITS == 32) return;
    m_top = __reduce_max_sync(0xFFFFFFFFu, m_top);
    v_top = __reduce_max_sync(0xFFFFFFFFu, v_top);
    const uint32_t mb = scale_byte(m_top), vb = scale_byte(v_top);
    const float mi = mb ? __uint_as_float((254u - mb) << 23) : 1.0f, vi = vb ? __uint_as_float((254u - vb) << 23) : 1.0f;
    float least = 256.0f;                    // root: moments that nothing moved for long are rare
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f.v[h][i] = __fmul_rn(f.v[h][i], vi);
            least = fminf(least, f.v[h][i]);
        }
    const bool low = __any_sync(0xFFFFFFFFu, !(least >= 0.015625f));
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const Words4 w = draw(tab, (uint32_t)((block * 256 + h * 128) >> 2) + lane, e.index);
#pragma unroll
        for (int i = 0; i < 4; ++i) f.m[h][i] = to_e4m3(__fmul_rn(f.m[h][i], mi), w.w[i]);
        if (low) {
#pragma unroll
            for (int i = 0; i < 4; ++i) f.v[h][i] = root_to_e4m3<true>(f.v[h][i], w.w[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) f.v[h][i] = root_to_e4m3<false>(f.v[h][i], w.w[i]);
        }
    }
    // the codes of a block with an infinity or NaN are no numbers
    const bool numbers = max(m_top, v_top) < 0x7F800000u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t at = block * 256 + h * 128 + lane * 4, left = e.n - at;
        store_codes<VEC>(static_cast<uint8_t*>(e.m) + at, left, numbers ? encode4(f.m[h]) : 0x7F7F7F7Fu);
        store_codes<VEC>(static_cast<uint8_t*>(e.v) + at, left, numbers ? encode4(f.v[h]) : 0x7F7F7F7Fu);
    }
    if (lane == 0) {
        e.m_scale[block] = (uint8_t)mb;
        e.v_scale[block] = (uint8_t)vb;
    }
}

// A warp's blocks.  With fp32 moments the next one's loads are under way while one is worked on; with e4m3 ones, which take four times the arithmetic, the
// registers are better spent on more warps.
template <int N, int BITS, bool VEC>
__device__ __forceinline__ void run(const Table<N>& tab, const Entry& e, int64_t block, float gs) {
    constexpr int kBlocks = kPerCta / 256 / kWarpsPerCta;
    Fetched<BITS> now, next;
    if (block * 256 >= e.n) return;
    if (BITS == 32) fetch<BITS, VEC>(e, block, now);
#pragma unroll 1
    for (int i = 0; i < kBlocks; ++i, block += kWarpsPerCta) {
        const int64_t after = block + kWarpsPerCta;
        const bool more = i + 1 < kBlocks && after * 256 < e.n;
        if (BITS == 8) fetch<BITS, VEC>(e, block, now);
        else if (more) fetch<BITS, VEC>(e, after, next);
        update<N, BITS, VEC>(tab, e, block, gs, now);
        if (!more) return;
        if (BITS == 32) now = next;
    }
}

template <int N, int BITS>
__global__ void __launch_bounds__(kWarpsPerCta * 32, BITS == 8 ? 5 : 3) adamw_kernel(const __grid_constant__ Table<N> tab) {
    __shared__ Entry entry;                  // out of the parameters, where every access by a computed index would be a trip of its own
    if (threadIdx.x < 32) {
        int lo = 0, hi = tab.n;              // the last entry with first <= blockIdx.x
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (tab.e[mid].first <= blockIdx.x) lo = mid; else hi = mid;
        }
        const uint32_t* from = reinterpret_cast<const uint32_t*>(&tab.e[lo]);
        if (threadIdx.x < sizeof(Entry) / 4) reinterpret_cast<uint32_t*>(&entry)[threadIdx.x] = from[threadIdx.x];
    }
    __syncthreads();
    const Entry& e = entry;
    const int64_t block = (int64_t)(blockIdx.x - e.first) * (kPerCta / 256) + (threadIdx.x >> 5);
    grid_dependency_wait();
    grid_dependency_release();
    float gs = 1.0f;
    if (tab.grad_scale) {
        gs = *tab.grad_scale;
        if (!(fabsf(gs) < INFINITY)) return;
    }
    if (e.flags & 2) run<N, BITS, true>(tab, e, block, gs);
    else run<N, BITS, false>(tab, e, block, gs);
}

template <int N, int BITS>
aa_status launch_some(aa_ctx_impl* c, const aa_adamw_tensor* t, int64_t count, const aa_adamw_rule* r, const float* grad_scale) {
    static_assert(sizeof(Table<N>) <= 32764, "kernel parameters");
    Table<N> tab;
    const double step = (double)(r->t + 1);
    tab.b1 = (float)r->beta1;
    tab.c1 = (float)(1.0 - r->beta1);
    tab.b2 = (float)r->beta2;
    tab.c2 = (float)(1.0 - r->beta2);
    tab.rate = (float)(r->lr / (1.0 - pow(r->beta1, step)));
    tab.root = (float)sqrt(1.0 / (1.0 - pow(r->beta2, step)));
    tab.eps = (float)r->eps;
    tab.t_lo = (uint32_t)(r->t + 1);
    tab.t_hi = (uint32_t)((uint64_t)(r->t + 1) >> 32);
    for (int i = 0; i < 10; ++i) {
        tab.keys[2 * i] = (uint32_t)r->seed + (uint32_t)i * 0x9E3779B9u;
        tab.keys[2 * i + 1] = (uint32_t)(r->seed >> 32) + (uint32_t)i * 0xBB67AE85u;
    }
    tab.grad_scale = grad_scale;
    int64_t at = 0;
    while (at < count) {
        tab.n = 0;
        uint32_t chunks = 0;
        for (; at < count && tab.n < N; ++at) {
            if (t[at].state_bits != BITS || t[at].n == 0) continue;
            const int64_t need = (t[at].n + kPerCta - 1) / kPerCta;
            if (chunks + need > 0x7FFFFFFFll) break;
            const auto on = [](const void* p, uintptr_t a) { return (uintptr_t)p % a == 0; };
            const bool bf16 = t[at].grad_dtype == AA_BF16, wide = BITS == 32;
            const bool vec = on(t[at].param, 16) && on(t[at].grad, bf16 ? 8 : 16) && on(t[at].m, wide ? 16 : 4) && on(t[at].v, wide ? 16 : 4) && on(t[at].copy, 8);
            tab.e[tab.n++] = Entry{t[at].param, t[at].grad, t[at].m, t[at].v, t[at].m_scale, t[at].v_scale, static_cast<uint16_t*>(t[at].copy), t[at].n,
                                   (float)(1.0 - r->lr * t[at].weight_decay), chunks, (uint32_t)at, (bf16 ? 1u : 0u) | (vec ? 2u : 0u)};
            chunks += (uint32_t)need;
        }
        if (tab.n == 0) break;
        void* args[] = {&tab};
        if (launch_overlapped(c, (const void*)adamw_kernel<N, BITS>, dim3(chunks), dim3(kWarpsPerCta * 32), args, 0, false) != cudaSuccess) return AA_ERR_CUDA;
        ++c->launches;
    }
    return AA_OK;
}

}  // namespace

}  // namespace aa

using namespace aa;

extern "C" aa_status aa_adamw(aa_ctx* ctx, const aa_adamw_tensor* tensors, int64_t n_tensors, aa_adamw_rule* rule, const float* grad_scale) {
    if (!ctx || !rule || n_tensors < 0 || (n_tensors > 0 && !tensors)) return AA_ERR_INVALID_ARG;
    const auto share = [](double x) { return x >= 0.0 && x < 1.0; };
    if (!(rule->lr >= 0.0) || !isfinite(rule->lr) || !share(rule->beta1) || !share(rule->beta2) || !(rule->eps >= 0.0) || !isfinite(rule->eps) || rule->t < 0)
        return AA_ERR_INVALID_ARG;
    if (n_tensors > 0x7FFFFFFFll) return AA_ERR_UNSUPPORTED;
    int64_t wide = 0, narrow = 0;
    for (int64_t i = 0; i < n_tensors; ++i) {
        const aa_adamw_tensor& t = tensors[i];
        if (t.n < 0 || (t.grad_dtype != AA_F32 && t.grad_dtype != AA_BF16) || (t.state_bits != 32 && t.state_bits != 8) || !isfinite(t.weight_decay)) return AA_ERR_INVALID_ARG;
        if (t.n == 0) continue;
        if (t.n > (1ll << 33)) return AA_ERR_UNSUPPORTED;
        const bool bytes = t.state_bits == 8;
        if (!t.param || !t.grad || !t.m || !t.v || (bytes && (!t.m_scale || !t.v_scale))) return AA_ERR_INVALID_ARG;
        const uintptr_t es = t.grad_dtype == AA_BF16 ? 2 : 4;
        if ((uintptr_t)t.param % 4 || (uintptr_t)t.grad % es || (uintptr_t)t.copy % 2 || (!bytes && ((uintptr_t)t.m % 4 || (uintptr_t)t.v % 4))) return AA_ERR_INVALID_ARG;
        // [begin, end) of each array: nothing written may lie in another
        const uintptr_t n = (uintptr_t)t.n, sb = bytes ? 1 : 4, blocks = bytes ? (n + 255) / 256 : 0;
        const struct { uintptr_t at, size; } a[7] = {{(uintptr_t)t.param, 4 * n},     {(uintptr_t)t.m, sb * n},         {(uintptr_t)t.v, sb * n},   {(uintptr_t)t.copy, t.copy ? 2 * n : 0},
                                                      {(uintptr_t)t.m_scale, blocks}, {(uintptr_t)t.v_scale, blocks}, {(uintptr_t)t.grad, es * n}};
        for (int x = 0; x < 7; ++x)
            for (int y = 0; y < x; ++y)
                if (a[x].size && a[y].size && a[x].at < a[y].at + a[y].size && a[y].at < a[x].at + a[x].size) return AA_ERR_INVALID_ARG;
        ++(bytes ? narrow : wide);
    }
    aa_ctx_impl* c = reinterpret_cast<aa_ctx_impl*>(ctx);
    aa_status st = AA_OK;
    // a long list takes a longer parameter block, which costs a launch little and saves several
    if (wide) st = wide <= 32 ? launch_some<32, 32>(c, tensors, n_tensors, rule, grad_scale) : launch_some<256, 32>(c, tensors, n_tensors, rule, grad_scale);
    if (st == AA_OK && narrow) st = narrow <= 32 ? launch_some<32, 8>(c, tensors, n_tensors, rule, grad_scale) : launch_some<256, 8>(c, tensors, n_tensors, rule, grad_scale);
    if (st == AA_OK) ++rule->t;
    return st;
}
