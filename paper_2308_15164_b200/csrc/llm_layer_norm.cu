// Layer norm, forward and backward (abs_layer_norm*).
//
//     n = (x - mean) r w + b,  r = 1 / sqrt(mean (x - mean)^2 + eps)
// Backward with c = x - mean, xh = c r, a = dn w:  dx = dskip + r (a - mean(a)) - c r^3 mean(a c),  dw = sum dn xh,  db = sum dn.
// Plain sums of x and x^2 would lose what a large common offset leaves of the variance.  A CTA that owns a row takes all sums about
// a pivot p, the mean of 32 of the row's elements, which every warp finds on its own: one reduction of the CTA instead of two.  The
// pivot is usually within a fifth of a standard deviation of the mean; where it is more than two off (the 32 happen to be far from the rest),
// mean (x - p)^2 - (mean - p)^2 would lose digits, and the sums are taken again about the mean.  A warp that owns a row takes its mean first.  Bound by memory: forward 2, backward 3 (4 with dskip) elements per position.
#include <math.h>

#include <algorithm>

#include "abs_internal.h"
#include "abs_llm.h"
#include "llm_host.h"
#include "llm_status.cuh"
#include "row_ring.cuh"

namespace abs_sgd {
namespace {

constexpr int kWidthMax = 32768;
constexpr int kSms = 148;
constexpr int kColumnParts = 296;    // most parts of the rows for the plain column sums
constexpr int kRingCtasMax = 16;
// Threads of an SM for the ring kernels and CTAs of the form with a warp per row, by the elements that a thread owns: what the
// registers leave room for.
constexpr int ring_threads(bool back, int elems) { return back && elems == 32 ? 256 : 512; }
constexpr int warp_ctas(bool back, int elems) { return back ? 2 : elems == 8 ? 4 : 3; }
constexpr size_t warp_row(size_t es) { return es == 2 ? 384 : 256; }
// Elements of a thread: what a row costs a thread beside its elements (reductions, waits, addresses, some 150 instructions forward and 300
// backward) is spread over them, but fewer leave more warps.  us with 16 / 32, bf16, 2^26 elements forward and 2^25 backward with dskip:
//     columns       392        512        520        768       1024       1536       2048       4096       8192
//     forward    80 / 98    63 / 75   123 / 83    84 / 61    66 / 54    68 / 63    71 / 55    74 / 54    86 / 57
//     columns       512       1024       2048       3584       4000       4096       4608       6144       6152       7168       8192
//     backward   64 / 88    63 / 68    65 / 70    72 / 74    69 / 71    70 / 71    92 / 99    81 / 86    86 / 86    81 / 79    78 / 77
// (without dskip the same borders; forward rows of 520 to 1024 columns, but few of them: 16 elements up to a tenth faster).  fp32 (half the elements a
// byte) forward 512 columns 46 / 83, 2048 47 / 58, 8192 56 / 61; backward 512 38 / 55, 2048 36 / 40, 8192 45 / 46.
constexpr int ring_elems(bool back, size_t es, size_t D) {
    if (D <= 8 * 32) return 8;
    if (es == 4) return D <= 16 * 512 ? 16 : 32;
    return D <= (back ? 6144 : 512) ? 16 : 32;
}

struct LnArgs {
    const void *x, *dn, *skip;       // forward: x only
    size_t ld_x, ld_dn, ld_skip;
    const float *w, *b;
    float eps, inv_d;
    size_t T;
    int D;
    void* out;                       // n; backward dx
    size_t ld_out;
    float* part;                     // [CTA][2][part_width(D)]: sum dn xh, sum dn
    float2* stats;                   // [T]: mean, r (plain backward kernels)
    int stages;
    uint32_t row_bytes;
};

// The variance from the mean square about a pivot; a NaN stays one.
__device__ __forceinline__ float var_of(float square, float d) {
    const float v = square - d * d;
    return v < 0.f ? 0.f : v;
}

// The pivot is so far from the mean that the sums about it lose digits.
__device__ __forceinline__ bool far_off(float d, float var) { return d * d > 4.f * var; }

// kV consecutive elements at a time, kV = 1 for rows that are not 16-byte aligned.
template <typename T, int kV>
__global__ void __launch_bounds__(256) k_layer_norm_plain(const __grid_constant__ LnArgs a) {
    __shared__ float sh[8];
    pdl_wait();
    pdl_trigger();
    for (size_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + t * a.ld_x;
        T* n = static_cast<T*>(a.out) + t * a.ld_out;
        float s[1] = {0.f};
        for (int c = threadIdx.x * kV; c < a.D; c += 256 * kV) {
            float v[kV];
            Pack<T, kV>::load(x + c, v);
#pragma unroll
            for (int k = 0; k < kV; ++k) s[0] += v[k];
        }
        group_sum<256, 1>(s, sh);
        const float mean = s[0] * a.inv_d;
        s[0] = 0.f;
        for (int c = threadIdx.x * kV; c < a.D; c += 256 * kV) {
            float v[kV];
            Pack<T, kV>::load(x + c, v);
#pragma unroll
            for (int k = 0; k < kV; ++k) s[0] += (v[k] - mean) * (v[k] - mean);
        }
        group_sum<256, 1>(s, sh);
        const float r = 1.f / sqrtf(s[0] * a.inv_d + a.eps);
        for (int c = threadIdx.x * kV; c < a.D; c += 256 * kV) {
            float v[kV];
            Pack<T, kV>::load(x + c, v);
#pragma unroll
            for (int k = 0; k < kV; ++k) v[k] = (v[k] - mean) * r * a.w[c + k] + (a.b ? a.b[c + k] : 0.f);
            Pack<T, kV>::store(n + c, v);
        }
    }
}

// The backward pass of matrices that are not aligned alike and of rows too wide for a CTA's registers: every row's mean and r, the column sums (a
// CTA that kept them for whole rows would add them up in memory: 4096 x 16384 bf16 1660 us), then dx, which may take the place of x or dn.
template <typename T, int kV>
__global__ void __launch_bounds__(256) k_layer_norm_stats(const __grid_constant__ LnArgs a) {
    __shared__ float sh[8];
    pdl_wait();
    pdl_trigger();
    for (size_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + t * a.ld_x;
        float s[1] = {0.f};
        for (int c = threadIdx.x * kV; c < a.D; c += 256 * kV) {
            float v[kV];
            Pack<T, kV>::load(x + c, v);
#pragma unroll
            for (int k = 0; k < kV; ++k) s[0] += v[k];
        }
        group_sum<256, 1>(s, sh);
        const float mean = s[0] * a.inv_d;
        s[0] = 0.f;
        for (int c = threadIdx.x * kV; c < a.D; c += 256 * kV) {
            float v[kV];
            Pack<T, kV>::load(x + c, v);
#pragma unroll
            for (int k = 0; k < kV; ++k) s[0] += (v[k] - mean) * (v[k] - mean);
        }
        group_sum<256, 1>(s, sh);
        if (threadIdx.x == 0) a.stats[t] = make_float2(mean, 1.f / sqrtf(s[0] * a.inv_d + a.eps));
    }
}
template <typename T, int kV>
__global__ void __launch_bounds__(256) k_layer_norm_back_plain(const __grid_constant__ LnArgs a) {
    __shared__ float sh[16];
    pdl_wait();
    pdl_trigger();
    for (size_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + t * a.ld_x;
        const T* dn = static_cast<const T*>(a.dn) + t * a.ld_dn;
        const T* skip = a.skip ? static_cast<const T*>(a.skip) + t * a.ld_skip : nullptr;
        T* dx = static_cast<T*>(a.out) + t * a.ld_out;
        const float mean = a.stats[t].x, r = a.stats[t].y;
        float s[2] = {0.f, 0.f};                 // sum a, a c
        for (int c = threadIdx.x * kV; c < a.D; c += 256 * kV) {
            float v[kV], d[kV];
            Pack<T, kV>::load(x + c, v);
            Pack<T, kV>::load(dn + c, d);
#pragma unroll
            for (int k = 0; k < kV; ++k) {
                const float f = d[k] * a.w[c + k];
                s[0] += f;
                s[1] += f * (v[k] - mean);
            }
        }
        group_sum<256, 2>(s, sh);
        const float level = s[0] * a.inv_d, along = s[1] * a.inv_d * r;
        for (int c = threadIdx.x * kV; c < a.D; c += 256 * kV) {
            float v[kV], d[kV], o[kV];
            Pack<T, kV>::load(x + c, v);
            Pack<T, kV>::load(dn + c, d);
            if (skip) Pack<T, kV>::load(skip + c, o);
#pragma unroll
            for (int k = 0; k < kV; ++k) o[k] = (skip ? o[k] : 0.f) + r * (d[k] * a.w[c + k] - level - (v[k] - mean) * r * along);
            Pack<T, kV>::store(dx + c, o);
        }
    }
}

// A thread per column.
template <typename T>
__global__ void __launch_bounds__(256) k_layer_norm_columns(const __grid_constant__ LnArgs a) {
    pdl_wait();
    pdl_trigger();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.D) return;
    float w = 0.f, b = 0.f;
    for (size_t t = blockIdx.y; t < a.T; t += 8 * (size_t)gridDim.y) {
        float x[8], d[8];
        float2 s[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const size_t u = t + k * (size_t)gridDim.y;
            x[k] = d[k] = 0.f;
            s[k] = make_float2(0.f, 0.f);
            if (u >= a.T) continue;
            x[k] = to_f(static_cast<const T*>(a.x)[u * a.ld_x + c]);
            d[k] = to_f(static_cast<const T*>(a.dn)[u * a.ld_dn + c]);
            s[k] = a.stats[u];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            w = fmaf(d[k], (x[k] - s[k].x) * s[k].y, w);
            b += d[k];
        }
    }
    float* part = a.part + blockIdx.y * 2 * part_width(a.D);
    part[c] = w;
    part[part_width(a.D) + c] = b;
}

// The mean of 32 elements of the current row's image of input 0, the same in every warp.  The image has 32 elements at least.
template <typename R>
__device__ __forceinline__ float pivot_of(const R& r) {
    const uint32_t all = (uint32_t)r.cut.pieces * kVec<typename R::Element>;
    const auto* image = reinterpret_cast<const typename R::Element*>(r.base + (size_t)r.st * R::kInputs * r.row_bytes);
    float v = to_f(image[threadIdx.x % 32 * (all / 32)]);
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v * (1.f / 32.f);
}

// Rows through a ring of images (row_ring.cuh); a thread owns kP pieces of 16 bytes and at most one single element.
template <typename T, int kP, bool kWarp>
__global__ void __launch_bounds__(kWarp ? kRowWarps * 32 : ring_threads(false, kP * kVec<T>), kWarp ? warp_ctas(false, kP * kVec<T>) : 1)
    k_layer_norm(const __grid_constant__ LnArgs a) {
    constexpr int kN = kPairs<T>;
    extern __shared__ __align__(16) uint8_t smem[];
    const int warps = blockDim.x / 32;
    const size_t t0 = kWarp ? (size_t)blockIdx.x * kRowWarps + threadIdx.x / 32 : blockIdx.x, G = kWarp ? (size_t)gridDim.x * kRowWarps : gridDim.x;
    Ring<T, 1, kP, kWarp> r;
    r.in[0] = static_cast<const T*>(a.x); r.ld[0] = a.ld_x;
    r.begin(smem, a.T, a.D, a.stages, a.row_bytes, r.in[0] + t0 * a.ld_x);
    pdl_wait();
    pdl_trigger();
    if (kWarp || threadIdx.x == 0)
        for (int i = 0; i < r.stages; ++i) r.load(i, t0 + i * G);
    float nx[1] = {};
    r.load_extra(t0, nx);
    float2 w[kP][kN], b[kP][kN];
    const float xw = r.weights(a.w, nullptr, w);
    float xb = 0.f;
    if (a.b) xb = r.weights(a.b, nullptr, b);
    else
#pragma unroll
        for (int j = 0; j < kP; ++j)
#pragma unroll
            for (int i = 0; i < kN; ++i) b[j][i] = both(0.f);

    int k = 0;
    for (size_t t = t0; t < a.T; t += G, ++k, r.next()) {
        const float ex = nx[0];
        r.load_extra(t + G, nx);
        r.wait();
        float2 v[kP][kN], s2 = both(0.f), t2 = both(0.f);
        float pivot = 0.f, d, q;                     // v: x - pivot; d: mean - pivot
        if (!kWarp) pivot = pivot_of(r);
#pragma unroll
        for (int j = 0; j < kP; ++j)
            if (r.has(j)) {
                r.piece(0, j, v[j]);
#pragma unroll
                for (int i = 0; i < kN; ++i) {
                    if (!kWarp) {
                        v[j][i] = add2(v[j][i], both(-pivot));
                        t2 = fma2(v[j][i], v[j][i], t2);
                    }
                    s2 = add2(s2, v[j][i]);
                }
            }
        const float xc = ex - pivot;
        if (kWarp) {
            r.release(t, G, warps);
            float s[1] = {sum2(s2) + (r.extra >= 0 ? xc : 0.f)};
            row_sum<true>(s, nullptr, 1);
            d = s[0] * a.inv_d;
#pragma unroll
            for (int j = 0; j < kP; ++j)
                if (r.has(j))
#pragma unroll
                    for (int i = 0; i < kN; ++i) {
                        const float2 c = add2(v[j][i], both(-d));
                        t2 = fma2(c, c, t2);
                    }
            s[0] = sum2(t2) + (r.extra >= 0 ? (xc - d) * (xc - d) : 0.f);
            row_sum<true>(s, nullptr, 1);
            q = rsqrtf(s[0] * a.inv_d + a.eps);
        } else {
            float s[2] = {sum2(s2), sum2(t2)};
            if (r.extra >= 0) {
                s[0] += xc;
                s[1] += xc * xc;
            }
            row_sum<false>(s, r.ctl->red[k & 1], warps);
            // every warp has read this row's image: it is filled again at once
            if (threadIdx.x == 0) r.load(r.st, t + (size_t)r.stages * G);
            d = s[0] * a.inv_d;
            float var = var_of(s[1] * a.inv_d, d);
            if (far_off(d, var)) {                   // the same for all threads
                t2 = both(0.f);
#pragma unroll
                for (int j = 0; j < kP; ++j)
                    if (r.has(j))
#pragma unroll
                        for (int i = 0; i < kN; ++i) {
                            const float2 c = add2(v[j][i], both(-d));
                            t2 = fma2(c, c, t2);
                        }
                float u[1] = {sum2(t2) + (r.extra >= 0 ? (xc - d) * (xc - d) : 0.f)};
                row_sum<false>(u, r.ctl->red[2], warps);
                var = u[0] * a.inv_d;
            }
            q = rsqrtf(var + a.eps);
        }
        T* n = static_cast<T*>(a.out) + t * a.ld_out;
#pragma unroll
        for (int j = 0; j < kP; ++j)
            if (r.has(j)) {
#pragma unroll
                for (int i = 0; i < kN; ++i) v[j][i] = fma2(mul2(add2(v[j][i], both(-d)), both(q)), w[j][i], b[j][i]);
                r.store(n, j, v[j]);
            }
        if (r.extra >= 0 && r.ok) n[r.extra] = from_f<T>((xc - d) * q * xw + xb);
    }
    if (!r.ok) report_timeout();
}

template <typename T, int kP, bool kWarp>
__global__ void __launch_bounds__(kWarp ? kRowWarps * 32 : ring_threads(true, kP * kVec<T>), kWarp ? warp_ctas(true, kP * kVec<T>) : 1)
    k_layer_norm_back(const __grid_constant__ LnArgs a) {
    constexpr int kN = kPairs<T>, kIn = 3;
    extern __shared__ __align__(16) uint8_t smem[];
    const int warps = blockDim.x / 32;
    const size_t t0 = kWarp ? (size_t)blockIdx.x * kRowWarps + threadIdx.x / 32 : blockIdx.x, G = kWarp ? (size_t)gridDim.x * kRowWarps : gridDim.x;
    Ring<T, kIn, kP, kWarp> r;
    r.in[0] = static_cast<const T*>(a.x); r.ld[0] = a.ld_x;
    r.in[1] = static_cast<const T*>(a.dn); r.ld[1] = a.ld_dn;
    r.in[2] = static_cast<const T*>(a.skip); r.ld[2] = a.ld_skip;
    const bool has_skip = a.skip != nullptr;
    r.begin(smem, a.T, a.D, a.stages, a.row_bytes, r.in[0] + t0 * a.ld_x);
    pdl_wait();
    pdl_trigger();
    if (kWarp || threadIdx.x == 0)
        for (int i = 0; i < r.stages; ++i) r.load(i, t0 + i * G);
    float nx[kIn] = {};
    r.load_extra(t0, nx);
    float2 w[kP][kN], c_w[kP][kN], c_b[kP][kN];
    const float xw = r.weights(a.w, nullptr, w);
    float x_w = 0.f, x_b = 0.f;
#pragma unroll
    for (int j = 0; j < kP; ++j)
#pragma unroll
        for (int i = 0; i < kN; ++i) c_w[j][i] = c_b[j][i] = both(0.f);

    int k = 0;
    for (size_t t = t0; t < a.T; t += G, ++k, r.next()) {
        float ex[kIn];
#pragma unroll
        for (int i = 0; i < kIn; ++i) ex[i] = nx[i];
        r.load_extra(t + G, nx);
        r.wait();
        float2 c[kP][kN], q2[4] = {both(0.f), both(0.f), both(0.f), both(0.f)};   // x - pivot; sums of c, c^2, a, a c
        float pivot = 0.f;
        if (kWarp) {                                             // the mean itself
            float2 s2 = both(0.f);
#pragma unroll
            for (int j = 0; j < kP; ++j)
                if (r.has(j)) {
                    r.piece(0, j, c[j]);
#pragma unroll
                    for (int i = 0; i < kN; ++i) s2 = add2(s2, c[j][i]);
                }
            float m[1] = {sum2(s2) + (r.extra >= 0 ? ex[0] : 0.f)};
            row_sum<true>(m, nullptr, 1);
            pivot = m[0] * a.inv_d;
        } else {
            pivot = pivot_of(r);
        }
#pragma unroll
        for (int j = 0; j < kP; ++j)
            if (r.has(j)) {
                float2 d[kN];
                if (!kWarp) r.piece(0, j, c[j]);
                r.piece(1, j, d);
#pragma unroll
                for (int i = 0; i < kN; ++i) {
                    c[j][i] = add2(c[j][i], both(-pivot));
                    c_b[j][i] = add2(c_b[j][i], d[i]);
                    d[i] = mul2(d[i], w[j][i]);
                    if (!kWarp) q2[0] = add2(q2[0], c[j][i]);
                    q2[1] = fma2(c[j][i], c[j][i], q2[1]);
                    q2[2] = add2(q2[2], d[i]);
                    q2[3] = fma2(d[i], c[j][i], q2[3]);
                }
            }
        float s[4] = {sum2(q2[0]), sum2(q2[1]), sum2(q2[2]), sum2(q2[3])};
        const float xc = ex[0] - pivot, xa = ex[1] * xw;
        if (r.extra >= 0) {
            if (!kWarp) s[0] += xc;
            s[1] += xc * xc;
            s[2] += xa;
            s[3] += xa * xc;
        }
        row_sum<kWarp>(s, r.ctl->red[k & 1], warps);
        const float d0 = kWarp ? 0.f : s[0] * a.inv_d;           // mean - pivot
        float var = var_of(s[1] * a.inv_d, d0), inner = s[3] - d0 * s[2];
        if (!kWarp && far_off(d0, var)) {                        // the same for all threads
            float2 u2[2] = {both(0.f), both(0.f)};
#pragma unroll
            for (int j = 0; j < kP; ++j)
                if (r.has(j)) {
                    float2 d[kN];
                    r.piece(1, j, d);
#pragma unroll
                    for (int i = 0; i < kN; ++i) {
                        const float2 e = add2(c[j][i], both(-d0));
                        u2[0] = fma2(e, e, u2[0]);
                        u2[1] = fma2(mul2(d[i], w[j][i]), e, u2[1]);
                    }
                }
            float u[2] = {sum2(u2[0]), sum2(u2[1])};
            if (r.extra >= 0) {
                u[0] += (xc - d0) * (xc - d0);
                u[1] += xa * (xc - d0);
            }
            row_sum<kWarp>(u, r.ctl->red[2], warps);
            var = u[0] * a.inv_d;
            inner = u[1];
        }
        const float q = rsqrtf(var + a.eps);
        const float along = -q * q * q * inner * a.inv_d;
        const float level = -q * s[2] * a.inv_d - d0 * along;    // dx = q a + (x - pivot) along + level
        T* dx = static_cast<T*>(a.out) + t * a.ld_out;
#pragma unroll
        for (int j = 0; j < kP; ++j)
            if (r.has(j)) {
                float2 d[kN], o[kN];
                r.piece(1, j, d);
                if (has_skip) r.piece(2, j, o);
#pragma unroll
                for (int i = 0; i < kN; ++i) {
                    c_w[j][i] = fma2(mul2(d[i], both(q)), add2(c[j][i], both(-d0)), c_w[j][i]);
                    d[i] = fma2(mul2(d[i], w[j][i]), both(q), fma2(c[j][i], both(along), both(level)));
                    if (has_skip) d[i] = add2(d[i], o[i]);
                }
                r.store(dx, j, d);
            }
        r.release(t, G, warps);
        if (r.extra >= 0) {
            x_w += ex[1] * q * (xc - d0);
            x_b += ex[1];
            if (r.ok) dx[r.extra] = from_f<T>(xa * q + (xc * along + level) + ex[2]);
        }
    }
    float* const part = a.part + blockIdx.x * 2 * part_width(a.D);
    float* const col = kWarp ? reinterpret_cast<float*>(r.base) : part;      // a warp's sums go over its row images, 8 bytes a column
    if (kWarp) {
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncwarp();
    }
    if (r.without(part, 2 * (int)part_width(a.D))) return;
#pragma unroll
    for (int j = 0; j < kP; ++j)
        if (r.has(j))
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                float* p = col + r.column(j) + 2 * i;
                p[0] = c_w[j][i].x;
                p[1] = c_w[j][i].y;
                p[part_width(a.D)] = c_b[j][i].x;
                p[part_width(a.D) + 1] = c_b[j][i].y;
            }
    if (r.extra >= 0) {
        col[r.extra] = x_w;
        col[part_width(a.D) + r.extra] = x_b;
    }
    if (kWarp) {
        __syncthreads();
        const size_t next = (size_t)r.stages * kIn * r.row_bytes / 4;
        const float* first = reinterpret_cast<const float*>(smem + kRingCtl);
        for (int c = threadIdx.x; c < 2 * (int)part_width(a.D); c += kRowWarps * 32) {
            float v = 0.f;
#pragma unroll
            for (int i = 0; i < kRowWarps; ++i) v += first[i * next + c];
            part[c] = v;
        }
    }
}

// How a call is launched.  ring: all matrices aligned alike and the row within the pieces that a CTA's threads own.
struct Plan {
    bool ring, warp;                 // warp: a warp per row
    int threads, elems;              // of a CTA; elements that a thread owns
    int grid, stages;
    int parts;                       // rows of partial column sums
    uint32_t row_bytes;
    size_t smem;
};
bool ring_shape(size_t es, size_t D, bool back, int* threads, int* elems) {
    *elems = ring_elems(back, es, D);
    const size_t need = (D + *elems - 1) / *elems;
    *threads = (int)(need <= 32 ? 32 : (need + 31) / 32 * 32);
    return *threads <= ring_threads(back, *elems);
}
int ring_ctas(bool back, int threads, int elems) {
    const int n = ring_threads(back, elems) / threads;
    return n < kRingCtasMax ? n : kRingCtasMax;
}
template <int N>
Plan plan_of(const Mat (&m)[N], size_t es, uint64_t T, uint64_t D, bool back) {
    Plan p{};
    size_t period = 1;
    p.ring = ring_shape(es, D, back, &p.threads, &p.elems) && aligned_alike(m, es, &period);
    p.row_bytes = (uint32_t)((D * es + 15) / 16 * 16);
    p.warp = D <= warp_row(es);
    if (p.warp) p.threads = kRowWarps * 32;
    const size_t images = back ? 3 : 1, row = images * p.row_bytes * (p.warp ? kRowWarps : 1);
    size_t ctas = 1;
    if (p.ring) {      // as many CTAs as the registers allow, fewer where two rows would not fit; then as many rows as fit
        ctas = (size_t)(p.warp ? warp_ctas(back, p.elems) : ring_ctas(back, p.threads, p.elems));
        while (ctas > 1 && kRingCtl + 2 * row > kRingSmem / ctas) --ctas;
        const size_t room = ctas > 1 ? kRingSmem / ctas : kSmemMax, most = p.warp ? 4 : kRingMax;
        const size_t fit = (room - kRingCtl) / row;
        p.ring = fit >= (p.warp ? 2 : 1);
        p.stages = (int)(fit < most ? fit : most);
        p.smem = kRingCtl + p.stages * row;
    }
    if (!p.ring) {
        p.grid = (int)std::min<uint64_t>(T, kSms * 8);
        if (back) {        // four CTAs an SM for the columns
            const uint64_t blocks = (D + 255) / 256, parts = std::max<uint64_t>(1, 4 * kSms / blocks);
            p.parts = (int)std::min(std::min<uint64_t>(parts, kColumnParts), (T + 7) / 8);
        }
        return p;
    }
    if (p.warp) {
        const uint64_t want = (T + kRowWarps - 1) / kRowWarps, all = (uint64_t)kSms * ctas;
        p.parts = p.grid = (int)(want < all ? want : all);
        return p;
    }
    if (back)          // at least two rows per CTA, whose column sums cost as much as a row
        while (ctas > 1 && kSms * ctas * 2 > T) --ctas;
    const size_t all = (size_t)kSms * ctas / period * period;       // a multiple of the period: rows of a CTA are cut alike
    const size_t want = (T + period - 1) / period * period;
    p.parts = p.grid = (int)(want < all ? want : all);
    return p;
}

template <typename T, int kE, bool kWarp>
cudaError_t run_ring(LnArgs a, bool back, const Plan& p, cudaStream_t s) {
    constexpr int kP = kE / kVec<T>;
    a.stages = p.stages;
    a.row_bytes = p.row_bytes;
    const cudaError_t e = back ? allow_smem<k_layer_norm_back<T, kP, kWarp>>() : allow_smem<k_layer_norm<T, kP, kWarp>>();
    if (e != cudaSuccess) return e;
    return launch_kernel(back ? k_layer_norm_back<T, kP, kWarp> : k_layer_norm<T, kP, kWarp>, p.grid, p.threads, p.smem, s, true, a);
}
template <typename T, int kV>
cudaError_t run_plain(const LnArgs& a, bool back, const Plan& p, cudaStream_t s) {
    if (!back) return launch_kernel(k_layer_norm_plain<T, kV>, p.grid, 256, 0, s, true, a);
    cudaError_t e = launch_kernel(k_layer_norm_stats<T, kV>, p.grid, 256, 0, s, true, a);
    if (e == cudaSuccess) e = launch_kernel(k_layer_norm_columns<T>, dim3((unsigned)((a.D + 255) / 256), p.parts), 256, 0, s, true, a);
    return e != cudaSuccess ? e : launch_kernel(k_layer_norm_back_plain<T, kV>, p.grid, 256, 0, s, true, a);
}
template <typename T>
cudaError_t run(const LnArgs& a, bool back, bool wide, const Plan& p, cudaStream_t s) {
    if (!p.ring) return wide ? run_plain<T, kVec<T>>(a, back, p, s) : run_plain<T, 1>(a, back, p, s);
    if (p.warp && p.elems == 8) return run_ring<T, 8, true>(a, back, p, s);
    if constexpr (warp_row(sizeof(T)) > 256)
        if (p.warp) return run_ring<T, 16, true>(a, back, p, s);
    return p.elems == 16 ? run_ring<T, 16, false>(a, back, p, s) : run_ring<T, 32, false>(a, back, p, s);
}

const char* check_common(uint32_t dtype, uint64_t width, const float* w, const float* b, float eps) {
    if (!known_dtype(dtype)) return "dtype must be ABS_F32 or ABS_BF16";
    if (width == 0) return "width must be at least 1";
    if (!w) return "w must not be NULL";
    if (misaligned(w, 4) || misaligned(b, 4)) return "a weight is not 4-byte aligned";
    if (!(eps > 0.f) || !isfinite(eps)) return "eps must be positive";
    return nullptr;
}

}  // namespace

cudaError_t take_status_layer_norm(int* status, cudaStream_t s) { return take_status(status, s); }

}  // namespace abs_sgd

using namespace abs_sgd;

extern "C" int abs_layer_norm(const void* x, uint64_t ld_x, const float* w, const float* b, float eps, uint32_t dtype, uint64_t tokens, uint64_t width, void* n,
                              uint64_t ld_n, void* stream) {
    if (const char* why = check_common(dtype, width, w, b, eps)) return thread_error(ABS_EINVAL, why);
    if (width > kWidthMax) return thread_error(ABS_ELIMIT, "width exceeds 32768");
    const size_t es = size_of(dtype);
    const MatrixArg q[2] = {{x, ld_x, width, es}, {n, ld_n, width, es}};
    if (const char* why = check_matrices(q)) return thread_error(ABS_EINVAL, why);
    if (const char* why = check_in_place(q[1], q[0], true)) return thread_error(ABS_EINVAL, why);
    if (tokens == 0) return ABS_OK;
    if (!x || !n) return thread_error(ABS_EINVAL, "x and n must not be NULL");
    const Mat m[2] = {{x, ld_x}, {n, ld_n}};
    LnArgs a{};
    a.x = x; a.ld_x = ld_x; a.w = w; a.b = b; a.eps = eps; a.inv_d = 1.f / (float)width; a.T = tokens; a.D = (int)width; a.out = n; a.ld_out = ld_n;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const Plan p = plan_of(m, es, tokens, width, false);
    const bool wide = rows_aligned(m, es, width);
    const cudaError_t e = dtype == ABS_F32 ? run<float>(a, false, wide, p, s) : run<bf16>(a, false, wide, p, s);
    return e == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(e));
}

// Partial column sums; behind them the rows' mean and r.
static size_t part_bytes(uint64_t tokens, uint64_t width) {
    uint64_t most = kColumnParts;
    for (size_t es : {2, 4}) {           // of either type
        int threads = 0, elems = 0;
        const uint64_t ring = ring_shape(es, width, true, &threads, &elems) ? (uint64_t)kSms * ring_ctas(true, threads, elems) : 0;
        if (ring > most) most = ring;
    }
    const uint64_t rows = (tokens + 7) / 8 * 8;
    return ((size_t)(rows < most ? rows : most) * 2 * part_width(width) * 4 + 255) / 256 * 256 + 256;
}
extern "C" size_t abs_layer_norm_workspace(uint64_t tokens, uint64_t width) { return part_bytes(tokens, width) + up256(tokens * sizeof(float2)); }

extern "C" int abs_layer_norm_backward(const void* dn, uint64_t ld_dn, const void* x, uint64_t ld_x, const void* dskip, uint64_t ld_dskip, const float* w, float eps,
                                       uint32_t dtype, uint64_t tokens, uint64_t width, void* dx, uint64_t ld_dx, float* dw, float* db, int accumulate,
                                       void* workspace, size_t workspace_bytes, void* stream) {
    if (const char* why = check_common(dtype, width, w, nullptr, eps)) return thread_error(ABS_EINVAL, why);
    if (width > kWidthMax) return thread_error(ABS_ELIMIT, "width exceeds 32768");
    const size_t es = size_of(dtype);
    const MatrixArg q[4] = {{dn, ld_dn, width, es}, {x, ld_x, width, es}, {dskip, ld_dskip, width, es}, {dx, ld_dx, width, es}};
    if (const char* why = check_matrices(q)) return thread_error(ABS_EINVAL, why);
    for (int i = 0; i < 3; ++i)
        if (const char* why = check_in_place(q[3], q[i], true)) return thread_error(ABS_EINVAL, why);
    if (!dw || misaligned(dw, 4) || misaligned(db, 4)) return thread_error(ABS_EINVAL, "dw must not be NULL, dw and db 4-byte aligned");
    if (dw == db) return thread_error(ABS_EINVAL, "two outputs are the same");
    if (tokens && (!dn || !x || !dx)) return thread_error(ABS_EINVAL, "dn, x and dx must not be NULL");
    if (!workspace || misaligned(workspace, 256)) return thread_error(ABS_EINVAL, "workspace must be non-NULL and 256-byte aligned");
    if (workspace_bytes < abs_layer_norm_workspace(tokens, width)) return thread_error(ABS_ENOMEM, "workspace too small");
    LnArgs a{};
    a.x = x; a.ld_x = ld_x; a.dn = dn; a.ld_dn = ld_dn; a.skip = dskip; a.ld_skip = ld_dskip; a.w = w; a.eps = eps; a.inv_d = 1.f / (float)width;
    a.T = tokens; a.D = (int)width; a.out = dx; a.ld_out = ld_dx; a.part = static_cast<float*>(workspace);
    a.stats = reinterpret_cast<float2*>(static_cast<char*>(workspace) + part_bytes(tokens, width));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaSuccess;
    Plan p{};
    if (tokens > 0) {
        const Mat m[4] = {{dn, ld_dn}, {x, ld_x}, {dskip, ld_dskip}, {dx, ld_dx}};
        p = plan_of(m, es, tokens, width, true);
        const bool wide = rows_aligned(m, es, width);
        e = dtype == ABS_F32 ? run<float>(a, true, wide, p, s) : run<bf16>(a, true, wide, p, s);
    }
    if (e == cudaSuccess) e = launch_column_sums(a.part, p.parts, (int)width, dw, db, accumulate, s);
    return e == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(e));
}
