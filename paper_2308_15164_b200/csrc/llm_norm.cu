// Residual join of a transformer block with its two norms and its gate, forward and backward (abs_residual_norm*).
//
//     u = h / rms(h) * w_post      y = scale x + G u      n = y / rms(y) * w_pre
// Backward with hn = h / rms(h), yn = y / rms(y): a channel gate g and w_post share one column sum, since
// dgate = w_post sum_t dY hn and dw_post = g sum_t dY hn.
// One row of the activations at a time: the two means make a row's work a chain of two reductions, and everything between
// them is elementwise.  Bound by memory: forward 4 (5 with an element gate) and backward 6 (8) elements per position.
#include <math.h>

#include "abs_internal.h"
#include "abs_llm.h"
#include "llm_status.cuh"
#include "row_ring.cuh"

namespace abs_sgd {
namespace {

constexpr int kWidthMax = 32768;
constexpr int kSms = 148;
constexpr int kBackCtas = 296;       // CTAs of the plain backward kernel
constexpr int kRingCtasMax = 16;
// Threads of an SM for the ring kernels, by the elements that a thread owns: what their registers (weights, column sums,
// the row's values) leave room for.
constexpr int ring_threads(bool back, int elems) { return back && elems == 32 ? 256 : 512; }
// Rows that one warp owns: CTAs of eight warps, each with rows of its own, copied by the lanes.  Bulk copies of short rows are bound by
// their number (some 35 ns each on an SM).  us with a warp per row / a CTA of one warp per row, forward and backward, bf16: 60000 x 100 with an
// element gate 33 / 44, 55 / 86; 32768 x 256 18 / 21, 34 / 47; 30000 x 300 22 / 29, 42 / 53; 20000 x 384 17 / 16, 30 / 36; 30000 x 512 34 / 29,
// 68 / 56.  fp32, 20000 x 320: 20 / 18, 36 / 33.  warp_ctas: how many CTAs an SM has registers for.
constexpr size_t warp_row(size_t es) { return es == 2 ? 384 : 256; }
constexpr int warp_ctas(bool back, int elems) { return back ? 2 : elems == 8 ? 4 : 3; }
// Elements of a thread.  Forward, 4096 columns, bf16, 16384 rows: 92 us with 16 (two CTAs of 256 threads an SM), 101 with 32
// (three of 128), 109 with 8 (two of 512).  Backward: 16 leave four warps a scheduler, 32 spread a row's fixed work further and pay
// where they fill two CTAs of 128 threads, or rows that are wide enough.  8192 rows of bf16, us with 16 / 32 by the gate (none without w_post,
// the others with it):
//     columns      2560       3584       3840       4096       4608       5120       6144       7168       8192
//     none       47 / 60    62 / 64    68 / 65    75 / 69    90 / 114   92 / 118   97 / 118  111 / 118  144 / 130
//     channel    65 / 79    88 / 84    89 / 86    94 / 91   142 / 151  145 / 157  150 / 160  175 / 162  180 / 170
//     element    72 / 97   105 / 105  104 / 104  109 / 109  170 / 192  179 / 202  183 / 202  218 / 207  217 / 211
// (beyond 4096 columns one CTA fills an SM).  4096 rows of fp32, channel / element gate, 16 / 32: 4096 columns 73 / 86, 93 / 111; 5120 columns
// 86 / 97, 110 / 124; 8192 columns 155 / 157, 192 / 192.  Up to 256 columns: what a warp has to own.
constexpr int ring_elems(bool back, size_t es, size_t D) {
    if (D <= 8 * 32) return 8;
    if (!back || es == 4) return D <= 16 * 512 ? 16 : 32;
    return D <= 3840 || (D > 4096 && D <= 6144) ? 16 : 32;
}
constexpr int ctas_per_sm(bool back, int threads, int elems) {
    const int n = ring_threads(back, elems) / threads;
    return n < kRingCtasMax ? n : kRingCtasMax;
}

struct NormArgs {
    const void *x, *h, *gate;        // backward: x is unused
    size_t ld_x, ld_h, ld_gate;
    const float *w_post, *w_pre;
    float scale, eps, inv_d;
    size_t T;
    int D;
    void *y, *n;                     // forward: out; backward: y is read
    size_t ld_y, ld_n;
    const void *dn, *dy;
    size_t ld_dn, ld_dy;
    void *dx, *dh, *dgate;           // dgate: element gate only
    size_t ld_dx, ld_dh, ld_dgate;
    float* part;                     // [CTA][2][part_width(D)]: sum dn yn; sum dY hn (channel gate) or dU hn
};

// 1 / (1 + 2^(-v log2 e)).  Relative error below 4e-7 for |v| < 8 (the exponent is rounded once), 0 and 1 in the limits.  The
// gradient's factor 1 - sigmoid is a difference and has an error of that size beside 1, as in any form that keeps the sigmoid alone:
// 1e-3 of itself at v = 8, zero from v = 17 on.  Formed to its own size, 2^(-v log2 e) sigmoid, it costs 3 to 7 % of the backward pass.
__device__ __forceinline__ float sigmoid(float v) {
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(v * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
    return r;
}

// kV consecutive elements at a time, kV = 1 for rows that are not 16-byte aligned; a thread keeps its columns throughout.
template <typename T, int kV, bool kPost, int kGate>
__global__ void __launch_bounds__(256) k_residual_norm(NormArgs a) {
    extern __shared__ float ybuf[];              // the row of y, unrounded
    __shared__ float sh[8];
    pdl_wait();
    pdl_trigger();
    for (size_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + t * a.ld_x;
        const T* h = static_cast<const T*>(a.h) + t * a.ld_h;
        const T* z = static_cast<const T*>(a.gate) + t * a.ld_gate;
        T* y = static_cast<T*>(a.y) + t * a.ld_y;
        T* n = static_cast<T*>(a.n) + t * a.ld_n;
        float rh = 1.f;
        if (kPost) {
            float s[1] = {0.f};
            for (int c = threadIdx.x * kV; c < a.D; c += 256 * kV) {
                float v[kV];
                Pack<T, kV>::load(h + c, v);
#pragma unroll
                for (int k = 0; k < kV; ++k) s[0] += v[k] * v[k];
            }
            group_sum<256, 1>(s, sh);
            rh = 1.f / sqrtf(s[0] * a.inv_d + a.eps);
        }
        float s[1] = {0.f};
        for (int c = threadIdx.x * kV; c < a.D; c += 256 * kV) {
            float u[kV], v[kV], g[kV];
            Pack<T, kV>::load(h + c, u);
            Pack<T, kV>::load(x + c, v);
            if (kGate == 2) Pack<T, kV>::load(z + c, g);
#pragma unroll
            for (int k = 0; k < kV; ++k) {
                if (kPost) u[k] *= rh * a.w_post[c + k];
                if (kGate == 1) u[k] *= static_cast<const float*>(a.gate)[c + k];
                if (kGate == 2) u[k] *= sigmoid(g[k]);
                v[k] = a.scale * v[k] + u[k];
                s[0] += v[k] * v[k];
                ybuf[c + k] = v[k];
            }
            Pack<T, kV>::store(y + c, v);
        }
        group_sum<256, 1>(s, sh);
        const float ry = 1.f / sqrtf(s[0] * a.inv_d + a.eps);
        for (int c = threadIdx.x * kV; c < a.D; c += 256 * kV) {
            float v[kV];
#pragma unroll
            for (int k = 0; k < kV; ++k) v[k] = ybuf[c + k] * (ry * a.w_pre[c + k]);
            Pack<T, kV>::store(n + c, v);
        }
    }
}

template <typename T, int kV, bool kPost, int kGate>
__global__ void __launch_bounds__(256) k_residual_norm_back(NormArgs a) {
    extern __shared__ float dubuf[];             // dU w_post of the row
    __shared__ float sh[24];
    pdl_wait();
    pdl_trigger();
    float *col = a.part + blockIdx.x * 2 * part_width(a.D), *col_h = col + part_width(a.D);
    for (int c = threadIdx.x * kV; c < a.D; c += 256 * kV)
#pragma unroll
        for (int k = 0; k < kV; ++k) col[c + k] = col_h[c + k] = 0.f;
    for (size_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const T* dn = static_cast<const T*>(a.dn) + t * a.ld_dn;
        const T* dy = a.dy ? static_cast<const T*>(a.dy) + t * a.ld_dy : nullptr;
        const T* y = static_cast<const T*>(a.y) + t * a.ld_y;
        const T* h = static_cast<const T*>(a.h) + t * a.ld_h;
        const T* z = static_cast<const T*>(a.gate) + t * a.ld_gate;
        T* dx = static_cast<T*>(a.dx) + t * a.ld_dx;
        T* dh = static_cast<T*>(a.dh) + t * a.ld_dh;
        T* dz = static_cast<T*>(a.dgate) + t * a.ld_dgate;
        float s[3] = {0.f, 0.f, 0.f};            // sum y^2, sum dn w_pre y, sum h^2
        for (int c = threadIdx.x * kV; c < a.D; c += 256 * kV) {
            float vy[kV], vn[kV], vh[kV];
            Pack<T, kV>::load(y + c, vy);
            Pack<T, kV>::load(dn + c, vn);
            if (kPost) Pack<T, kV>::load(h + c, vh);
#pragma unroll
            for (int k = 0; k < kV; ++k) {
                s[0] += vy[k] * vy[k];
                s[1] += vn[k] * a.w_pre[c + k] * vy[k];
                if (kPost) s[2] += vh[k] * vh[k];
            }
        }
        group_sum<256, 3>(s, sh);
        const float ry = 1.f / sqrtf(s[0] * a.inv_d + a.eps);
        const float along = s[1] * a.inv_d * ry;                 // mean(dn w_pre yn)
        const float rh = kPost ? 1.f / sqrtf(s[2] * a.inv_d + a.eps) : 1.f;
        float q[1] = {0.f};                                      // sum dU w_post hn
        for (int c = threadIdx.x * kV; c < a.D; c += 256 * kV) {
            float vy[kV], vn[kV], vh[kV], vd[kV], vg[kV], o[kV];
            Pack<T, kV>::load(y + c, vy);
            Pack<T, kV>::load(dn + c, vn);
            Pack<T, kV>::load(h + c, vh);
            if (dy) Pack<T, kV>::load(dy + c, vd);
            if (kGate == 2) Pack<T, kV>::load(z + c, vg);
#pragma unroll
            for (int k = 0; k < kV; ++k) {
                const float yn = vy[k] * ry;
                const float d = (dy ? vd[k] : 0.f) + ry * (vn[k] * a.w_pre[c + k] - yn * along);
                o[k] = a.scale * d;
                col[c + k] += vn[k] * yn;
                const float hn = vh[k] * rh;
                const float w = kPost ? a.w_post[c + k] : 1.f;
                float du = d;
                if (kGate == 1) {
                    col_h[c + k] += d * hn;
                    du *= static_cast<const float*>(a.gate)[c + k];
                }
                if (kGate == 2) {
                    const float g = sigmoid(vg[k]);
                    du *= g;
                    vg[k] = du * (hn * w) * (1.f - g);
                }
                if (kPost) {
                    if (kGate != 1) col_h[c + k] += du * hn;
                    q[0] += du * w * hn;
                }
                vh[k] = du * w;
                dubuf[c + k] = du * w;
            }
            Pack<T, kV>::store(dx + c, o);
            if (kGate == 2) Pack<T, kV>::store(dz + c, vg);
            if (!kPost) Pack<T, kV>::store(dh + c, vh);
        }
        if (kPost) {
            group_sum<256, 1>(q, sh);
            const float m = q[0] * a.inv_d;
            for (int c = threadIdx.x * kV; c < a.D; c += 256 * kV) {
                float vh[kV];
                Pack<T, kV>::load(h + c, vh);
#pragma unroll
                for (int k = 0; k < kV; ++k) vh[k] = rh * (dubuf[c + k] - vh[k] * rh * m);
                Pack<T, kV>::store(dh + c, vh);
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------
// The same rows through a ring of row images in shared memory.  A CTA takes rows b, b + G, ...; one thread keeps the
// ring's rows of copies in flight (cp.async.bulk, one per input matrix), so that the chain of reductions of a row hides
// behind the copies of the next ones.  A thread owns kP pieces of 16 bytes, up to 32 elements (what a row costs a thread
// beside its elements -- reductions, waits, addresses, some 150 instructions -- is spread over them: with 8 elements the
// kernels were bound by instruction issue at half the memory's rate), and at most one single element.
// Rows of odd width start at every alignment.  G is a multiple of the period with which the alignment repeats, so that
// all rows of one CTA are cut alike: single elements up to the first 16-byte boundary, pieces, single elements.  The
// copies move the pieces (nothing outside the row is read), the single elements are plain loads.  All matrices of the
// call have to be aligned alike.  Short rows: a warp per row, each lane copies the pieces that it reads (kWarp).
// Weights and column sums stay in registers; two fp32 operations per instruction where the order of a sum allows it.
// ------------------------------------------------------------------------------------------------
struct RingArgs {
    NormArgs n;
    int stages;
    uint32_t row_bytes;              // room for one row image, a multiple of 16
};

template <typename T, int kP, bool kPost, int kGate, bool kWarp>
__global__ void __launch_bounds__(kWarp ? kRowWarps * 32 : ring_threads(false, kP * kVec<T>), kWarp ? warp_ctas(false, kP * kVec<T>) : 1) k_join(const __grid_constant__ RingArgs ra) {
    constexpr int kN = kPairs<T>, kIn = kGate == 2 ? 3 : 2;
    constexpr bool kScaled = kPost || kGate == 1;    // u carries a weight: w_post, the channel gate, or their product
    const NormArgs& a = ra.n;
    extern __shared__ __align__(16) uint8_t smem[];
    const int warps = blockDim.x / 32;
    const size_t t0 = kWarp ? (size_t)blockIdx.x * kRowWarps + threadIdx.x / 32 : blockIdx.x, G = kWarp ? (size_t)gridDim.x * kRowWarps : gridDim.x;
    Ring<T, kIn, kP, kWarp> r;
    r.in[0] = static_cast<const T*>(a.x); r.ld[0] = a.ld_x;
    r.in[1] = static_cast<const T*>(a.h); r.ld[1] = a.ld_h;
    if (kGate == 2) { r.in[kIn - 1] = static_cast<const T*>(a.gate); r.ld[kIn - 1] = a.ld_gate; }
    r.begin(smem, a.T, a.D, ra.stages, ra.row_bytes, r.in[0] + t0 * a.ld_x);
    pdl_wait();
    pdl_trigger();
    if (kWarp || threadIdx.x == 0)
        for (int i = 0; i < r.stages; ++i) r.load(i, t0 + i * G);
    float nx[kIn] = {};
    r.load_extra(t0, nx);
    float2 w_u[kP][kN], w_pre[kP][kN];
    const float* gate = kGate == 1 ? static_cast<const float*>(a.gate) : nullptr;
    const float xw_u = kScaled ? r.weights(kPost ? a.w_post : gate, kPost ? gate : nullptr, w_u) : 1.f;
    const float xw_pre = r.weights(a.w_pre, nullptr, w_pre);

    int k = 0;
    for (size_t t = t0; t < a.T; t += G, ++k, r.next()) {
        float (*red)[16] = r.ctl->red[k & 1];
        float ex[kIn];
#pragma unroll
        for (int i = 0; i < kIn; ++i) ex[i] = nx[i];
        r.load_extra(t + G, nx);
        r.wait();
        float rh = 1.f;
        if (kPost) {
            float2 s2 = both(0.f);
#pragma unroll
            for (int j = 0; j < kP; ++j)
                if (r.has(j)) {
                    float2 v[kN];
                    r.piece(1, j, v);
#pragma unroll
                    for (int i = 0; i < kN; ++i) s2 = fma2(v[i], v[i], s2);
                }
            float s[1] = {sum2(s2) + (r.extra >= 0 ? ex[1] * ex[1] : 0.f)};
            row_sum<kWarp>(s, red, warps);
            if (!kWarp) r.refill(t, G, k);
            rh = rsqrtf(s[0] * a.inv_d + a.eps);
        }
        float2 y[kP][kN], s2 = both(0.f);
        T* yrow = static_cast<T*>(a.y) + t * a.ld_y;
#pragma unroll
        for (int j = 0; j < kP; ++j)
            if (r.has(j)) {
                float2 u[kN], g[kN];
                r.piece(0, j, y[j]);
                r.piece(1, j, u);
                if (kGate == 2) r.piece(kIn - 1, j, g);
#pragma unroll
                for (int i = 0; i < kN; ++i) {
                    if (kPost) u[i] = mul2(u[i], both(rh));
                    if (kScaled) u[i] = mul2(u[i], w_u[j][i]);
                    if (kGate == 2) u[i] = mul2(u[i], make_float2(sigmoid(g[i].x), sigmoid(g[i].y)));
                    y[j][i] = fma2(y[j][i], both(a.scale), u[i]);
                    s2 = fma2(y[j][i], y[j][i], s2);
                }
                r.store(yrow, j, y[j]);
            }
        if (kWarp) r.release(t, G, warps);
        float s[1] = {sum2(s2)}, xy = 0.f;
        if (r.extra >= 0) {
            float u = ex[1] * rh * xw_u;
            if (kGate == 2) u *= sigmoid(ex[kIn - 1]);
            xy = a.scale * ex[0] + u;
            s[0] += xy * xy;
            if (r.ok) yrow[r.extra] = from_f<T>(xy);
        }
        row_sum<kWarp>(s, kPost ? r.ctl->red[2] : red, warps);
        if (!kPost && !kWarp) r.refill(t, G, k);
        const float ry = rsqrtf(s[0] * a.inv_d + a.eps);
        T* nrow = static_cast<T*>(a.n) + t * a.ld_n;
#pragma unroll
        for (int j = 0; j < kP; ++j)
            if (r.has(j)) {
#pragma unroll
                for (int i = 0; i < kN; ++i) y[j][i] = mul2(mul2(y[j][i], both(ry)), w_pre[j][i]);
                r.store(nrow, j, y[j]);
            }
        if (r.extra >= 0 && r.ok) nrow[r.extra] = from_f<T>(xy * ry * xw_pre);
    }
    if (!r.ok) report_timeout();
}

template <typename T, int kP, bool kPost, int kGate, bool kWarp>
__global__ void __launch_bounds__(kWarp ? kRowWarps * 32 : ring_threads(true, kP * kVec<T>), kWarp ? warp_ctas(true, kP * kVec<T>) : 1) k_join_back(const __grid_constant__ RingArgs ra) {
    constexpr int kN = kPairs<T>, kIn = kGate == 2 ? 5 : 4;
    constexpr bool kScaled = kPost || kGate == 1;    // dh carries a weight: w_post, the channel gate, or their product
    constexpr bool kSum = kPost || kGate == 1;       // the second column sum
    constexpr int kSums = kPost ? 6 : 2, kH = kPost ? 2 : 0, kE = kPost ? 3 : 0, kY = kPost ? 4 : 0, kDy = kPost ? 5 : 0;
    const NormArgs& a = ra.n;
    extern __shared__ __align__(16) uint8_t smem[];
    const int warps = blockDim.x / 32;
    const size_t t0 = kWarp ? (size_t)blockIdx.x * kRowWarps + threadIdx.x / 32 : blockIdx.x, G = kWarp ? (size_t)gridDim.x * kRowWarps : gridDim.x;
    Ring<T, kIn, kP, kWarp> r;
    r.in[0] = static_cast<const T*>(a.y); r.ld[0] = a.ld_y;
    r.in[1] = static_cast<const T*>(a.dn); r.ld[1] = a.ld_dn;
    r.in[2] = static_cast<const T*>(a.h); r.ld[2] = a.ld_h;
    r.in[3] = static_cast<const T*>(a.dy); r.ld[3] = a.ld_dy;
    if (kGate == 2) { r.in[kIn - 1] = static_cast<const T*>(a.gate); r.ld[kIn - 1] = a.ld_gate; }
    const bool has_dy = a.dy != nullptr;
    r.begin(smem, a.T, a.D, ra.stages, ra.row_bytes, r.in[0] + t0 * a.ld_y);
    pdl_wait();
    pdl_trigger();
    if (kWarp || threadIdx.x == 0)
        for (int i = 0; i < r.stages; ++i) r.load(i, t0 + i * G);
    float nx[kIn] = {};
    r.load_extra(t0, nx);
    float2 w_u[kP][kN], w_pre[kP][kN], c_pre[kP][kN], c_h[kP][kN];
    const float* gate = kGate == 1 ? static_cast<const float*>(a.gate) : nullptr;
    const float xw_u = kScaled ? r.weights(kPost ? a.w_post : gate, kPost ? gate : nullptr, w_u) : 1.f;
    const float xw_pre = r.weights(a.w_pre, nullptr, w_pre);
    float x_pre = 0.f, x_h = 0.f;
#pragma unroll
    for (int j = 0; j < kP; ++j)
#pragma unroll
        for (int i = 0; i < kN; ++i) c_pre[j][i] = c_h[j][i] = both(0.f);

    int k = 0;
    for (size_t t = t0; t < a.T; t += G, ++k, r.next()) {
        float ex[kIn];
#pragma unroll
        for (int i = 0; i < kIn; ++i) ex[i] = nx[i];
        r.load_extra(t + G, nx);
        r.wait();
        // With e = dn w_pre: sums of y^2, e y, and with f = gate w_post h, of h^2, f e, f y, f dy, of which the inner product of
        // dU w_post with h is made when dY's factors are known: one synchronisation per row instead of two.
        float2 s2[kSums];
        float2 sg[kP][kN];                                       // sigmoid of the gate
#pragma unroll
        for (int n = 0; n < kSums; ++n) s2[n] = both(0.f);
#pragma unroll
        for (int j = 0; j < kP; ++j)
            if (r.has(j)) {
                float2 y[kN], e[kN], f[kN];
                r.piece(0, j, y);
                r.piece(1, j, e);
#pragma unroll
                for (int i = 0; i < kN; ++i) {
                    e[i] = mul2(e[i], w_pre[j][i]);
                    s2[0] = fma2(y[i], y[i], s2[0]);
                    s2[1] = fma2(e[i], y[i], s2[1]);
                }
                if (kGate == 2) {
                    r.piece(kIn - 1, j, f);
#pragma unroll
                    for (int i = 0; i < kN; ++i) sg[j][i] = make_float2(sigmoid(f[i].x), sigmoid(f[i].y));
                }
                if (kPost) {
                    r.piece(2, j, f);
#pragma unroll
                    for (int i = 0; i < kN; ++i) {
                        s2[kH] = fma2(f[i], f[i], s2[kH]);
                        f[i] = mul2(f[i], w_u[j][i]);
                        if (kGate == 2) f[i] = mul2(f[i], sg[j][i]);
                        s2[kE] = fma2(f[i], e[i], s2[kE]);
                        s2[kY] = fma2(f[i], y[i], s2[kY]);
                    }
                    if (has_dy) {
                        r.piece(3, j, e);
#pragma unroll
                        for (int i = 0; i < kN; ++i) s2[kDy] = fma2(f[i], e[i], s2[kDy]);
                    }
                }
            }
        float s[kSums];
#pragma unroll
        for (int n = 0; n < kSums; ++n) s[n] = sum2(s2[n]);
        if (r.extra >= 0) {
            const float e = ex[1] * xw_pre;
            s[0] += ex[0] * ex[0];
            s[1] += e * ex[0];
            if (kPost) {
                float f = ex[2] * xw_u;
                if (kGate == 2) f *= sigmoid(ex[kIn - 1]);
                s[kH] += ex[2] * ex[2];
                s[kE] += f * e;
                s[kY] += f * ex[0];
                s[kDy] += f * ex[3];
            }
        }
        row_sum<kWarp>(s, r.ctl->red[k & 1], warps);
        const float ry = rsqrtf(s[0] * a.inv_d + a.eps);
        const float along = -s[1] * a.inv_d * ry * ry;          // d = ry (dn w_pre) + yn along
        const float rh = kPost ? rsqrtf(s[kH] * a.inv_d + a.eps) : 1.f;
        // dh = rh dU w_post + h m, dY = ry e + y ry along + dy
        const float m = kPost ? -(ry * (s[kE] + along * s[kY]) + s[kDy]) * a.inv_d * rh * rh * rh : 0.f;
        T* dx = static_cast<T*>(a.dx) + t * a.ld_dx;
        T* dh = static_cast<T*>(a.dh) + t * a.ld_dh;
        T* dz = static_cast<T*>(a.dgate) + t * a.ld_dgate;
#pragma unroll
        for (int j = 0; j < kP; ++j)
            if (r.has(j)) {
                float2 d[kN], v[kN];
                r.piece(0, j, v);
                r.piece(1, j, d);
#pragma unroll
                for (int i = 0; i < kN; ++i) {
                    v[i] = mul2(v[i], both(ry));                 // yn
                    c_pre[j][i] = fma2(d[i], v[i], c_pre[j][i]);
                    d[i] = fma2(v[i], both(along), mul2(mul2(d[i], w_pre[j][i]), both(ry)));
                }
                if (has_dy) {
                    r.piece(3, j, v);
#pragma unroll
                    for (int i = 0; i < kN; ++i) d[i] = add2(d[i], v[i]);
                }
#pragma unroll
                for (int i = 0; i < kN; ++i) v[i] = mul2(d[i], both(a.scale));
                r.store(dx, j, v);
                r.piece(2, j, v);
                if (kGate == 2) {
                    float2 g[kN];
#pragma unroll
                    for (int i = 0; i < kN; ++i) {
                        d[i] = mul2(d[i], sg[j][i]);
                        const float2 u = mul2(d[i], kPost ? mul2(mul2(v[i], both(rh)), w_u[j][i]) : v[i]);
                        g[i] = fma2(make_float2(-sg[j][i].x, -sg[j][i].y), u, u);       // dU u (1 - g)
                    }
                    r.store(dz, j, g);
                }
#pragma unroll
                for (int i = 0; i < kN; ++i) {
                    if (kPost) d[i] = mul2(d[i], both(rh));
                    if (kSum) c_h[j][i] = fma2(d[i], v[i], c_h[j][i]);
                    if (kScaled) d[i] = mul2(d[i], w_u[j][i]);
                    if (kPost) d[i] = fma2(v[i], both(m), d[i]);
                }
                r.store(dh, j, d);
            }
        r.release(t, G, warps);
        if (r.extra >= 0) {
            const float yn = ex[0] * ry, hn = ex[2] * rh;
            x_pre += ex[1] * yn;
            float d = yn * along + ex[1] * xw_pre * ry;
            d += ex[3];
            const float xdx = a.scale * d;
            float xdz = 0.f;
            if (kGate == 2) {
                const float g = sigmoid(ex[kIn - 1]);
                d *= g;
                xdz = d * (hn * xw_u);
                xdz = xdz - g * xdz;
            }
            x_h += d * hn;
            if (r.ok) {
                dx[r.extra] = from_f<T>(xdx);
                if (kGate == 2) dz[r.extra] = from_f<T>(xdz);
                dh[r.extra] = from_f<T>(kPost ? ex[2] * m + rh * (d * xw_u) : d * xw_u);
            }
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
                float* c = col + r.column(j) + 2 * i;
                c[0] = c_pre[j][i].x;
                c[1] = c_pre[j][i].y;
                if (kSum) {
                    c[part_width(a.D)] = c_h[j][i].x;
                    c[part_width(a.D) + 1] = c_h[j][i].y;
                }
            }
    if (r.extra >= 0) {
        col[r.extra] = x_pre;
        if (kSum) col[part_width(a.D) + r.extra] = x_h;
    }
    if (kWarp) {
        __syncthreads();
        const size_t next = (size_t)r.stages * kIn * r.row_bytes / 4;
        const float* first = reinterpret_cast<const float*>(smem + kRingCtl);
        for (int c = threadIdx.x; c < (kSum ? 2 : 1) * (int)part_width(a.D); c += kRowWarps * 32) {
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < kRowWarps; ++w) v += first[w * next + c];
            part[c] = v;
        }
    }
}

// Column sums over the CTAs of part[cta][which][c], 32 columns per CTA, joined in a fixed order: eight threads with a piece of 16 bytes
// each make a line, 128 lines and four loads of each thread are in flight (few CTAs, latency: 16384 x 1024 bf16, 1184 partial sums, 8.1 us
// with a cold cache, 14.6 with a thread per column).
// which 0: dw_pre; which 1, with S the sum: dw_post = S (times the channel gate), channel dgate = S (times w_post).
__global__ void __launch_bounds__(1024) k_column_sums(const float* part, int n, int D, float* dw_pre, float* dw_post, float* dgate, const float* w_post,
                                                      const float* gate, int accumulate) {
    __shared__ __align__(16) float sh[128][36];
    pdl_wait();
    pdl_trigger();
    const int piece = threadIdx.x % 8, line = threadIdx.x / 8;
    const size_t width = part_width(D), c = (size_t)blockIdx.x * 32 + piece * 4;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < width) {
        const float* p = part + blockIdx.y * width + c;
        for (int i = line; i < n; i += 4 * 128) {
            float4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                v[k] = i + 128 * k < n ? *reinterpret_cast<const float4*>(p + (size_t)(i + 128 * k) * 2 * width) : make_float4(0.f, 0.f, 0.f, 0.f);
            sum.x += (v[0].x + v[1].x) + (v[2].x + v[3].x);
            sum.y += (v[0].y + v[1].y) + (v[2].y + v[3].y);
            sum.z += (v[0].z + v[1].z) + (v[2].z + v[3].z);
            sum.w += (v[0].w + v[1].w) + (v[2].w + v[3].w);
        }
    }
    *reinterpret_cast<float4*>(&sh[line][piece * 4]) = sum;
    __syncthreads();
    const int lane = threadIdx.x % 32, r = threadIdx.x / 32;       // a warp per column
    float s = (sh[lane][r] + sh[lane + 32][r]) + (sh[lane + 64][r] + sh[lane + 96][r]);
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    const int cc = blockIdx.x * 32 + r;
    if (cc >= D) return;
    if (s != s) {                                                  // a partial sum that its kernel could not form: nothing is written
        bool missing = false;
        for (int i = lane; i < n; i += 32) missing = missing || unformed(part[(size_t)i * 2 * width + blockIdx.y * width + cc]);
        if (__any_sync(0xffffffffu, missing)) return;
    }
    if (lane != 0) return;
    auto put = [&](float* out, float v) { out[cc] = accumulate ? out[cc] + v : v; };
    if (blockIdx.y == 0) put(dw_pre, s);
    else {
        if (dw_post) put(dw_post, gate ? gate[cc] * s : s);
        if (dgate) put(dgate, w_post ? w_post[cc] * s : s);
    }
}

// How a call is launched.  ring: all matrices aligned alike and the row within the pieces that a CTA's threads own.
struct Plan {
    bool ring, warp;                 // warp: a warp per row
    int threads, elems;              // of a CTA; elements that a thread owns
    int grid, stages;
    uint32_t row_bytes;
    size_t smem;
};

template <typename T, int kV, bool kPost, int kGate>
cudaError_t run_plain(const NormArgs& a, bool back, int grid, cudaStream_t s) {
    const size_t smem = (size_t)a.D * 4;
    const cudaError_t e = back ? allow_smem<k_residual_norm_back<T, kV, kPost, kGate>>() : allow_smem<k_residual_norm<T, kV, kPost, kGate>>();
    if (e != cudaSuccess) return e;
    return launch_kernel(back ? k_residual_norm_back<T, kV, kPost, kGate> : k_residual_norm<T, kV, kPost, kGate>, grid, 256, smem, s, true, a);
}
template <typename T, int kE, bool kPost, int kGate, bool kWarp>
cudaError_t run_ring(const NormArgs& a, bool back, const Plan& p, cudaStream_t s) {
    constexpr int kP = kE / kVec<T>;
    const RingArgs r{a, p.stages, p.row_bytes};
    const cudaError_t e = back ? allow_smem<k_join_back<T, kP, kPost, kGate, kWarp>>() : allow_smem<k_join<T, kP, kPost, kGate, kWarp>>();
    if (e != cudaSuccess) return e;
    return launch_kernel(back ? k_join_back<T, kP, kPost, kGate, kWarp> : k_join<T, kP, kPost, kGate, kWarp>, p.grid, p.threads, p.smem, s, true, r);
}
template <typename T, bool kPost, int kGate>
cudaError_t run(const NormArgs& a, bool back, bool wide, const Plan& p, cudaStream_t s) {
    if (!p.ring) return wide ? run_plain<T, kVec<T>, kPost, kGate>(a, back, p.grid, s) : run_plain<T, 1, kPost, kGate>(a, back, p.grid, s);
    if (p.warp && p.elems == 8) return run_ring<T, 8, kPost, kGate, true>(a, back, p, s);
    if constexpr (warp_row(sizeof(T)) > 256)
        if (p.warp) return run_ring<T, 16, kPost, kGate, true>(a, back, p, s);
    return p.elems == 16 ? run_ring<T, 16, kPost, kGate, false>(a, back, p, s) : run_ring<T, 32, kPost, kGate, false>(a, back, p, s);
}
template <typename T>
cudaError_t run_kind(const NormArgs& a, bool back, uint32_t gate, bool wide, const Plan& p, cudaStream_t s) {
    if (a.w_post)
        return gate == 0 ? run<T, true, 0>(a, back, wide, p, s) : gate == 1 ? run<T, true, 1>(a, back, wide, p, s) : run<T, true, 2>(a, back, wide, p, s);
    return gate == 0 ? run<T, false, 0>(a, back, wide, p, s) : gate == 1 ? run<T, false, 1>(a, back, wide, p, s) : run<T, false, 2>(a, back, wide, p, s);
}

// Elements that a thread owns and threads of a CTA for rows of `D` elements of `es` bytes; false: more than a CTA can own.
bool ring_shape(size_t es, size_t D, bool back, int* threads, int* elems) {
    *elems = ring_elems(back, es, D);
    const size_t need = (D + *elems - 1) / *elems;
    *threads = (int)(need <= 32 ? 32 : (need + 31) / 32 * 32);
    return *threads <= ring_threads(back, *elems);
}
template <int N>
Plan plan_of(const Mat (&m)[N], size_t es, uint64_t T, uint64_t D, bool back, uint32_t gate_kind) {
    Plan p{};
    size_t period = 1;
    p.ring = ring_shape(es, D, back, &p.threads, &p.elems) && aligned_alike(m, es, &period);
    p.row_bytes = (uint32_t)((D * es + 15) / 16 * 16);
    p.warp = D <= warp_row(es);
    if (p.warp) p.threads = kRowWarps * 32;
    const size_t images = (back ? 4 : 2) + (gate_kind == ABS_GATE_ELEMENT ? 1 : 0), row = images * p.row_bytes * (p.warp ? kRowWarps : 1);
    size_t ctas = 1;
    if (p.ring) {      // as many CTAs as the registers allow, fewer where two rows would not fit; then as many rows as fit
        ctas = (size_t)(p.warp ? warp_ctas(back, p.elems) : ctas_per_sm(back, p.threads, p.elems));
        while (ctas > 1 && kRingCtl + 2 * row > kRingSmem / ctas) --ctas;
        const size_t room = ctas > 1 ? kRingSmem / ctas : kSmemMax, most = p.warp ? 4 : kRingMax;
        const size_t fit = (room - kRingCtl) / row;
        p.ring = fit >= (back ? 1 : 2);
        p.stages = (int)(fit < most ? fit : most);
        p.smem = kRingCtl + p.stages * row;
    }
    if (!p.ring) {
        const uint64_t cap = back ? kBackCtas : kSms * 8;
        p.grid = (int)(T < cap ? T : cap);
        return p;
    }
    if (p.warp) {
        const uint64_t want = (T + kRowWarps - 1) / kRowWarps, all = (uint64_t)kSms * ctas;
        p.grid = (int)(want < all ? want : all);
        return p;
    }
    // backward: at least two rows per CTA, whose column sums cost as much as a row (1003 x 1537 fp32: 16.4 us, with four 19.4)
    if (back)
        while (ctas > 1 && kSms * ctas * 2 > T) --ctas;
    const size_t all = (size_t)kSms * ctas / period * period;       // a multiple of the period: rows of a CTA are cut alike
    const size_t want = (T + period - 1) / period * period;
    p.grid = (int)(want < all ? want : all);
    return p;
}
template <int N>
const char* check_mats(const Mat (&m)[N], size_t es, size_t D) {
    for (const Mat& q : m) {
        if (misaligned(q.p, es)) return "a pointer is not aligned to its elements";
        if (q.p && q.ld < D) return "a leading dimension is shorter than the row";
    }
    return nullptr;
}
// An output in place of an input has to have its leading dimension.
const char* check_in_place(Mat out, Mat in) { return out.p && out.p == in.p && out.ld != in.ld ? "an output in place of an input needs the same leading dimension" : nullptr; }
// Outputs have to be different ones.
template <int N>
const char* check_apart(const void* const (&out)[N]) {
    for (int i = 0; i < N; ++i)
        for (int j = 0; j < i; ++j)
            if (out[i] && out[i] == out[j]) return "two outputs are the same";
    return nullptr;
}
const char* check_common(uint32_t dtype, uint64_t width, uint32_t gate_kind, const void* gate, const float* w_post, const float* w_pre,
                         float scale, float eps) {
    if (dtype != ABS_F32 && dtype != ABS_BF16) return "dtype must be ABS_F32 or ABS_BF16";
    if (width == 0) return "width must be at least 1";
    if (gate_kind > ABS_GATE_ELEMENT) return "unknown gate kind";
    if ((gate_kind != ABS_GATE_NONE) != (gate != nullptr)) return "a gate must be given exactly when the gate kind asks for one";
    if (gate_kind == ABS_GATE_CHANNEL && misaligned(gate, 4)) return "a channel gate is fp32, 4-byte aligned";
    if (!w_pre) return "w_pre must not be NULL";
    if (misaligned(w_pre, 4) || misaligned(w_post, 4)) return "a weight is not 4-byte aligned";
    if (!isfinite(scale) || !(eps > 0.f) || !isfinite(eps)) return "scale must be finite, eps positive";
    return nullptr;
}

}  // namespace
}  // namespace abs_sgd

namespace abs_sgd {
cudaError_t take_status_norm(int* status, cudaStream_t s) { return take_status(status, s); }
cudaError_t launch_column_sums(const float* part, int n, int D, float* first, float* second, int accumulate, cudaStream_t s) {
    return launch_kernel(k_column_sums, dim3((unsigned)((D + 31) / 32), second ? 2 : 1), 1024, 0, s, true, part, n, D, first, second, (float*)nullptr,
                         (const float*)nullptr, (const float*)nullptr, accumulate);
}
}  // namespace abs_sgd

using namespace abs_sgd;

extern "C" int abs_residual_norm(const void* x, uint64_t ld_x, const void* h, uint64_t ld_h, const void* gate, uint64_t ld_gate,
                                 uint32_t gate_kind, const float* w_post, const float* w_pre, float scale, float eps, uint32_t dtype,
                                 uint64_t tokens, uint64_t width, void* y, uint64_t ld_y, void* n, uint64_t ld_n, void* stream) {
    if (const char* why = check_common(dtype, width, gate_kind, gate, w_post, w_pre, scale, eps)) return thread_error(ABS_EINVAL, why);
    if (width > kWidthMax) return thread_error(ABS_ELIMIT, "width exceeds 32768");
    const size_t es = dtype == ABS_F32 ? 4 : 2;
    const Mat m[5] = {{x, ld_x}, {h, ld_h}, {gate_kind == ABS_GATE_ELEMENT ? gate : nullptr, ld_gate}, {y, ld_y}, {n, ld_n}};
    if (const char* why = check_mats(m, es, width)) return thread_error(ABS_EINVAL, why);
    for (const Mat& out : {m[3], m[4]})
        for (const Mat& in : {m[0], m[1], m[2]})
            if (const char* why = check_in_place(out, in)) return thread_error(ABS_EINVAL, why);
    if (tokens == 0) return ABS_OK;
    if (!x || !h || !y || !n) return thread_error(ABS_EINVAL, "x, h, y and n must not be NULL");
    if (const char* why = check_apart({y, n})) return thread_error(ABS_EINVAL, why);
    NormArgs a{};
    a.x = x; a.ld_x = ld_x; a.h = h; a.ld_h = ld_h; a.gate = gate; a.ld_gate = ld_gate;
    a.w_post = w_post; a.w_pre = w_pre; a.scale = scale; a.eps = eps; a.inv_d = 1.f / (float)width; a.T = tokens; a.D = (int)width;
    a.y = y; a.ld_y = ld_y; a.n = n; a.ld_n = ld_n;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool wide = rows_aligned(m, es, width);
    const Plan p = plan_of(m, es, tokens, width, false, gate_kind);
    const cudaError_t e = dtype == ABS_F32 ? run_kind<float>(a, false, gate_kind, wide, p, s) : run_kind<bf16>(a, false, gate_kind, wide, p, s);
    return e == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(e));
}

extern "C" size_t abs_residual_norm_workspace(uint64_t tokens, uint64_t width) {
    uint64_t most = kBackCtas;       // of either type
    for (size_t es : {2, 4}) {
        int threads = 0, elems = 0;
        const uint64_t ring = width > warp_row(es) && ring_shape(es, width, true, &threads, &elems) ? (uint64_t)kSms * ctas_per_sm(true, threads, elems) : 0;
        if (ring > most) most = ring;
    }
    const uint64_t rows = (tokens + 7) / 8 * 8;
    return ((size_t)(rows < most ? rows : most) * 2 * part_width(width) * 4 + 255) / 256 * 256 + 256;
}

extern "C" int abs_residual_norm_backward(const void* dn, uint64_t ld_dn, const void* dy, uint64_t ld_dy, const void* y, uint64_t ld_y,
                                          const void* h, uint64_t ld_h, const void* gate, uint64_t ld_gate, uint32_t gate_kind,
                                          const float* w_post, const float* w_pre, float scale, float eps, uint32_t dtype,
                                          uint64_t tokens, uint64_t width, void* dx, uint64_t ld_dx, void* dh, uint64_t ld_dh,
                                          void* dgate, uint64_t ld_dgate, float* dw_pre, float* dw_post, int accumulate,
                                          void* workspace, size_t workspace_bytes, void* stream) {
    if (const char* why = check_common(dtype, width, gate_kind, gate, w_post, w_pre, scale, eps)) return thread_error(ABS_EINVAL, why);
    if (width > kWidthMax) return thread_error(ABS_ELIMIT, "width exceeds 32768");
    const bool element = gate_kind == ABS_GATE_ELEMENT;
    const size_t es = dtype == ABS_F32 ? 4 : 2;
    const Mat m[8] = {{dn, ld_dn}, {dy, ld_dy}, {y, ld_y}, {h, ld_h}, {element ? gate : nullptr, ld_gate},
                      {dx, ld_dx}, {dh, ld_dh}, {element ? dgate : nullptr, ld_dgate}};
    if (const char* why = check_mats(m, es, width)) return thread_error(ABS_EINVAL, why);
    for (const Mat& out : {m[5], m[6], m[7]})
        for (const Mat& in : {m[0], m[1], m[2], m[3], m[4]})
            if (const char* why = check_in_place(out, in)) return thread_error(ABS_EINVAL, why);
    if ((gate != nullptr) != (dgate != nullptr)) return thread_error(ABS_EINVAL, "dgate must be given exactly when there is a gate");
    if ((w_post != nullptr) != (dw_post != nullptr)) return thread_error(ABS_EINVAL, "dw_post must be given exactly when w_post is");
    if (!dw_pre) return thread_error(ABS_EINVAL, "dw_pre must not be NULL");
    if (misaligned(dw_pre, 4) || misaligned(dw_post, 4) || misaligned(dgate, element ? es : 4))
        return thread_error(ABS_EINVAL, "a gradient is not aligned to its elements");
    if (tokens && (!dn || !y || !h || !dx || !dh)) return thread_error(ABS_EINVAL, "dn, y, h, dx and dh must not be NULL");
    if (!workspace || misaligned(workspace, 256)) return thread_error(ABS_EINVAL, "workspace must be non-NULL and 256-byte aligned");
    if (workspace_bytes < abs_residual_norm_workspace(tokens, width)) return thread_error(ABS_ENOMEM, "workspace too small");
    if (tokens) {
        if (const char* why = check_apart({dx, dh, dgate, static_cast<void*>(dw_pre), static_cast<void*>(dw_post)})) return thread_error(ABS_EINVAL, why);
        // dh is formed from h after dx and dgate of the row are written (k_residual_norm_back)
        if (w_post && (dx == h || (element && dgate == h))) return thread_error(ABS_EINVAL, "with w_post dx and dgate must not be h");
    }
    NormArgs a{};
    a.h = h; a.ld_h = ld_h; a.gate = gate; a.ld_gate = ld_gate;
    a.w_post = w_post; a.w_pre = w_pre; a.scale = scale; a.eps = eps; a.inv_d = 1.f / (float)width; a.T = tokens; a.D = (int)width;
    a.y = const_cast<void*>(y); a.ld_y = ld_y; a.dn = dn; a.ld_dn = ld_dn; a.dy = dy; a.ld_dy = ld_dy;
    a.dx = dx; a.ld_dx = ld_dx; a.dh = dh; a.ld_dh = ld_dh; a.dgate = element ? dgate : nullptr; a.ld_dgate = ld_dgate;
    a.part = static_cast<float*>(workspace);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaSuccess;
    Plan p{};
    if (tokens > 0) {
        const bool wide = rows_aligned(m, es, width);
        p = plan_of(m, es, tokens, width, true, gate_kind);
        e = dtype == ABS_F32 ? run_kind<float>(a, true, gate_kind, wide, p, s) : run_kind<bf16>(a, true, gate_kind, wide, p, s);
    }
    if (e == cudaSuccess)
        e = launch_kernel(k_column_sums, dim3((unsigned)((width + 31) / 32), w_post || gate_kind == ABS_GATE_CHANNEL ? 2 : 1), 1024, 0, s, true,
                          (const float*)a.part, p.grid, (int)width, dw_pre, dw_post, gate_kind == ABS_GATE_CHANNEL ? static_cast<float*>(dgate) : nullptr,
                          w_post, gate_kind == ABS_GATE_CHANNEL ? static_cast<const float*>(gate) : nullptr, accumulate);
    return e == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(e));
}
