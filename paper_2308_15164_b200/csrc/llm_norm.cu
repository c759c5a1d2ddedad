// Residual join of a transformer block with its two norms and its gate, forward and backward (abs_residual_norm*).
//
//     u = h / rms(h) * w_post      y = scale x + G u      n = y / rms(y) * w_pre
// One row of the activations at a time: the two means make a row's work a chain of two reductions, and everything between
// them is elementwise.  Bound by memory: forward 4 (5 with an element gate) and backward 6 (8) elements per position.
#include <math.h>

#include "abs_internal.h"
#include "abs_llm.h"
#include "bulk_copy.cuh"
#include "llm_status.cuh"
#include "row_ops.cuh"

namespace abs_sgd {
namespace {

constexpr int kWidthMax = 32768;
constexpr int kSms = 148;
constexpr int kBackCtas = 296;       // CTAs of the plain backward kernel
constexpr int kRingThreads = 512;    // most threads of a CTA of the ring kernels
constexpr int kRingSmem = 216 * 1024;   // shared memory of an SM that their CTAs share (1 KB per CTA is the system's)
constexpr size_t kSmemMax = 227 * 1024; // of one CTA
constexpr int kRingCtasMax = 8;
// CTAs of an SM: 1024 threads forward (64 registers), 512 backward (the column sums take up to 128).
constexpr int ctas_per_sm(bool back, int threads) {
    const int n = (back ? 512 : 1024) / threads;
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
    float* part;                     // [CTA][3][D]: dw_pre, dw_post, channel dgate
};

__device__ __forceinline__ float sigmoid(float v) { return 1.f / (1.f + expf(-v)); }

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
    float* col = a.part + (size_t)blockIdx.x * 3 * a.D;
    for (int c = threadIdx.x * kV; c < a.D; c += 256 * kV)
#pragma unroll
        for (int k = 0; k < kV; ++k) col[c + k] = col[a.D + c + k] = col[2 * (size_t)a.D + c + k] = 0.f;
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
                    col[2 * (size_t)a.D + c + k] += d * (hn * w);
                    du *= static_cast<const float*>(a.gate)[c + k];
                }
                if (kGate == 2) {
                    const float g = sigmoid(vg[k]);
                    du *= g;
                    vg[k] = d * (hn * w) * g * (1.f - g);
                }
                if (kPost) {
                    col[a.D + c + k] += du * hn;
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
// The same rows through a ring of row images in shared memory.  A CTA takes rows b, b + G, ...; one thread keeps kS
// rows of copies in flight (cp.async.bulk, one per input matrix), so that the chain of reductions of a row hides
// behind the copies of the next ones.  A thread owns kP pieces of 16 bytes and at most one single element.
// Rows of odd width start at every alignment.  G is a multiple of the period with which the alignment repeats, so that
// all rows of one CTA are cut alike: single elements up to the first 16-byte boundary, pieces, single elements.  The
// copies move the pieces (nothing outside the row is read), the single elements are plain loads.  All matrices of the
// call have to be aligned alike.
// The weights are kept in shared memory, cut like the rows; the column sums in registers.
// ------------------------------------------------------------------------------------------------
constexpr int kRingMax = 8;

struct RingArgs {
    NormArgs n;
    int stages;
    uint32_t row_bytes;              // room for one row image, a multiple of 16
};

struct RingCtl {
    alignas(8) uint64_t full[kRingMax];
    float red[2][3 * 32];
    float red2[32];
};

// Sums over the CTA's threads, one synchronisation: `sh` must not be the buffer of the reduction just before.
template <int kN>
__device__ __forceinline__ void cta_sum(float (&v)[kN], float* sh) {
    const int warps = blockDim.x / 32, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
#pragma unroll
    for (int k = 0; k < kN; ++k) {
#pragma unroll
        for (int o = 16; o; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
        if (lane == 0) sh[k * 32 + warp] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kN; ++k) {
        float s = lane < warps ? sh[k * 32 + lane] : 0.f;
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        v[k] = s;
    }
}

// What a thread needs to know of its rows' cut, and the ring's copies.
template <typename T, int kP, int kIn>
struct Ring {
    RowCut cut;
    int extra;                       // column of this thread's single element, or -1
    const T* in[kIn];
    size_t ld[kIn];
    RingCtl* ctl;
    uint8_t* base;
    uint32_t row_bytes, bytes;
    int stages;
    size_t rows;
    int st = 0;
    uint32_t phase = 0;
    bool ok = true;

    __device__ __forceinline__ void cut_rows(const T* row0, int D) {
        cut = cut_row(row0, D);
        bytes = (uint32_t)cut.pieces * 16u;
        const int tid = threadIdx.x;
        extra = tid < cut.head ? tid : tid < cut.head + cut.tail ? D - cut.tail + tid - cut.head : -1;
    }
    __device__ __forceinline__ void load(int stage, size_t t) {       // one thread
        if (t >= rows || bytes == 0) return;
        uint32_t total = 0;
#pragma unroll
        for (int i = 0; i < kIn; ++i) total += in[i] ? bytes : 0;
        mbar_expect_tx(&ctl->full[stage], total);
#pragma unroll
        for (int i = 0; i < kIn; ++i)
            if (in[i]) bulk_load(base + ((size_t)stage * kIn + i) * row_bytes, in[i] + t * ld[i] + cut.head, bytes, &ctl->full[stage]);
    }
    __device__ __forceinline__ void load_extra(size_t t, float (&v)[kIn]) const {
#pragma unroll
        for (int i = 0; i < kIn; ++i) v[i] = extra >= 0 && t < rows && in[i] ? to_f(in[i][t * ld[i] + extra]) : 0.f;
    }
    __device__ __forceinline__ void wait() {
        if (bytes != 0 && !mbar_wait(&ctl->full[st], phase, ok ? kSpinLimit : 1u)) ok = false;
    }
    __device__ __forceinline__ void next() {
        if (++st == stages) { st = 0; phase ^= 1u; }
    }
    // Piece j of this thread of input i, in the current row's image.
    __device__ __forceinline__ void piece(int i, int j, float (&v)[kVec<T>]) const {
        Pack<T, kVec<T>>::load(reinterpret_cast<const T*>(base + ((size_t)st * kIn + i) * row_bytes) + (threadIdx.x + j * blockDim.x) * kVec<T>, v);
    }
    __device__ __forceinline__ bool has(int j) const { return (int)(threadIdx.x + j * blockDim.x) < cut.pieces; }
    __device__ __forceinline__ int column(int j) const { return cut.head + (int)(threadIdx.x + j * blockDim.x) * kVec<T>; }
};

// A weight vector in shared memory, four floats of a piece side by side: [kP][kVec / 4][threads].
template <typename T, int kP>
__device__ __forceinline__ float4* weight_slot(float4* w, int j, int q) { return w + ((size_t)j * (kVec<T> / 4) + q) * blockDim.x + threadIdx.x; }
template <typename T, int kP>
constexpr int kWeightVecs = kP * (kVec<T> / 4);      // float4 per thread
template <typename T, int kP, typename R>
__device__ __forceinline__ float stage_weight(float4* w, const float* src, const R& r) {
#pragma unroll
    for (int j = 0; j < kP; ++j)
        if (r.has(j))
#pragma unroll
            for (int q = 0; q < kVec<T> / 4; ++q) {
                const float* p = src + r.column(j) + 4 * q;
                *weight_slot<T, kP>(w, j, q) = make_float4(p[0], p[1], p[2], p[3]);
            }
    return r.extra >= 0 ? src[r.extra] : 0.f;
}
template <typename T, int kP>
__device__ __forceinline__ void weight(float4* w, int j, float (&v)[kVec<T>]) {
#pragma unroll
    for (int q = 0; q < kVec<T> / 4; ++q) {
        const float4 f = *weight_slot<T, kP>(w, j, q);
        v[4 * q] = f.x; v[4 * q + 1] = f.y; v[4 * q + 2] = f.z; v[4 * q + 3] = f.w;
    }
}

template <typename T, int kP, bool kPost, int kGate>
__global__ void __launch_bounds__(512, kP == 4 ? 1 : 2) k_join(const __grid_constant__ RingArgs ra) {
    constexpr int kV = kVec<T>, kIn = kGate == 2 ? 3 : 2;
    const NormArgs& a = ra.n;
    extern __shared__ __align__(16) uint8_t smem[];
    Ring<T, kP, kIn> r;
    r.ctl = reinterpret_cast<RingCtl*>(smem);
    float4* w_pre = reinterpret_cast<float4*>(smem + (sizeof(RingCtl) + 15) / 16 * 16);
    float4* w_post = w_pre + kWeightVecs<T, kP> * blockDim.x;
    float4* w_gate = w_post + (kPost ? kWeightVecs<T, kP> * blockDim.x : 0);
    r.base = reinterpret_cast<uint8_t*>(w_gate + (kGate == 1 ? kWeightVecs<T, kP> * blockDim.x : 0));
    r.row_bytes = ra.row_bytes; r.stages = ra.stages; r.rows = a.T;
    r.in[0] = static_cast<const T*>(a.x); r.ld[0] = a.ld_x;
    r.in[1] = static_cast<const T*>(a.h); r.ld[1] = a.ld_h;
    if (kGate == 2) { r.in[kIn - 1] = static_cast<const T*>(a.gate); r.ld[kIn - 1] = a.ld_gate; }
    const size_t t0 = blockIdx.x, G = gridDim.x;
    r.cut_rows(r.in[0] + t0 * a.ld_x, a.D);
    if (threadIdx.x == 0) {
        for (int i = 0; i < r.stages; ++i) mbar_init(&r.ctl->full[i], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    pdl_wait();
    pdl_trigger();
    if (threadIdx.x == 0)
        for (int i = 0; i < r.stages; ++i) r.load(i, t0 + i * G);
    float ex[kIn], nx[kIn];
    r.load_extra(t0, nx);
    const float xw_pre = stage_weight<T, kP>(w_pre, a.w_pre, r);
    const float xw_post = kPost ? stage_weight<T, kP>(w_post, a.w_post, r) : 1.f;
    const float xw_gate = kGate == 1 ? stage_weight<T, kP>(w_gate, static_cast<const float*>(a.gate), r) : 1.f;

    int k = 0;
    for (size_t t = t0; t < a.T; t += G, ++k, r.next()) {
        float* red = r.ctl->red[k & 1];
#pragma unroll
        for (int i = 0; i < kIn; ++i) ex[i] = nx[i];
        r.load_extra(t + G, nx);
        r.wait();
        const auto refill = [&] {              // everybody has passed the first synchronisation: the previous row's image is free
            if (threadIdx.x == 0 && k > 0) r.load((r.st == 0 ? r.stages : r.st) - 1, t + (size_t)(r.stages - 1) * G);
        };
        float rh = 1.f;
        if (kPost) {
            float s[1] = {r.extra >= 0 ? ex[1] * ex[1] : 0.f};
#pragma unroll
            for (int j = 0; j < kP; ++j)
                if (r.has(j)) {
                    float v[kV];
                    r.piece(1, j, v);
#pragma unroll
                    for (int i = 0; i < kV; ++i) s[0] += v[i] * v[i];
                }
            cta_sum<1>(s, red);
            refill();
            rh = 1.f / sqrtf(s[0] * a.inv_d + a.eps);
        }
        float y[kP][kV], s[1] = {0.f}, xy = 0.f;
        T* yrow = static_cast<T*>(a.y) + t * a.ld_y;
#pragma unroll
        for (int j = 0; j < kP; ++j)
            if (r.has(j)) {
                float u[kV], g[kV];
                r.piece(0, j, y[j]);
                r.piece(1, j, u);
                if (kPost) {
                    weight<T, kP>(w_post, j, g);
#pragma unroll
                    for (int i = 0; i < kV; ++i) u[i] *= rh * g[i];
                }
                if (kGate == 1) {
                    weight<T, kP>(w_gate, j, g);
#pragma unroll
                    for (int i = 0; i < kV; ++i) u[i] *= g[i];
                }
                if (kGate == 2) {
                    r.piece(kIn - 1, j, g);
#pragma unroll
                    for (int i = 0; i < kV; ++i) u[i] *= sigmoid(g[i]);
                }
#pragma unroll
                for (int i = 0; i < kV; ++i) {
                    y[j][i] = a.scale * y[j][i] + u[i];
                    s[0] += y[j][i] * y[j][i];
                }
                if (r.ok) Pack<T, kV>::store(yrow + r.column(j), y[j]);
            }
        if (r.extra >= 0) {
            float u = ex[1] * rh * xw_post * xw_gate;
            if (kGate == 2) u *= sigmoid(ex[kIn - 1]);
            xy = a.scale * ex[0] + u;
            s[0] += xy * xy;
            if (r.ok) yrow[r.extra] = from_f<T>(xy);
        }
        cta_sum<1>(s, kPost ? r.ctl->red2 : red);
        if (!kPost) refill();
        const float ry = 1.f / sqrtf(s[0] * a.inv_d + a.eps);
        T* nrow = static_cast<T*>(a.n) + t * a.ld_n;
#pragma unroll
        for (int j = 0; j < kP; ++j)
            if (r.has(j) && r.ok) {
                float g[kV];
                weight<T, kP>(w_pre, j, g);
#pragma unroll
                for (int i = 0; i < kV; ++i) y[j][i] *= ry * g[i];
                Pack<T, kV>::store(nrow + r.column(j), y[j]);
            }
        if (r.extra >= 0 && r.ok) nrow[r.extra] = from_f<T>(xy * (ry * xw_pre));
    }
    if (!r.ok) report_timeout();
}

template <typename T, int kP, bool kPost, int kGate>
__global__ void __launch_bounds__(512, 1) k_join_back(const __grid_constant__ RingArgs ra) {
    constexpr int kV = kVec<T>, kIn = kGate == 2 ? 5 : 4;
    const NormArgs& a = ra.n;
    extern __shared__ __align__(16) uint8_t smem[];
    Ring<T, kP, kIn> r;
    r.ctl = reinterpret_cast<RingCtl*>(smem);
    float4* w_pre = reinterpret_cast<float4*>(smem + (sizeof(RingCtl) + 15) / 16 * 16);
    float4* w_post = w_pre + kWeightVecs<T, kP> * blockDim.x;
    float4* w_gate = w_post + (kPost ? kWeightVecs<T, kP> * blockDim.x : 0);
    r.base = reinterpret_cast<uint8_t*>(w_gate + (kGate == 1 ? kWeightVecs<T, kP> * blockDim.x : 0));
    r.row_bytes = ra.row_bytes; r.stages = ra.stages; r.rows = a.T;
    r.in[0] = static_cast<const T*>(a.y); r.ld[0] = a.ld_y;
    r.in[1] = static_cast<const T*>(a.dn); r.ld[1] = a.ld_dn;
    r.in[2] = static_cast<const T*>(a.h); r.ld[2] = a.ld_h;
    r.in[3] = static_cast<const T*>(a.dy); r.ld[3] = a.ld_dy;
    if (kGate == 2) { r.in[kIn - 1] = static_cast<const T*>(a.gate); r.ld[kIn - 1] = a.ld_gate; }
    const bool has_dy = a.dy != nullptr;
    const size_t t0 = blockIdx.x, G = gridDim.x;
    r.cut_rows(r.in[0] + t0 * a.ld_y, a.D);
    if (threadIdx.x == 0) {
        for (int i = 0; i < r.stages; ++i) mbar_init(&r.ctl->full[i], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    pdl_wait();
    pdl_trigger();
    if (threadIdx.x == 0)
        for (int i = 0; i < r.stages; ++i) r.load(i, t0 + i * G);
    float ex[kIn], nx[kIn];
    r.load_extra(t0, nx);
    const float xw_pre = stage_weight<T, kP>(w_pre, a.w_pre, r);
    const float xw_post = kPost ? stage_weight<T, kP>(w_post, a.w_post, r) : 1.f;
    const float xw_gate = kGate == 1 ? stage_weight<T, kP>(w_gate, static_cast<const float*>(a.gate), r) : 1.f;
    float c_pre[kP][kV], c_post[kP][kV], c_gate[kP][kV], x_pre = 0.f, x_post = 0.f, x_gate = 0.f;
#pragma unroll
    for (int j = 0; j < kP; ++j)
#pragma unroll
        for (int i = 0; i < kV; ++i) c_pre[j][i] = c_post[j][i] = c_gate[j][i] = 0.f;

    int k = 0;
    for (size_t t = t0; t < a.T; t += G, ++k, r.next()) {
#pragma unroll
        for (int i = 0; i < kIn; ++i) ex[i] = nx[i];
        r.load_extra(t + G, nx);
        r.wait();
        float s[3] = {0.f, 0.f, 0.f};            // sum y^2, sum dn w_pre y, sum h^2
#pragma unroll
        for (int j = 0; j < kP; ++j)
            if (r.has(j)) {
                float y[kV], n[kV], w[kV];
                r.piece(0, j, y);
                r.piece(1, j, n);
                weight<T, kP>(w_pre, j, w);
#pragma unroll
                for (int i = 0; i < kV; ++i) {
                    s[0] += y[i] * y[i];
                    s[1] += n[i] * w[i] * y[i];
                }
                if (kPost) {
                    r.piece(2, j, y);
#pragma unroll
                    for (int i = 0; i < kV; ++i) s[2] += y[i] * y[i];
                }
            }
        if (r.extra >= 0) {
            s[0] += ex[0] * ex[0];
            s[1] += ex[1] * xw_pre * ex[0];
            if (kPost) s[2] += ex[2] * ex[2];
        }
        cta_sum<3>(s, r.ctl->red[k & 1]);
        if (threadIdx.x == 0 && k > 0) r.load((r.st == 0 ? r.stages : r.st) - 1, t + (size_t)(r.stages - 1) * G);   // the previous row's image is free
        const float ry = 1.f / sqrtf(s[0] * a.inv_d + a.eps);
        const float along = s[1] * a.inv_d * ry;
        const float rh = kPost ? 1.f / sqrtf(s[2] * a.inv_d + a.eps) : 1.f;
        float q[1] = {0.f}, du[kP][kV], xdu = 0.f;
        T* dx = static_cast<T*>(a.dx) + t * a.ld_dx;
        T* dh = static_cast<T*>(a.dh) + t * a.ld_dh;
        T* dz = static_cast<T*>(a.dgate) + t * a.ld_dgate;
#pragma unroll
        for (int j = 0; j < kP; ++j)
            if (r.has(j)) {
                float d[kV], v[kV], w[kV];
                r.piece(0, j, v);                // yn
                r.piece(1, j, d);                // dn
                weight<T, kP>(w_pre, j, w);
#pragma unroll
                for (int i = 0; i < kV; ++i) {
                    v[i] *= ry;
                    c_pre[j][i] += d[i] * v[i];
                    d[i] = ry * (d[i] * w[i] - v[i] * along);
                }
                if (has_dy) {
                    r.piece(3, j, v);
#pragma unroll
                    for (int i = 0; i < kV; ++i) d[i] += v[i];
                }
#pragma unroll
                for (int i = 0; i < kV; ++i) v[i] = a.scale * d[i];
                if (r.ok) Pack<T, kV>::store(dx + r.column(j), v);
                r.piece(2, j, v);                // hn, or h without w_post
                if (kPost) {
                    weight<T, kP>(w_post, j, w);
#pragma unroll
                    for (int i = 0; i < kV; ++i) v[i] *= rh;
                }
                if (kGate == 1) {
                    float g[kV];
                    weight<T, kP>(w_gate, j, g);
#pragma unroll
                    for (int i = 0; i < kV; ++i) {
                        c_gate[j][i] += d[i] * (kPost ? v[i] * w[i] : v[i]);
                        d[i] *= g[i];
                    }
                }
                if (kGate == 2) {
                    float g[kV];
                    r.piece(kIn - 1, j, g);
#pragma unroll
                    for (int i = 0; i < kV; ++i) {
                        g[i] = sigmoid(g[i]);
                        const float dg = d[i] * g[i];
                        g[i] = dg * (1.f - g[i]) * (kPost ? v[i] * w[i] : v[i]);
                        d[i] = dg;
                    }
                    if (r.ok) Pack<T, kV>::store(dz + r.column(j), g);
                }
                if (kPost) {
#pragma unroll
                    for (int i = 0; i < kV; ++i) {
                        c_post[j][i] += d[i] * v[i];
                        du[j][i] = d[i] * w[i];
                        q[0] += du[j][i] * v[i];
                    }
                } else if (r.ok) {
                    Pack<T, kV>::store(dh + r.column(j), d);
                }
            }
        if (r.extra >= 0) {
            const float yn = ex[0] * ry, hn = ex[2] * rh;
            x_pre += ex[1] * yn;
            float d = ry * (ex[1] * xw_pre - yn * along) + ex[3];
            const float xdx = a.scale * d;
            if (kGate == 1) {
                x_gate += d * (hn * xw_post);
                d *= xw_gate;
            }
            float xdz = 0.f;
            if (kGate == 2) {
                const float g = sigmoid(ex[kIn - 1]);
                d *= g;
                xdz = d * (1.f - g) * (hn * xw_post);
            }
            x_post += d * hn;
            xdu = d * xw_post;
            q[0] += xdu * hn;
            if (r.ok) {
                dx[r.extra] = from_f<T>(xdx);
                if (kGate == 2) dz[r.extra] = from_f<T>(xdz);
                if (!kPost) dh[r.extra] = from_f<T>(xdu);
            }
        }
        if (kPost) {
            cta_sum<1>(q, r.ctl->red2);
            const float m = q[0] * a.inv_d * rh;
#pragma unroll
            for (int j = 0; j < kP; ++j)
                if (r.has(j)) {
                    float h[kV];
                    r.piece(2, j, h);
#pragma unroll
                    for (int i = 0; i < kV; ++i) h[i] = rh * (du[j][i] - h[i] * m);
                    if (r.ok) Pack<T, kV>::store(dh + r.column(j), h);
                }
            if (r.extra >= 0 && r.ok) dh[r.extra] = from_f<T>(rh * (xdu - ex[2] * m));
        }
    }
    float* col = a.part + (size_t)blockIdx.x * 3 * a.D;
#pragma unroll
    for (int j = 0; j < kP; ++j)
        if (r.has(j))
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                const int c = r.column(j) + i;
                col[c] = c_pre[j][i];
                if (kPost) col[a.D + c] = c_post[j][i];
                if (kGate == 1) col[2 * (size_t)a.D + c] = c_gate[j][i];
            }
    if (r.extra >= 0) {
        col[r.extra] = x_pre;
        if (kPost) col[a.D + r.extra] = x_post;
        if (kGate == 1) col[2 * (size_t)a.D + r.extra] = x_gate;
    }
    if (!r.ok) report_timeout();
}

// out[c] (+)= sum over the CTAs of part[cta][which][c]: 32 columns per CTA, 32 threads a column, joined in a fixed order.
__global__ void __launch_bounds__(1024) k_column_sums(const float* part, int n, int D, float* o0, float* o1, float* o2, int accumulate) {
    __shared__ float sh[32][33];
    pdl_wait();
    pdl_trigger();
    float* out = blockIdx.y == 0 ? o0 : blockIdx.y == 1 ? o1 : o2;
    if (!out) return;
    const int lane = threadIdx.x % 32, r = threadIdx.x / 32;
    const int c = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (c < D) {
        const float* p = part + (size_t)blockIdx.y * D + c;
#pragma unroll 4
        for (int i = r; i < n; i += 32) s += p[(size_t)i * 3 * D];
    }
    sh[r][lane] = s;
    __syncthreads();
    s = sh[lane][r];                               // column r of this CTA's 32, partial sum `lane`
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    const int cc = blockIdx.x * 32 + r;
    if (lane == 0 && cc < D) out[cc] = accumulate ? out[cc] + s : s;
}

template <typename K>
cudaError_t allow_smem(K kernel, size_t bytes) {
    return bytes > 48 * 1024 ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) : cudaSuccess;
}

// How a call is launched.  ring: all matrices aligned alike and the row within the pieces that a CTA's threads own.
struct Plan {
    bool ring;
    int threads, pieces;             // of a CTA; of a thread
    int grid, stages;
    uint32_t row_bytes;
    size_t smem;
};

template <typename T, int kV, bool kPost, int kGate>
cudaError_t run_plain(const NormArgs& a, bool back, int grid, cudaStream_t s) {
    const size_t smem = (size_t)a.D * 4;
    auto k = back ? k_residual_norm_back<T, kV, kPost, kGate> : k_residual_norm<T, kV, kPost, kGate>;
    const cudaError_t e = allow_smem(k, smem);
    if (e != cudaSuccess) return e;
    return launch_kernel(k, grid, 256, smem, s, true, a);
}
template <typename T, int kP, bool kPost, int kGate>
cudaError_t run_ring(const NormArgs& a, bool back, const Plan& p, cudaStream_t s) {
    const RingArgs r{a, p.stages, p.row_bytes};
    if (back) {
        if constexpr (kP <= 2) {
            const cudaError_t e = allow_smem(k_join_back<T, kP, kPost, kGate>, p.smem);
            return e != cudaSuccess ? e : launch_kernel(k_join_back<T, kP, kPost, kGate>, p.grid, p.threads, p.smem, s, true, r);
        }
        return cudaErrorInvalidValue;
    }
    const cudaError_t e = allow_smem(k_join<T, kP, kPost, kGate>, p.smem);
    return e != cudaSuccess ? e : launch_kernel(k_join<T, kP, kPost, kGate>, p.grid, p.threads, p.smem, s, true, r);
}
template <typename T, bool kPost, int kGate>
cudaError_t run(const NormArgs& a, bool back, bool wide, const Plan& p, cudaStream_t s) {
    if (!p.ring) return wide ? run_plain<T, kVec<T>, kPost, kGate>(a, back, p.grid, s) : run_plain<T, 1, kPost, kGate>(a, back, p.grid, s);
    return p.pieces == 1 ? run_ring<T, 1, kPost, kGate>(a, back, p, s)
         : p.pieces == 2 ? run_ring<T, 2, kPost, kGate>(a, back, p, s) : run_ring<T, 4, kPost, kGate>(a, back, p, s);
}
template <typename T>
cudaError_t run_kind(const NormArgs& a, bool back, uint32_t gate, bool wide, const Plan& p, cudaStream_t s) {
    if (a.w_post)
        return gate == 0 ? run<T, true, 0>(a, back, wide, p, s) : gate == 1 ? run<T, true, 1>(a, back, wide, p, s) : run<T, true, 2>(a, back, wide, p, s);
    return gate == 0 ? run<T, false, 0>(a, back, wide, p, s) : gate == 1 ? run<T, false, 1>(a, back, wide, p, s) : run<T, false, 2>(a, back, wide, p, s);
}

bool misaligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

struct Mat {
    const void* p;
    size_t ld;
};
// All rows t of these matrices (a NULL one does not matter) start at the same offset from a 16-byte boundary; *period: after
// how many rows the offset repeats.
template <int N>
bool aligned_alike(const Mat (&m)[N], size_t es, size_t* period) {
    size_t off = 16, step = 16;
    for (const Mat& q : m)
        if (q.p) {
            const size_t o = reinterpret_cast<uintptr_t>(q.p) & 15, st = q.ld * es & 15;
            if (off == 16) { off = o; step = st; }
            if (off != o || step != st) return false;
        }
    *period = 1;
    while ((*period * step & 15) != 0) *period *= 2;
    return true;
}
template <int N>
bool rows_aligned(const Mat (&m)[N], size_t es, size_t D) {
    size_t period = 0;
    if (D * es % 16 || !aligned_alike(m, es, &period) || period != 1) return false;
    for (const Mat& q : m)
        if (q.p) return (reinterpret_cast<uintptr_t>(q.p) & 15) == 0;
    return true;
}
// Threads of a CTA for rows of this many pieces, and pieces per thread (at most `most`; 0: more than they can own).
void ring_shape(size_t pieces, int most, int* threads, int* per_thread) {
    *per_thread = pieces <= kRingThreads ? 1 : pieces <= 2 * kRingThreads ? 2 : pieces <= 4 * kRingThreads ? 4 : 8;
    if (*per_thread > most) *per_thread = 0;
    const size_t per = *per_thread ? (pieces + *per_thread - 1) / *per_thread : kRingThreads;
    *threads = (int)(per <= 32 ? 32 : (per + 31) / 32 * 32);
}
template <int N>
Plan plan_of(const Mat (&m)[N], size_t es, uint64_t T, uint64_t D, bool back, uint32_t gate_kind, bool post) {
    Plan p{};
    size_t period = 1;
    ring_shape(D * es / 16, back ? 2 : 4, &p.threads, &p.pieces);
    p.ring = p.pieces > 0 && aligned_alike(m, es, &period);
    p.row_bytes = (uint32_t)((D * es + 15) / 16 * 16);
    const size_t in = back ? (gate_kind == ABS_GATE_ELEMENT ? 5 : 4) : (gate_kind == ABS_GATE_ELEMENT ? 3 : 2);
    const size_t weights = 1 + (post ? 1 : 0) + (gate_kind == ABS_GATE_CHANNEL ? 1 : 0);
    const size_t fixed = (sizeof(RingCtl) + 15) / 16 * 16 + weights * p.pieces * (4 / es) * p.threads * 16;
    size_t ctas = 0;
    if (p.ring) {      // as many CTAs as the registers allow, fewer where two rows would not fit; then as many rows as fit
        ctas = (size_t)ctas_per_sm(back, p.threads);
        while (ctas > 1 && fixed + 2 * in * p.row_bytes > kRingSmem / ctas) --ctas;
        const size_t room = ctas > 1 ? kRingSmem / ctas : kSmemMax;
        if (fixed + 2 * in * p.row_bytes > room) p.ring = false;
        else {
            const size_t fit = (room - fixed) / (in * p.row_bytes);
            p.stages = (int)(fit < (size_t)kRingMax ? fit : (size_t)kRingMax);
            p.smem = fixed + p.stages * in * p.row_bytes;
        }
    }
    if (!p.ring) {
        const uint64_t cap = back ? kBackCtas : kSms * 8;
        p.grid = (int)(T < cap ? T : cap);
        return p;
    }
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
    if (tokens == 0) return ABS_OK;
    if (!x || !h || !y || !n) return thread_error(ABS_EINVAL, "x, h, y and n must not be NULL");
    NormArgs a{};
    a.x = x; a.ld_x = ld_x; a.h = h; a.ld_h = ld_h; a.gate = gate; a.ld_gate = ld_gate;
    a.w_post = w_post; a.w_pre = w_pre; a.scale = scale; a.eps = eps; a.inv_d = 1.f / (float)width; a.T = tokens; a.D = (int)width;
    a.y = y; a.ld_y = ld_y; a.n = n; a.ld_n = ld_n;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool wide = rows_aligned(m, es, width);
    const Plan p = plan_of(m, es, tokens, width, false, gate_kind, w_post != nullptr);
    const cudaError_t e = dtype == ABS_F32 ? run_kind<float>(a, false, gate_kind, wide, p, s) : run_kind<bf16>(a, false, gate_kind, wide, p, s);
    return e == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(e));
}

extern "C" size_t abs_residual_norm_workspace(uint64_t tokens, uint64_t width) {
    int threads = 0, per_thread = 0;
    ring_shape(width / 8, 2, &threads, &per_thread);      // bf16: the smaller CTAs, so more of them
    const uint64_t ring = (uint64_t)kSms * ctas_per_sm(true, threads);
    const uint64_t most = ring > kBackCtas ? ring : kBackCtas, rows = (tokens + 7) / 8 * 8;
    return ((size_t)(rows < most ? rows : most) * 3 * width * 4 + 255) / 256 * 256 + 256;
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
    if ((gate != nullptr) != (dgate != nullptr)) return thread_error(ABS_EINVAL, "dgate must be given exactly when there is a gate");
    if ((w_post != nullptr) != (dw_post != nullptr)) return thread_error(ABS_EINVAL, "dw_post must be given exactly when w_post is");
    if (!dw_pre) return thread_error(ABS_EINVAL, "dw_pre must not be NULL");
    if (misaligned(dw_pre, 4) || misaligned(dw_post, 4) || misaligned(dgate, element ? es : 4))
        return thread_error(ABS_EINVAL, "a gradient is not aligned to its elements");
    if (tokens && (!dn || !y || !h || !dx || !dh)) return thread_error(ABS_EINVAL, "dn, y, h, dx and dh must not be NULL");
    if (!workspace || misaligned(workspace, 256)) return thread_error(ABS_EINVAL, "workspace must be non-NULL and 256-byte aligned");
    if (workspace_bytes < abs_residual_norm_workspace(tokens, width)) return thread_error(ABS_ENOMEM, "workspace too small");
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
        p = plan_of(m, es, tokens, width, true, gate_kind, w_post != nullptr);
        e = dtype == ABS_F32 ? run_kind<float>(a, true, gate_kind, wide, p, s) : run_kind<bf16>(a, true, gate_kind, wide, p, s);
    }
    if (e == cudaSuccess)
        e = launch_kernel(k_column_sums, dim3((unsigned)((width + 31) / 32), 3), 1024, 0, s, true, (const float*)a.part, p.grid, (int)width, dw_pre,
                          dw_post, gate_kind == ABS_GATE_CHANNEL ? static_cast<float*>(dgate) : nullptr, accumulate);
    return e == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(e));
}
