// Residual join of a transformer block with its two norms and its gate, forward and backward (abs_residual_norm*).
//
//     u = h / rms(h) * w_post      y = scale x + G u      n = y / rms(y) * w_pre
// One row of the activations at a time: the two means make a row's work a chain of two reductions, and everything between
// them is elementwise.  Bound by memory: forward 4 (5 with an element gate) and backward 6 (8) elements per position.
#include <math.h>

#include "abs_internal.h"
#include "abs_llm.h"
#include "row_ops.cuh"

namespace abs_sgd {
namespace {

constexpr int kWidthMax = 32768;
constexpr int kBackCtas = 296;       // CTAs that leave partial column sums: two for each of 148 SMs

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

// out[c] (+)= sum over the CTAs of part[cta][which][c]: 32 columns per CTA, 8 threads a column, joined in a fixed order.
__global__ void __launch_bounds__(256) k_column_sums(const float* part, int n, int D, float* o0, float* o1, float* o2, int accumulate) {
    __shared__ float sh[8][32];
    pdl_wait();
    pdl_trigger();
    float* out = blockIdx.y == 0 ? o0 : blockIdx.y == 1 ? o1 : o2;
    const int c = blockIdx.x * 32 + threadIdx.x % 32, r = threadIdx.x / 32;
    if (!out) return;
    float s = 0.f;
    if (c < D)
        for (int i = r; i < n; i += 8) s += part[((size_t)i * 3 + blockIdx.y) * D + c];
    sh[r][threadIdx.x % 32] = s;
    __syncthreads();
    if (r == 0 && c < D) {
        for (int i = 1; i < 8; ++i) s += sh[i][threadIdx.x];
        out[c] = accumulate ? out[c] + s : s;
    }
}

template <typename K>
cudaError_t allow_smem(K kernel, size_t bytes) {
    return bytes > 48 * 1024 ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) : cudaSuccess;
}

template <typename T, int kV, bool kPost, int kGate>
cudaError_t run(const NormArgs& a, bool back, int grid, cudaStream_t s) {
    const size_t smem = (size_t)a.D * 4;
    auto k = back ? k_residual_norm_back<T, kV, kPost, kGate> : k_residual_norm<T, kV, kPost, kGate>;
    const cudaError_t e = allow_smem(k, smem);
    if (e != cudaSuccess) return e;
    return launch_kernel(k, grid, 256, smem, s, true, a);
}
template <typename T, int kV>
cudaError_t run_kind(const NormArgs& a, bool back, uint32_t gate, int grid, cudaStream_t s) {
    if (a.w_post)
        return gate == 0 ? run<T, kV, true, 0>(a, back, grid, s) : gate == 1 ? run<T, kV, true, 1>(a, back, grid, s) : run<T, kV, true, 2>(a, back, grid, s);
    return gate == 0 ? run<T, kV, false, 0>(a, back, grid, s) : gate == 1 ? run<T, kV, false, 1>(a, back, grid, s) : run<T, kV, false, 2>(a, back, grid, s);
}

bool misaligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// Rows of all these matrices start on 16-byte boundaries (a NULL matrix does not matter).
struct Mat {
    const void* p;
    size_t ld;
};
template <int N>
bool rows_aligned(const Mat (&m)[N], size_t es, size_t D) {
    if (D * es % 16) return false;
    for (const Mat& q : m)
        if (q.p && (misaligned(q.p, 16) || q.ld * es % 16)) return false;
    return true;
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
    const int grid = (int)(tokens < 148 * 8 ? tokens : 148 * 8);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool wide = rows_aligned(m, es, width);
    const cudaError_t e = dtype == ABS_F32 ? (wide ? run_kind<float, 4>(a, false, gate_kind, grid, s) : run_kind<float, 1>(a, false, gate_kind, grid, s))
                                           : (wide ? run_kind<bf16, 8>(a, false, gate_kind, grid, s) : run_kind<bf16, 1>(a, false, gate_kind, grid, s));
    return e == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(e));
}

extern "C" size_t abs_residual_norm_workspace(uint64_t tokens, uint64_t width) {
    const uint64_t ctas = tokens < (uint64_t)kBackCtas ? tokens : (uint64_t)kBackCtas;
    return ((size_t)ctas * 3 * width * 4 + 255) / 256 * 256 + 256;
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
    const int grid = (int)(tokens < (uint64_t)kBackCtas ? tokens : (uint64_t)kBackCtas);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaSuccess;
    if (grid > 0) {
        const bool wide = rows_aligned(m, es, width);
        e = dtype == ABS_F32 ? (wide ? run_kind<float, 4>(a, true, gate_kind, grid, s) : run_kind<float, 1>(a, true, gate_kind, grid, s))
                             : (wide ? run_kind<bf16, 8>(a, true, gate_kind, grid, s) : run_kind<bf16, 1>(a, true, gate_kind, grid, s));
    }
    if (e == cudaSuccess)
        e = launch_kernel(k_column_sums, dim3((unsigned)((width + 31) / 32), 3), 256, 0, s, true, (const float*)a.part, grid, (int)width, dw_pre,
                          dw_post, gate_kind == ABS_GATE_CHANNEL ? static_cast<float*>(dgate) : nullptr, accumulate);
    return e == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(e));
}
