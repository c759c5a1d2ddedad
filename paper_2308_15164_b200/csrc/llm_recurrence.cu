// Gated linear recurrence over packed sequences (abs_recurrence*).
//
//     h_t = a_t h_{t-1} + b_t,   a = sigmoid(g),  b = (1 - a) x  or  x
// Composed, rows i..j act on the state in front of them as h -> A h + B with A = a_i ... a_j, and two such maps compose to
// (A2 A1, A2 B1 + B2): that is what lets a long sequence be worked on in parallel.  Backward with e_t = a_t d_t, what row t hands
// to row t - 1, is the same recurrence in reversed time: e_t = a_t e_{t+1} + a_t dy_t, d_t = dy_t + e_{t+1}.
// A sequence's first row forgets what is in front of it; as a map that is A = -0, which stays -0 in every product with later
// factors (a >= +0) and is told from an underflow by its sign, so that no infinity or NaN of one sequence reaches the next.
#include <math.h>

#include <algorithm>

#include "abs_internal.h"
#include "abs_llm.h"
#include "bulk_copy.cuh"
#include "llm_host.h"
#include "llm_status.cuh"
#include "row_ops.cuh"

namespace abs_sgd {
namespace {

constexpr int kWarps = 8, kRows = 16, kTile = kWarps * kRows;   // rows of a warp, of a CTA
constexpr int kGroup = 32;               // tiles between two published states
constexpr uint64_t kSizeMax = 0x7ffffc00ull;

struct RecArgs {
    const void *x, *g, *dy, *y;          // y: of the forward pass (backward only)
    size_t ld_x, ld_g, ld_dy, ld_y;
    void *out, *out2;                    // forward: y; backward: dx, dg
    size_t ld_out, ld_out2;
    const int32_t* offsets;
    const float *h0, *before;            // before: h0, backward dlast: the state in front of a sequence in scan order
    float* after;                        // last, backward dh0
    int T, D, seqs;
    int tiles, strips;
    uint32_t* ctl;                       // [0]: tickets; then a flag per (tile, strip)
    float2* maps;                        // [tile][strip][lanes' columns]: a tile's map (A, B), or (0, state) for the last of a group
};

// sigmoid(g) and 1 - sigmoid(g), each to its own precision.
__device__ __forceinline__ void gate_of(float g, float& a, float& rest, bf16) {
    float v = g * -1.4426950408889634f;
    v = v > 126.f ? 126.f : v;           // keeps a NaN
    const float e = exp2_of(v);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a) : "f"(1.f + e));
    rest = e * a;
}
__device__ __forceinline__ void gate_of(float g, float& a, float& rest, float) {
    const float v = g < -87.f ? 87.f : -g;
    const float e = expf(v);
    a = 1.f / (1.f + e);
    rest = e * a;
}
__device__ __forceinline__ bool forgets(float A) { return __float_as_uint(A) == 0x80000000u; }
// (A, B) followed by (A2, B2).
__device__ __forceinline__ void compose(float& A, float& B, float A2, float B2) {
    if (forgets(A2)) {
        A = A2;
        B = B2;
    } else {
        B = fmaf(A2, B, B2);
        A *= A2;
    }
}
__device__ __forceinline__ float apply(float A, float B, float s) { return forgets(A) ? B : fmaf(A, s, B); }

template <typename T, int kV>
__device__ __forceinline__ void load_v(const T* p, int n, float (&v)[kV]) {
    if (kV == 2 && n == 2) {
        if constexpr (sizeof(T) == 2) {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(p);
            v[0] = __uint_as_float(w << 16);
            v[kV - 1] = __uint_as_float(w & 0xFFFF0000u);
        } else {
            const float2 f = *reinterpret_cast<const float2*>(p);
            v[0] = f.x;
            v[kV - 1] = f.y;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < kV; ++i) v[i] = i < n ? to_f(p[i]) : 0.f;
}
template <typename T, int kV>
__device__ __forceinline__ void store_v(T* p, int n, const float (&v)[kV]) {
    if (kV == 2 && n == 2) {
        if constexpr (sizeof(T) == 2) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[0], v[kV - 1]);
            *reinterpret_cast<__nv_bfloat162*>(p) = b;
        } else {
            *reinterpret_cast<float2*>(p) = make_float2(v[0], v[kV - 1]);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < kV; ++i)
        if (i < n) p[i] = from_f<T>(v[i]);
}

// Which sequence row t belongs to: the number of sequences that end at or before it.
__device__ __forceinline__ int begin_of(const RecArgs& a, int q) { return a.offsets ? min(max(a.offsets[q], 0), a.T) : q == 0 ? 0 : a.T; }
__device__ __forceinline__ int sequence_of(const RecArgs& a, int t) {
    int lo = 0, hi = a.seqs;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (begin_of(a, mid + 1) <= t) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

// A tile: kTile rows (in scan order: backward from the last one) of 32 kV columns; a lane owns kV columns, a warp kRows rows.
template <typename T, int kV, uint32_t kKind, bool kBack>
__global__ void __launch_bounds__(kWarps * 32) k_recurrence(const __grid_constant__ RecArgs a) {
    __shared__ float2 sh_map[kWarps][32 * kV];
    __shared__ float sh_state[32 * kV];
    __shared__ int sh_ticket;
    __shared__ int sh_ok;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    pdl_wait();
    pdl_trigger();
    if (threadIdx.x == 0) {
        sh_ticket = a.tiles > 1 ? (int)atomicAdd(&a.ctl[0], 1u) : blockIdx.x;
        sh_ok = 1;
    }
    __syncthreads();
    const int tile = sh_ticket / a.strips, strip = sh_ticket % a.strips;
    const int c = (strip * 32 + lane) * kV, n = min(max(a.D - c, 0), kV);
    const int u0 = tile * kTile + warp * kRows;          // first row of the warp, in scan order
    auto row = [&](int u) { return kBack ? a.T - 1 - u : u; };

    // ---- rows
    float keep[kRows][kV], feed[kRows][kV];              // a; b, backward dy
    float rest[kBack ? kRows : 1][kV], other[kBack ? kRows : 1][kV];   // 1 - a; h_{t-1} (- x)
    int seq = 0;
    uint32_t member, first, final;                       // of the warp's rows: in a sequence; first and last one in scan order
    {
        bool m = false, f = false, l = false;
        if (lane < kRows && u0 + lane < a.T) {
            const int t = row(u0 + lane);
            seq = sequence_of(a, t);
            m = seq < a.seqs && t >= begin_of(a, seq);
            if (m) {
                f = t == begin_of(a, seq);
                l = t == begin_of(a, seq + 1) - 1;
            }
        }
        member = __ballot_sync(0xffffffffu, m);
        first = __ballot_sync(0xffffffffu, kBack ? l : f);
        final = __ballot_sync(0xffffffffu, kBack ? f : l);
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        float gv[kV], xv[kV], dv[kV], hv[kV];
#pragma unroll
        for (int i = 0; i < kV; ++i) gv[i] = xv[i] = dv[i] = hv[i] = 0.f;
        const bool in = (member >> r & 1) != 0;
        if (in && n > 0) {
            const size_t t = (size_t)row(u0 + r);
            load_v<T, kV>(static_cast<const T*>(a.g) + t * a.ld_g + c, n, gv);
            load_v<T, kV>(static_cast<const T*>(a.x) + t * a.ld_x + c, n, xv);
            if (kBack) {
                load_v<T, kV>(static_cast<const T*>(a.dy) + t * a.ld_dy + c, n, dv);
                if (!(final >> r & 1)) load_v<T, kV>(static_cast<const T*>(a.y) + (t - 1) * a.ld_y + c, n, hv);
            }
        }
        if (kBack && (final >> r & 1) && a.h0) {
            const int q = __shfl_sync(0xffffffffu, seq, r);
#pragma unroll
            for (int i = 0; i < kV; ++i)
                if (i < n) hv[i] = a.h0[(size_t)q * a.D + c + i];
        }
        // the state in front of a sequence goes into its first row's input: read once, since `after` may be `before`
        float init[kV];
#pragma unroll
        for (int i = 0; i < kV; ++i) init[i] = 0.f;
        if ((first >> r & 1) && a.before) {
            const int q = __shfl_sync(0xffffffffu, seq, r);
#pragma unroll
            for (int i = 0; i < kV; ++i)
                if (i < n) init[i] = a.before[(size_t)q * a.D + c + i];
        }
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            float k, z;
            gate_of(gv[i], k, z, T());
            keep[r][i] = in ? k : 1.f;
            if (kBack) {
                feed[r][i] = dv[i] + init[i];
                rest[r % (kBack ? kRows : 1)][i] = z;
                other[r % (kBack ? kRows : 1)][i] = kKind == ABS_RECURRENCE_BLEND ? hv[i] - xv[i] : hv[i];
            } else {
                feed[r][i] = !in ? 0.f : kKind == ABS_RECURRENCE_BLEND ? xv[i] * z : xv[i];
                if (first >> r & 1) feed[r][i] = fmaf(k, init[i], feed[r][i]);
            }
        }
    }
    // ---- the warp's map, then what is in front of the warp within the tile
    float A[kV], B[kV];
#pragma unroll
    for (int i = 0; i < kV; ++i) {
        A[i] = 1.f;
        B[i] = 0.f;
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        if (first >> r & 1)
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                A[i] = -0.f;
                B[i] = 0.f;
            }
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            B[i] = kBack ? keep[r][i] * (B[i] + feed[r][i]) : fmaf(keep[r][i], B[i], feed[r][i]);
            A[i] *= keep[r][i];
        }
    }
#pragma unroll
    for (int i = 0; i < kV; ++i) sh_map[warp][lane * kV + i] = make_float2(A[i], B[i]);
    __syncthreads();
    float s[kV];                                         // state in front of the tile
#pragma unroll
    for (int i = 0; i < kV; ++i) s[i] = 0.f;
    if (a.tiles > 1) {
        constexpr int kCols = 32 * kV;
        uint32_t* flags = a.ctl + 1;
        if (warp == 0) {
            const bool closes = tile % kGroup == kGroup - 1;
            float P[kV], Q[kV];
#pragma unroll
            for (int i = 0; i < kV; ++i) {
                P[i] = 1.f;
                Q[i] = 0.f;
            }
#pragma unroll
            for (int w = 0; w < kWarps; ++w)
#pragma unroll
                for (int i = 0; i < kV; ++i) {
                    const float2 m = sh_map[w][lane * kV + i];
                    compose(P[i], Q[i], m.x, m.y);
                }
            auto publish = [&]() {
                float2* p = a.maps + ((size_t)tile * a.strips + strip) * kCols + lane * kV;
#pragma unroll
                for (int i = 0; i < kV; ++i) p[i] = make_float2(P[i], Q[i]);
                __threadfence();
                __syncwarp();
                if (lane == 0) asm volatile("st.release.gpu.global.u32 [%0], %1;" ::"l"(flags + (size_t)tile * a.strips + strip), "r"(1u) : "memory");
            };
            if (!closes) publish();
            // the state behind the last group, then the maps of the tiles since, in order
            const int from = max(tile / kGroup * kGroup - 1, 0), count = tile - from;
            bool ok = true;
            if (lane < count) {
                const uint32_t* f = flags + (size_t)(from + lane) * a.strips + strip;
                uint32_t seen = 0, it = 0;
                while (it++ < kSpinLimit) {
                    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(f) : "memory");
                    if (seen) break;
                }
                ok = seen != 0;
            }
            ok = __all_sync(0xffffffffu, ok);
            if (ok) {
                for (int k = 0; k < count; ++k) {
                    const float2* p = a.maps + ((size_t)(from + k) * a.strips + strip) * kCols + lane * kV;
#pragma unroll
                    for (int i = 0; i < kV; ++i) {
                        const float2 m = __ldcg(p + i);
                        s[i] = apply(m.x, m.y, s[i]);
                    }
                }
                if (closes) {
#pragma unroll
                    for (int i = 0; i < kV; ++i) {
                        Q[i] = apply(P[i], Q[i], s[i]);
                        P[i] = -0.f;
                    }
                    publish();
                }
            } else if (lane == 0) {
                report_timeout();
                sh_ok = 0;
            }
#pragma unroll
            for (int i = 0; i < kV; ++i) sh_state[lane * kV + i] = s[i];
        }
        __syncthreads();
        if (!sh_ok) return;
#pragma unroll
        for (int i = 0; i < kV; ++i) s[i] = sh_state[lane * kV + i];
    }
    for (int w = 0; w < warp; ++w)
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            const float2 m = sh_map[w][lane * kV + i];
            s[i] = apply(m.x, m.y, s[i]);
        }
    // ---- the rows from their state
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        if (first >> r & 1)
#pragma unroll
            for (int i = 0; i < kV; ++i) s[i] = 0.f;
        const bool in = (member >> r & 1) != 0;
        float o[kV], o2[kV];
#pragma unroll
        for (int i = 0; i < kV; ++i) {
            if (kBack) {
                const float d = s[i] + feed[r][i], z = rest[r % (kBack ? kRows : 1)][i];
                s[i] = keep[r][i] * d;
                o[i] = kKind == ABS_RECURRENCE_BLEND ? z * d : d;
                o2[i] = s[i] * z * other[r % (kBack ? kRows : 1)][i];
            } else {
                s[i] = fmaf(keep[r][i], s[i], feed[r][i]);
                o[i] = s[i];
            }
            if (!in) o[i] = o2[i] = 0.f;
        }
        if (n > 0 && u0 + r < a.T) {
            const size_t t = (size_t)row(u0 + r);
            store_v<T, kV>(static_cast<T*>(a.out) + t * a.ld_out + c, n, o);
            if (kBack) store_v<T, kV>(static_cast<T*>(a.out2) + t * a.ld_out2 + c, n, o2);
        }
        if ((final >> r & 1) && a.after) {
            const int q = __shfl_sync(0xffffffffu, seq, r);
#pragma unroll
            for (int i = 0; i < kV; ++i)
                if (i < n) a.after[(size_t)q * a.D + c + i] = s[i];
        }
    }
    // ---- sequences without rows
    if (tile == 0 && a.after && (a.T == 0 || a.offsets))
        for (int q = warp; q < a.seqs; q += kWarps)
            if (begin_of(a, q + 1) <= begin_of(a, q))
#pragma unroll
                for (int i = 0; i < kV; ++i)
                    if (i < n) a.after[(size_t)q * a.D + c + i] = a.before ? a.before[(size_t)q * a.D + c + i] : 0.f;
}

template <typename T, uint32_t kKind>
__global__ void __launch_bounds__(256) k_recurrence_step(const T* x, size_t ld_x, const T* g, size_t ld_g, const float* h, size_t rows, int D, T* y, size_t ld_y,
                                                         float* out) {
    pdl_wait();
    pdl_trigger();
    for (size_t t = blockIdx.y; t < rows; t += gridDim.y) {
        const int c = blockIdx.x * 256 + threadIdx.x;
        if (c >= D) return;
        float a, z;
        gate_of(to_f(g[t * ld_g + c]), a, z, T());
        const float v = to_f(x[t * ld_x + c]), s = fmaf(a, h[t * D + c], kKind == ABS_RECURRENCE_BLEND ? z * v : v);
        out[t * D + c] = s;
        y[t * ld_y + c] = from_f<T>(s);
    }
}

size_t flags_bytes(uint64_t tiles, uint64_t strips) { return up256((1 + tiles * strips) * 4); }

template <typename T, int kV, uint32_t kKind>
cudaError_t run_tiles(const RecArgs& a, bool back, cudaStream_t s) {
    return launch_kernel(back ? k_recurrence<T, kV, kKind, true> : k_recurrence<T, kV, kKind, false>, dim3((unsigned)(a.tiles * a.strips)), kWarps * 32, 0, s, a.tiles == 1, a);
}
template <typename T>
cudaError_t run(const RecArgs& a, uint32_t kind, bool back, bool pairs, cudaStream_t s) {
    if (kind == ABS_RECURRENCE_BLEND) return pairs ? run_tiles<T, 2, ABS_RECURRENCE_BLEND>(a, back, s) : run_tiles<T, 1, ABS_RECURRENCE_BLEND>(a, back, s);
    return pairs ? run_tiles<T, 2, ABS_RECURRENCE_ADD>(a, back, s) : run_tiles<T, 1, ABS_RECURRENCE_ADD>(a, back, s);
}

const char* check_sizes(uint64_t tokens, uint64_t width, uint64_t seqs, uint32_t kind, uint32_t dtype, int* code) {
    *code = ABS_EINVAL;
    if (!known_dtype(dtype)) return "dtype must be ABS_F32 or ABS_BF16";
    if (kind > ABS_RECURRENCE_ADD) return "unknown kind of recurrence";
    if (width == 0) return "width must be at least 1";
    if (tokens <= kSizeMax && width <= kSizeMax && seqs <= kSizeMax && ((tokens + kTile - 1) / kTile) * ((width + 31) / 32) <= kSizeMax) return nullptr;
    *code = ABS_ELIMIT;
    return "a size exceeds 2^31 - 1024, or there are too many tiles of 128 rows and 32 columns";
}

// tokens > 0: `mats` are the matrices that the vector form depends on.
template <int N>
int launch_scan(RecArgs& a, const MatrixArg (&mats)[N], uint32_t kind, uint32_t dtype, bool back, void* workspace, size_t workspace_bytes, cudaStream_t s) {
    bool pairs = true;
    for (const MatrixArg& m : mats) pairs = pairs && rows_at(m, 2 * m.es);
    a.tiles = std::max(1, (a.T + kTile - 1) / kTile);
    a.strips = (a.D + (pairs ? 63 : 31)) / (pairs ? 64 : 32);
    cudaError_t e = cudaSuccess;
    if (a.tiles > 1) {
        if (!workspace || misaligned(workspace, 256)) return thread_error(ABS_EINVAL, "workspace must be non-NULL and 256-byte aligned");
        if (workspace_bytes < abs_recurrence_workspace((uint64_t)a.T, (uint64_t)a.D)) return thread_error(ABS_ENOMEM, "workspace too small");
        const size_t flags = flags_bytes(a.tiles, a.strips);
        a.ctl = static_cast<uint32_t*>(workspace);
        a.maps = reinterpret_cast<float2*>(static_cast<char*>(workspace) + flags);
        e = cudaMemsetAsync(workspace, 0, flags, s);
    }
    if (e == cudaSuccess) e = dtype == ABS_F32 ? run<float>(a, kind, back, pairs, s) : run<bf16>(a, kind, back, pairs, s);
    return e == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(e));
}

}  // namespace

cudaError_t take_status_recurrence(int* status, cudaStream_t s) { return take_status(status, s); }

}  // namespace abs_sgd

using namespace abs_sgd;

extern "C" size_t abs_recurrence_workspace(uint64_t tokens, uint64_t width) {
    if (tokens > kSizeMax || width > kSizeMax) return 0;
    const uint64_t tiles = (tokens + kTile - 1) / kTile, strips = (width + 31) / 32;
    return tiles > 1 ? flags_bytes(tiles, strips) + tiles * (strips + 1) * 32 * sizeof(float2) : 0;
}

extern "C" int abs_recurrence(const void* x, uint64_t ld_x, const void* g, uint64_t ld_g, const int32_t* offsets, uint64_t seqs, const float* h0, uint32_t kind,
                              uint32_t dtype, uint64_t tokens, uint64_t width, void* y, uint64_t ld_y, float* last, void* workspace, size_t workspace_bytes,
                              void* stream) {
    int code = 0;
    if (const char* why = check_sizes(tokens, width, seqs, kind, dtype, &code)) return thread_error(code, why);
    const size_t es = size_of(dtype);
    const MatrixArg m[3] = {{x, ld_x, width, es}, {g, ld_g, width, es}, {y, ld_y, width, es}};
    if (const char* why = check_matrices(m)) return thread_error(ABS_EINVAL, why);
    for (int i = 0; i < 2; ++i)
        if (const char* why = check_in_place(m[2], m[i], true)) return thread_error(ABS_EINVAL, why);
    if (!offsets && seqs != 1) return thread_error(ABS_EINVAL, "without offsets there is one sequence");
    if (misaligned(offsets, 4) || misaligned(h0, 4) || misaligned(last, 4)) return thread_error(ABS_EINVAL, "offsets, h0 and last must be 4-byte aligned");
    if (tokens && (!x || !g || !y)) return thread_error(ABS_EINVAL, "x, g and y must not be NULL");
    if (tokens == 0 && (!last || seqs == 0)) return ABS_OK;
    RecArgs a{};
    a.x = x; a.ld_x = ld_x; a.g = g; a.ld_g = ld_g; a.out = y; a.ld_out = ld_y;
    a.offsets = offsets; a.before = h0; a.after = last; a.T = (int)tokens; a.D = (int)width; a.seqs = (int)seqs;
    return launch_scan(a, m, kind, dtype, false, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
}

extern "C" int abs_recurrence_backward(const void* dy, uint64_t ld_dy, const void* x, uint64_t ld_x, const void* g, uint64_t ld_g, const void* y, uint64_t ld_y,
                                       const int32_t* offsets, uint64_t seqs, const float* h0, const float* dlast, uint32_t kind, uint32_t dtype, uint64_t tokens,
                                       uint64_t width, void* dx, uint64_t ld_dx, void* dg, uint64_t ld_dg, float* dh0, void* workspace, size_t workspace_bytes,
                                       void* stream) {
    int code = 0;
    if (const char* why = check_sizes(tokens, width, seqs, kind, dtype, &code)) return thread_error(code, why);
    const size_t es = size_of(dtype);
    const MatrixArg m[6] = {{dy, ld_dy, width, es}, {x, ld_x, width, es}, {g, ld_g, width, es}, {y, ld_y, width, es}, {dx, ld_dx, width, es}, {dg, ld_dg, width, es}};
    if (const char* why = check_matrices(m)) return thread_error(ABS_EINVAL, why);
    for (int o = 4; o < 6; ++o)
        for (int i = 0; i < 4; ++i)
            if (const char* why = check_in_place(m[o], m[i], i < 3)) return thread_error(ABS_EINVAL, why);
    if (!offsets && seqs != 1) return thread_error(ABS_EINVAL, "without offsets there is one sequence");
    if (misaligned(offsets, 4) || misaligned(h0, 4) || misaligned(dlast, 4) || misaligned(dh0, 4))
        return thread_error(ABS_EINVAL, "offsets, h0, dlast and dh0 must be 4-byte aligned");
    if (tokens && (!dy || !x || !g || !y || !dx || !dg)) return thread_error(ABS_EINVAL, "dy, x, g, y, dx and dg must not be NULL");
    if (tokens && dx == dg) return thread_error(ABS_EINVAL, "two outputs are the same");
    if (dh0 && dh0 == h0) return thread_error(ABS_EINVAL, "dh0 must not be h0");
    if (tokens == 0 && (!dh0 || seqs == 0)) return ABS_OK;
    RecArgs a{};
    a.x = x; a.ld_x = ld_x; a.g = g; a.ld_g = ld_g; a.dy = dy; a.ld_dy = ld_dy; a.y = y; a.ld_y = ld_y;
    a.out = dx; a.ld_out = ld_dx; a.out2 = dg; a.ld_out2 = ld_dg;
    a.offsets = offsets; a.h0 = h0; a.before = dlast; a.after = dh0; a.T = (int)tokens; a.D = (int)width; a.seqs = (int)seqs;
    return launch_scan(a, m, kind, dtype, true, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
}

extern "C" int abs_recurrence_step(const void* x, uint64_t ld_x, const void* g, uint64_t ld_g, const float* h, uint32_t kind, uint32_t dtype, uint64_t seqs,
                                   uint64_t width, void* y, uint64_t ld_y, float* out, void* stream) {
    int code = 0;
    if (const char* why = check_sizes(0, width, seqs, kind, dtype, &code)) return thread_error(code, why);
    const size_t es = size_of(dtype);
    const MatrixArg m[3] = {{x, ld_x, width, es}, {g, ld_g, width, es}, {y, ld_y, width, es}};
    if (const char* why = check_matrices(m)) return thread_error(ABS_EINVAL, why);
    for (int i = 0; i < 2; ++i)
        if (const char* why = check_in_place(m[2], m[i], true)) return thread_error(ABS_EINVAL, why);
    if (misaligned(h, 4) || misaligned(out, 4)) return thread_error(ABS_EINVAL, "h and out must be 4-byte aligned");
    if (seqs == 0) return ABS_OK;
    if (!x || !g || !h || !y || !out) return thread_error(ABS_EINVAL, "x, g, h, y and out must not be NULL");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const dim3 grid((unsigned)((width + 255) / 256), (unsigned)std::min<uint64_t>(seqs, 32768));
    auto go = [&](auto kernel, auto zero) {
        using T = decltype(zero);
        return launch_kernel(kernel, grid, 256, 0, s, true, static_cast<const T*>(x), (size_t)ld_x, static_cast<const T*>(g), (size_t)ld_g, h, (size_t)seqs, (int)width,
                             static_cast<T*>(y), (size_t)ld_y, out);
    };
    const bool blend = kind == ABS_RECURRENCE_BLEND;
    const cudaError_t e = dtype == ABS_F32 ? (blend ? go(k_recurrence_step<float, ABS_RECURRENCE_BLEND>, 0.f) : go(k_recurrence_step<float, ABS_RECURRENCE_ADD>, 0.f))
                                           : (blend ? go(k_recurrence_step<bf16, ABS_RECURRENCE_BLEND>, bf16()) : go(k_recurrence_step<bf16, ABS_RECURRENCE_ADD>, bf16()));
    return e == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(e));
}
