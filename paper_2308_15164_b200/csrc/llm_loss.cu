// Losses of a language model on its logits, with the gradient of the logits (abs_policy_loss, abs_preference_loss).
//
// Both need, for every row z of the logits, M = max_v z_v and S = sum_v exp(z_v - M): then logp(y) = z_y - M - log S and
// softmax_v = exp(z_v - M) / S.  Both losses depend on the logits through logp(y) alone, so that the gradient of a row is
// g ([v = y] - softmax_v) with one number g per row.  Per element: one comparison, two exponentials, a few additions --
// the work is bound by the memory the logits come from and the gradient goes to.
#include <math.h>

#include "abs_internal.h"
#include "abs_llm.h"
#include "row_ops.cuh"

namespace abs_sgd {
namespace {

constexpr int kStatCtasMax = 1024;   // CTAs that leave partial sums of the policy loss
constexpr float kLog2e = 1.4426950408889634f;

// exp(z - m): the difference is rounded once, the base-2 exponential takes the rest (relative error about 2e-7 where
// the result is not negligible beside exp(0)).  m is finite.
__device__ __forceinline__ float exp_diff(float z, float m) { return exp2f((z - m) * kLog2e); }

struct RowStat {
    float m, s;      // largest element; sum of exp(z - m).  m = -inf: no element is above -inf
};

template <int G>
__device__ __forceinline__ RowStat group_stat(RowStat a, float* sh) {
    float m = a.m;
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (G > 32) {
        constexpr int kWarps = G / 32;
        const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
        __syncthreads();
        if (lane == 0) sh[warp] = m;
        __syncthreads();
        m = lane < kWarps ? sh[lane] : -INFINITY;
#pragma unroll
        for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    }
    float v[1] = {a.m == -INFINITY ? a.s : a.s * exp_diff(a.m, m)};   // a.s is 0 there, or NaN from NaN elements
    group_sum<G, 1>(v, sh);
    return RowStat{m, v[0]};
}

// Adds N elements to a thread's running maximum and sum.  Elements of -inf add nothing, NaN makes the sum NaN.
template <int N>
__device__ __forceinline__ void stat_add(RowStat& a, const float (&z)[N]) {
    float m = z[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = fmaxf(m, z[i]);
    if (m > a.m) {
        a.s = a.m == -INFINITY ? a.s : a.s * exp_diff(a.m, m);
        a.m = m;
    }
    const float ref = a.m == -INFINITY ? 0.f : a.m;
#pragma unroll
    for (int i = 0; i < N; ++i) a.s += exp_diff(z[i], ref);
}

template <typename T, int G>
__device__ __forceinline__ RowStat row_stat(const T* row, int V, int tid, float* sh) {
    const RowCut c = cut_row(row, V);
    RowStat a{-INFINITY, 0.f};
    for (int i = tid; i < c.pieces; i += G) {
        float z[kVec<T>];
        Pack<T, kVec<T>>::load(row + c.head + i * kVec<T>, z);
        stat_add(a, z);
    }
    if (tid < c.head + c.tail) {
        float z[1] = {to_f(row[tid < c.head ? tid : V - c.tail + (tid - c.head)])};
        stat_add(a, z);
    }
    return group_stat<G>(a, sh);
}

// One row of the gradient, g ([v = y] - exp(z_v - m) / s), or zeros.  out may be the row itself.
template <typename T, int G>
__device__ __forceinline__ void row_grad(const T* row, T* out, int V, int y, float g, RowStat st, int tid) {
    const float c = -g / st.s;
    const bool zero = g == 0.f;
    const RowCut o = cut_row(out, V);
    const bool same = cut_row(row, V).head == o.head;    // the pieces of row and out are aligned alike
    auto one = [&](int v) {
        float d = zero ? 0.f : exp_diff(to_f(row[v]), st.m) * c;
        if (v == y) d += g;
        out[v] = from_f<T>(d);
    };
    if (same || zero) {
        for (int i = tid; i < o.pieces; i += G) {
            const int v0 = o.head + i * kVec<T>;
            float z[kVec<T>];
            if (zero) {
#pragma unroll
                for (int k = 0; k < kVec<T>; ++k) z[k] = 0.f;
            } else {
                Pack<T, kVec<T>>::load(row + v0, z);
#pragma unroll
                for (int k = 0; k < kVec<T>; ++k) z[k] = exp_diff(z[k], st.m) * c + (v0 + k == y ? g : 0.f);
            }
            Pack<T, kVec<T>>::store(out + v0, z);
        }
        if (tid < o.head + o.tail) one(tid < o.head ? tid : V - o.tail + (tid - o.head));
    } else {
        for (int v = tid; v < V; v += G) one(v);
    }
}

struct PolicyArgs {
    const void* logits;
    void* dlogits;
    size_t ld, ld_d, T;
    int V;
    const int32_t* labels;
    const float *logp_old, *logp_ref, *adv, *weight;
    float clip_low, clip_high, kl_coef;
    float* logp;
    double* part;      // [CTA][3]
};

struct TokenLoss {
    float loss, kl, clipped, slope;   // slope: d loss / d logp; all without the token's weight
};
__device__ __forceinline__ TokenLoss token_loss(const PolicyArgs& a, size_t t, float logp) {
    TokenLoss r{0.f, 0.f, 0.f, 0.f};
    const float A = a.adv[t];
    if (A != 0.f) {      // the term is 0 there whatever the ratio is (exp may overflow for a token that counts for nothing)
        const float ratio = expf(logp - a.logp_old[t]);
        const bool up = A > 0.f && ratio > 1.f + a.clip_high, down = A < 0.f && ratio < 1.f - a.clip_low;
        r.loss = -(up ? 1.f + a.clip_high : down ? 1.f - a.clip_low : ratio) * A;
        r.slope = up || down ? 0.f : -ratio * A;
        r.clipped = up || down ? 1.f : 0.f;
    }
    if (a.logp_ref) {
        const float d = a.logp_ref[t] - logp, e = expm1f(d);
        r.kl = e - d;
        r.loss += a.kl_coef * r.kl;
        r.slope -= a.kl_coef * e;
    }
    return r;
}

// One group of G threads per row at a time, kGroups rows per CTA.
template <typename T, int G, int kGroups>
__global__ void __launch_bounds__(G * kGroups) k_policy_rows(PolicyArgs a) {
    static_assert(G == 32 || kGroups == 1, "a group is a warp or the whole CTA");
    __shared__ float sh[32];
    __shared__ double acc[kGroups][3];
    const int group = threadIdx.x / G, tid = threadIdx.x % G;
    pdl_wait();
    pdl_trigger();
    if (tid < 3) acc[group][tid] = 0.0;
    if (G == 32) __syncwarp();
    for (size_t t = (size_t)blockIdx.x * kGroups + group; t < a.T; t += (size_t)gridDim.x * kGroups) {
        const T* row = static_cast<const T*>(a.logits) + t * a.ld;
        const int y = a.labels[t];
        const float w = a.weight[t];
        RowStat st{0.f, 1.f};
        float g = 0.f, logp = 0.f;
        if (w != 0.f && y >= 0 && y < a.V) {
            const float zy = to_f(row[y]);
            st = row_stat<T, G>(row, a.V, tid, sh);
            if (st.m != -INFINITY || st.s != 0.f) {
                logp = zy - st.m - logf(st.s);
                const TokenLoss l = token_loss(a, t, logp);
                g = w * l.slope;
                if (tid == 0) {
                    acc[group][0] += (double)w * l.loss;
                    acc[group][1] += (double)w * l.kl;
                    acc[group][2] += (double)w * l.clipped;
                }
            }
        }
        if (tid == 0) a.logp[t] = logp;
        if (a.dlogits) {
            if (G > 32) __syncthreads();      // in place: zy has been read by everybody
            row_grad<T, G>(row, static_cast<T*>(a.dlogits) + t * a.ld_d, a.V, y, g, st, tid);
        }
    }
    __syncthreads();
    if (threadIdx.x < 3) {
        double s = 0.0;
        for (int k = 0; k < kGroups; ++k) s += acc[k][threadIdx.x];
        a.part[(size_t)blockIdx.x * 3 + threadIdx.x] = s;
    }
}

// stats[k] = sum over the CTAs of part[cta][k], one warp each.
__global__ void __launch_bounds__(96) k_policy_stats(const double* part, int n, float* stats) {
    const int k = threadIdx.x / 32, lane = threadIdx.x % 32;
    pdl_wait();
    pdl_trigger();
    double s = 0.0;
    for (int i = lane; i < n; i += 32) s += part[(size_t)i * 3 + k];
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane == 0) stats[k] = (float)s;
}

struct PrefArgs {
    const void* logits;
    void* dlogits;
    size_t ld, ld_d, T, pairs;
    int V;
    const int32_t *labels, *offsets;
    const float* logp_ref;
    float beta, smoothing, scale;
    float *stats, *pair_loss, *seq_logp;
    float *m, *s, *logp, *g;     // workspace, [T] each
};

template <typename T, int G, int kGroups>
__global__ void __launch_bounds__(G * kGroups) k_pref_stats(PrefArgs a) {
    __shared__ float sh[32];
    const int group = threadIdx.x / G, tid = threadIdx.x % G;
    pdl_wait();
    pdl_trigger();
    for (size_t t = (size_t)blockIdx.x * kGroups + group; t < a.T; t += (size_t)gridDim.x * kGroups) {
        const T* row = static_cast<const T*>(a.logits) + t * a.ld;
        const int y = a.labels[t];
        RowStat st{-INFINITY, 0.f};
        float logp = 0.f;
        if (y >= 0 && y < a.V) {
            const float zy = to_f(row[y]);
            st = row_stat<T, G>(row, a.V, tid, sh);
            if (st.m != -INFINITY || st.s != 0.f) logp = zy - st.m - logf(st.s);
        }
        if (tid == 0) {
            a.m[t] = st.m;
            a.s[t] = st.s;
            a.logp[t] = logp;
            a.g[t] = 0.f;
        }
    }
}

// One CTA per pair at a time: the two sums, the loss, and g of every counted row.
__global__ void __launch_bounds__(256) k_pref_pairs(PrefArgs a) {
    __shared__ double sh[8];
    __shared__ double total[2];
    pdl_wait();
    pdl_trigger();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const long long T = (long long)a.T;
    for (size_t p = blockIdx.x; p < a.pairs; p += gridDim.x) {
        long long at[3];
        for (int k = 0; k < 3; ++k) at[k] = min(max((long long)a.offsets[2 * p + k], 0ll), T);
        for (int k = 0; k < 2; ++k) {
            double s = 0.0;
            for (long long t = at[k] + threadIdx.x; t < at[k + 1]; t += 256) s += (double)a.logp[t];
#pragma unroll
            for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            __syncthreads();
            if (lane == 0) sh[warp] = s;
            __syncthreads();
            if (threadIdx.x == 0) {
                for (int i = 1; i < 8; ++i) s += sh[i];
                total[k] = s;
                a.seq_logp[2 * p + k] = (float)s;
            }
        }
        __syncthreads();
        const double h = (double)a.beta * ((total[0] - (double)a.logp_ref[2 * p]) - (total[1] - (double)a.logp_ref[2 * p + 1]));
        const double e = exp(-fabs(h)), soft = log1p(e);                     // -log sigmoid(+-h) = soft + max(-+h, 0)
        const double sig = h >= 0.0 ? 1.0 / (1.0 + e) : e / (1.0 + e);
        if (threadIdx.x == 0)
            a.pair_loss[p] = (float)((1.0 - (double)a.smoothing) * (soft + fmax(-h, 0.0)) + (double)a.smoothing * (soft + fmax(h, 0.0)) + 0.0 * h);
        const float g = (float)((double)a.scale * (double)a.beta * (sig - (1.0 - (double)a.smoothing)));
        for (int k = 0; k < 2; ++k)
            for (long long t = at[k] + threadIdx.x; t < at[k + 1]; t += 256)
                a.g[t] = a.m[t] == -INFINITY && a.s[t] == 0.f ? 0.f : k ? -g : g;
        __syncthreads();
    }
}

// The gradient of the rows; CTA 0 also adds up the loss.
template <typename T, int G, int kGroups>
__global__ void __launch_bounds__(G * kGroups) k_pref_grad(PrefArgs a) {
    const int group = threadIdx.x / G, tid = threadIdx.x % G;
    pdl_wait();
    pdl_trigger();
    if (a.dlogits)
        for (size_t t = (size_t)blockIdx.x * kGroups + group; t < a.T; t += (size_t)gridDim.x * kGroups) {
            const float g = a.g[t];
            row_grad<T, G>(static_cast<const T*>(a.logits) + t * a.ld, static_cast<T*>(a.dlogits) + t * a.ld_d, a.V,
                           g == 0.f ? -1 : a.labels[t], g, RowStat{a.m[t], a.s[t]}, tid);
        }
    if (blockIdx.x == 0 && threadIdx.x < 32) {
        double s = 0.0;
        for (size_t p = threadIdx.x; p < a.pairs; p += 32) s += (double)a.pair_loss[p];
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (threadIdx.x == 0) a.stats[0] = (float)(s * (double)a.scale);
    }
}

constexpr int kWarpRowMax = 1024;    // rows up to this length are taken by one warp each

int current_sms() {
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    return sms;
}

template <typename T>
cudaError_t launch_policy(const PolicyArgs& a, float* stats, int sms, cudaStream_t s) {
    const bool warp_rows = a.V <= kWarpRowMax;
    const size_t want = warp_rows ? (a.T + 7) / 8 : a.T;
    const int grid = (int)(want < (size_t)(4 * sms) ? want : (size_t)(4 * sms));
    cudaError_t e = cudaSuccess;
    if (grid > 0)
        e = warp_rows ? launch_kernel(k_policy_rows<T, 32, 8>, grid, 256, 0, s, true, a)
                      : launch_kernel(k_policy_rows<T, 512, 1>, grid, 512, 0, s, true, a);
    if (e != cudaSuccess) return e;
    return launch_kernel(k_policy_stats, 1, 96, 0, s, true, (const double*)a.part, grid, stats);
}

template <typename T>
cudaError_t launch_pref(const PrefArgs& a, int sms, cudaStream_t s) {
    const bool warp_rows = a.V <= kWarpRowMax;
    const size_t want = warp_rows ? (a.T + 7) / 8 : a.T;
    const int grid = (int)(want < (size_t)(4 * sms) ? want : (size_t)(4 * sms));
    cudaError_t e = cudaSuccess;
    if (grid > 0)
        e = warp_rows ? launch_kernel(k_pref_stats<T, 32, 8>, grid, 256, 0, s, true, a)
                      : launch_kernel(k_pref_stats<T, 512, 1>, grid, 512, 0, s, true, a);
    if (e != cudaSuccess) return e;
    if (a.pairs > 0) {
        e = launch_kernel(k_pref_pairs, (int)(a.pairs < (size_t)sms ? a.pairs : (size_t)sms), 256, 0, s, true, a);
        if (e != cudaSuccess) return e;
    }
    const int g2 = a.dlogits && grid > 0 ? grid : 1;
    return warp_rows ? launch_kernel(k_pref_grad<T, 32, 8>, g2, 256, 0, s, true, a)
                     : launch_kernel(k_pref_grad<T, 512, 1>, g2, 512, 0, s, true, a);
}

bool misaligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// What the two losses ask of logits, labels and dlogits; nullptr if all is well.
const char* check_logits(const void* logits, uint32_t dtype, uint64_t T, uint64_t V, uint64_t ld, const int32_t* labels,
                         const void* dlogits, uint64_t ld_d) {
    if (dtype != ABS_F32 && dtype != ABS_BF16) return "dtype must be ABS_F32 or ABS_BF16";
    const size_t es = dtype == ABS_F32 ? 4 : 2;
    if (V == 0) return "vocab must be at least 1";
    if (ld < V || (dlogits && ld_d < V)) return "a leading dimension is shorter than the row";
    if (T && (!logits || !labels)) return "logits and labels must not be NULL";
    if (misaligned(logits, es) || misaligned(dlogits, es) || misaligned(labels, 4)) return "a pointer is not aligned to its elements";
    if (dlogits && dlogits == logits && ld_d != ld) return "dlogits in place of the logits needs the same leading dimension";
    return nullptr;
}

size_t up256(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace
}  // namespace abs_sgd

using namespace abs_sgd;

extern "C" size_t abs_policy_loss_workspace(void) { return up256(sizeof(double) * 3 * kStatCtasMax); }

extern "C" int abs_policy_loss(const void* logits, uint32_t dtype, uint64_t tokens, uint64_t vocab, uint64_t ld, const int32_t* labels,
                               const float* logp_old, const float* logp_ref, const float* advantage, const float* weight,
                               float clip_low, float clip_high, float kl_coef, float* stats, float* logp, void* dlogits,
                               uint64_t ld_d, void* workspace, size_t workspace_bytes, void* stream) {
    if (const char* why = check_logits(logits, dtype, tokens, vocab, ld, labels, dlogits, ld_d)) return thread_error(ABS_EINVAL, why);
    if (vocab > 0x7fffffffull) return thread_error(ABS_ELIMIT, "vocab exceeds 2^31 - 1");
    if (tokens && (!logp_old || !advantage || !weight || !logp)) return thread_error(ABS_EINVAL, "a per-token array is NULL");
    if (!stats) return thread_error(ABS_EINVAL, "stats must not be NULL");
    if (misaligned(logp_old, 4) || misaligned(logp_ref, 4) || misaligned(advantage, 4) || misaligned(weight, 4) || misaligned(stats, 4) || misaligned(logp, 4))
        return thread_error(ABS_EINVAL, "a per-token array is not 4-byte aligned");
    if (!(clip_low >= 0.f) || !(clip_high >= 0.f) || !isfinite(kl_coef)) return thread_error(ABS_EINVAL, "clip_low, clip_high must be >= 0 and kl_coef finite");
    if (!logp_ref && kl_coef != 0.f) return thread_error(ABS_EINVAL, "kl_coef without logp_ref");
    if (!workspace || misaligned(workspace, 256)) return thread_error(ABS_EINVAL, "workspace must be non-NULL and 256-byte aligned");
    if (workspace_bytes < abs_policy_loss_workspace()) return thread_error(ABS_ENOMEM, "workspace too small");
    const int sms = current_sms();
    if (!sms) return thread_error(ABS_ECUDA, "no current CUDA device");
    PolicyArgs a{};
    a.logits = logits; a.dlogits = dlogits; a.ld = ld; a.ld_d = ld_d; a.T = tokens; a.V = (int)vocab;
    a.labels = labels; a.logp_old = logp_old; a.logp_ref = logp_ref; a.adv = advantage; a.weight = weight;
    a.clip_low = clip_low; a.clip_high = clip_high; a.kl_coef = kl_coef; a.logp = logp;
    a.part = static_cast<double*>(workspace);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == ABS_F32 ? launch_policy<float>(a, stats, sms, s) : launch_policy<bf16>(a, stats, sms, s);
    return e == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(e));
}

extern "C" size_t abs_preference_loss_workspace(uint64_t tokens) { return 4 * up256(tokens * 4) + 256; }

extern "C" int abs_preference_loss(const void* logits, uint32_t dtype, uint64_t tokens, uint64_t vocab, uint64_t ld, const int32_t* labels,
                                   const int32_t* offsets, uint64_t pairs, const float* logp_ref, float beta, float smoothing,
                                   float scale, float* stats, float* pair_loss, float* seq_logp, void* dlogits, uint64_t ld_d,
                                   void* workspace, size_t workspace_bytes, void* stream) {
    if (const char* why = check_logits(logits, dtype, tokens, vocab, ld, labels, dlogits, ld_d)) return thread_error(ABS_EINVAL, why);
    if (vocab > 0x7fffffffull || tokens > 0x7fffffffull) return thread_error(ABS_ELIMIT, "vocab or tokens exceeds 2^31 - 1");
    if (pairs && (!offsets || !logp_ref || !pair_loss || !seq_logp)) return thread_error(ABS_EINVAL, "a per-pair array is NULL");
    if (!stats) return thread_error(ABS_EINVAL, "stats must not be NULL");
    if (misaligned(offsets, 4) || misaligned(logp_ref, 4) || misaligned(stats, 4) || misaligned(pair_loss, 4) || misaligned(seq_logp, 4))
        return thread_error(ABS_EINVAL, "a per-pair array is not 4-byte aligned");
    if (!isfinite(beta) || !isfinite(scale) || !(smoothing >= 0.f && smoothing <= 1.f)) return thread_error(ABS_EINVAL, "beta and scale must be finite, smoothing in [0, 1]");
    if (!workspace || misaligned(workspace, 256)) return thread_error(ABS_EINVAL, "workspace must be non-NULL and 256-byte aligned");
    if (workspace_bytes < abs_preference_loss_workspace(tokens)) return thread_error(ABS_ENOMEM, "workspace too small");
    const int sms = current_sms();
    if (!sms) return thread_error(ABS_ECUDA, "no current CUDA device");
    PrefArgs a{};
    a.logits = logits; a.dlogits = dlogits; a.ld = ld; a.ld_d = ld_d; a.T = tokens; a.pairs = pairs; a.V = (int)vocab;
    a.labels = labels; a.offsets = offsets; a.logp_ref = logp_ref; a.beta = beta; a.smoothing = smoothing; a.scale = scale;
    a.stats = stats; a.pair_loss = pair_loss; a.seq_logp = seq_logp;
    char* w = static_cast<char*>(workspace);
    const size_t step = up256(tokens * 4);
    a.m = reinterpret_cast<float*>(w);
    a.s = reinterpret_cast<float*>(w + step);
    a.logp = reinterpret_cast<float*>(w + 2 * step);
    a.g = reinterpret_cast<float*>(w + 3 * step);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dtype == ABS_F32 ? launch_pref<float>(a, sms, s) : launch_pref<bf16>(a, sms, s);
    return e == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(e));
}
