// Losses of a language model on its logits, with the gradient of the logits (abs_policy_loss, abs_preference_loss).
//
// Both need, for every row z of the logits, M = max_v z_v and S = sum_v exp(z_v - M): then logp(y) = z_y - M - log S and
// softmax_v = exp(z_v - M) / S.  Both losses depend on the logits through logp(y) alone, so that the gradient of a row is
// g ([v = y] - softmax_v) with one number g per row.  Per element: one comparison, two exponentials, a few additions --
// the work is bound by the memory the logits come from and the gradient goes to.
#include <math.h>

#include "abs_internal.h"
#include "abs_llm.h"
#include "bulk_copy.cuh"
#include "llm_status.cuh"
#include "row_ops.cuh"

namespace abs_sgd {
namespace {

constexpr int kStatCtasMax = 2048;   // CTAs that leave partial sums of the policy loss
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kHuge = 1073741824.f;      // 2^30

// exp(z - m) as 2^(a z - m2) with m2 = a m rounded, one fused multiply-add and the approximate base-2 unit (relative error
// about 2e-7 where the result is not negligible beside 1).  The rounding of m2 is common to all that is computed with one
// m, and a change of m is a factor 2^(m2 - m2'), so that it cancels in every quotient; a logarithm of such a sum is corrected
// for it (log_sum).  a = log2 e below 2^30, where half a unit in the last place of m2, the exponent of that common factor, is at
// most 64; from there on different z are 64 or more apart (128 in general), exp(z - m) is 1 or nothing beside it, and a = 1 gives that
// exactly where z = m.  m = -inf (nothing above -inf yet): a = 1, m2 = 0.
struct Base {
    float a, m2;
};
__device__ __forceinline__ Base base_of(float m) {
    const float a = fabsf(m) >= kHuge ? 1.f : kLog2e;
    return Base{a, m == -INFINITY ? 0.f : __fmul_rn(a, m)};      // rounded: not to be drawn into a fused multiply-add
}
__device__ __forceinline__ float exp_at(float z, Base b) { return exp2_of(fmaf(z, b.a, -b.m2)); }
__device__ __forceinline__ float2 exp_at(float2 z, Base b) { return exp2_of(fma2(z, both(b.a), both(-b.m2))); }

struct RowStat {
    float m, s;      // largest element; sum of exp(z - m).  m = -inf: no element is above -inf
};
// log sum exp(z - m).  s carries the factor 2^(a m - m2), up to half a unit in the last place of m2 (4e-4 in the logarithm at m = 5000);
// the product's rounding is exact by one fused multiply-add.
__device__ __forceinline__ float log_sum(RowStat a) {
    const Base b = base_of(a.m);
    return logf(a.s) - 0.693147180559945309f * fmaf(a.m, b.a, -b.m2);
}

// Maximum over a warp (NaN is left out).
__device__ __forceinline__ float warp_max(float v) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
// The factor that takes sums relative to the maximum `from` (above -inf) to those relative to `to` >= from.  Maxima on
// either side of kHuge are 64 or more apart: nothing is left.
__device__ __forceinline__ float rescale(float from, float to) {
    const Base f = base_of(from), t = base_of(to);
    return f.a == t.a ? exp2_of(f.m2 - t.m2) : 0.f;
}
// The sum of `a`, relative to a maximum m >= a.m (where a.m = -inf it is 0, or NaN from NaN elements).
__device__ __forceinline__ float at_max(RowStat a, float m) { return a.m == -INFINITY ? a.s : a.s * rescale(a.m, m); }

template <int G>
__device__ __forceinline__ RowStat group_stat(RowStat a, float* sh) {
    float m = warp_max(a.m);
    if (G > 32) {
        constexpr int kWarps = G / 32;
        const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
        __syncthreads();
        if (lane == 0) sh[warp] = m;
        __syncthreads();
        m = warp_max(lane < kWarps ? sh[lane] : -INFINITY);
    }
    float v[1] = {at_max(a, m)};
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
        a.s = at_max(a, m);
        a.m = m;
    }
    const Base b = base_of(a.m);
#pragma unroll
    for (int i = 0; i < N; ++i) a.s += exp_at(z[i], b);
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
    const Base b = base_of(st.m);
    const bool zero = g == 0.f;
    const RowCut o = cut_row(out, V);
    const bool same = cut_row(row, V).head == o.head;    // the pieces of row and out are aligned alike
    auto one = [&](int v) {
        float d = zero ? 0.f : exp_at(to_f(row[v]), b) * c;
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
                for (int k = 0; k < kVec<T>; ++k) z[k] = exp_at(z[k], b) * c + (v0 + k == y ? g : 0.f);
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
struct TokenIn {
    float adv, old, ref;
};
__device__ __forceinline__ TokenIn token_in(const PolicyArgs& a, size_t t) {
    return TokenIn{a.adv[t], a.logp_old[t], a.logp_ref ? a.logp_ref[t] : 0.f};
}
__device__ __forceinline__ TokenLoss token_loss(const PolicyArgs& a, TokenIn in, float logp) {
    TokenLoss r{0.f, 0.f, 0.f, 0.f};
    const float A = in.adv;
    if (A != 0.f) {      // the term is 0 there whatever the ratio is (exp may overflow for a token that counts for nothing)
        const float ratio = expf(logp - in.old);
        const bool up = A > 0.f && ratio > 1.f + a.clip_high, down = A < 0.f && ratio < 1.f - a.clip_low;
        r.loss = -(up ? 1.f + a.clip_high : down ? 1.f - a.clip_low : ratio) * A;
        r.slope = up || down ? 0.f : -ratio * A;
        r.clipped = up || down ? 1.f : 0.f;
    }
    if (a.logp_ref) {
        const float d = in.ref - logp, e = expm1f(d);
        r.kl = e - d;
        if (a.kl_coef != 0.f) {      // as above: e may be infinite where the term counts for nothing
            r.loss += a.kl_coef * r.kl;
            r.slope -= a.kl_coef * e;
        }
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
                logp = zy - st.m - log_sum(st);
                const TokenLoss l = token_loss(a, token_in(a, t), logp);
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

// One CTA per pair at a time: the two sums (half of the CTA each, in 64 bits), the loss, and g of every counted row.
__global__ void __launch_bounds__(1024) k_pref_pairs(PrefArgs a) {
    __shared__ double sh[32];
    __shared__ float slope;
    pdl_wait();
    pdl_trigger();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, half = threadIdx.x / 512, tid = threadIdx.x % 512;
    const int T = (int)a.T;
    for (size_t p = blockIdx.x; p < a.pairs; p += gridDim.x) {
        const int begin = min(max(a.offsets[2 * p + half], 0), T), end = min(max(a.offsets[2 * p + half + 1], 0), T);
        double s = 0.0;
        for (int t = begin + tid; t < end; t += 512) s += (double)a.logp[t];
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0) sh[warp] = s;
        __syncthreads();
        if (warp == 0) {
            // lanes 0 - 15: the preferred answer's warps, 16 - 31 the other's
            s = sh[lane];
#pragma unroll
            for (int o = 8; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            const double other = __shfl_sync(0xffffffffu, s, 16);
            if (lane == 0) {
                a.seq_logp[2 * p] = (float)s;
                a.seq_logp[2 * p + 1] = (float)other;
                // the difference in 64 bits, what comes after it in 32
                const float h = (float)((double)a.beta * ((s - (double)a.logp_ref[2 * p]) - (other - (double)a.logp_ref[2 * p + 1])));
                const float e = expf(-fabsf(h)), soft = log1pf(e);               // -log sigmoid(+-h) = soft + max(-+h, 0)
                const float tail = e / (1.f + e), head = 1.f / (1.f + e);         // sigmoid(-|h|), sigmoid(|h|)
                const float worse = h < 0.f ? -h : 0.f, better = h > 0.f ? h : 0.f;
                a.pair_loss[p] = h == h ? (1.f - a.smoothing) * (soft + worse) + a.smoothing * (soft + better) : h;
                // sigmoid(h) - (1 - smoothing) without the difference of nearly equal numbers that it is for a well separated pair
                slope = a.scale * a.beta * (a.smoothing * (h >= 0.f ? head : tail) - (1.f - a.smoothing) * (h >= 0.f ? tail : head));
            }
        }
        __syncthreads();
        const float g = half ? -slope : slope;
        for (int t = begin + tid; t < end; t += 512) a.g[t] = a.m[t] == -INFINITY && a.s[t] == 0.f ? 0.f : g;
        __syncthreads();
    }
}

// The loss over all pairs; one warp.
__device__ __forceinline__ void pref_total(const PrefArgs& a) {
    double s = 0.0;
    for (size_t p = threadIdx.x % 32; p < a.pairs; p += 32) s += (double)a.pair_loss[p];
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (threadIdx.x % 32 == 0) a.stats[0] = (float)(s * (double)a.scale);
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
    if (blockIdx.x == 0 && threadIdx.x < 32) pref_total(a);
}

// ------------------------------------------------------------------------------------------------
// Rows through a ring of chunks in shared memory.  A CTA takes rows b, b + G, ...; a producer warp keeps the ring full
// (cp.async.bulk), kT consumer threads take a chunk as kU 16-byte pieces each.  The gradient needs every number of a row
// a second time, after its maximum and sum are known: the last kRing chunks of the row are then still in the ring, only what
// came before them is loaded again (it is in L2).  Rows up to the ring's size are read once.
// Rows of odd length start at every alignment: the chunks start at the row's first 16-byte boundary, the few elements in
// front of it and behind the last whole piece are taken by one thread each with plain accesses; nothing outside a row is
// touched.  logits and dlogits have to be aligned alike.
// The chain from a row's last number to its first gradient (reductions, logarithm, the token's loss) leaves the memory idle,
// so an SM holds several CTAs whose rows are at different points.
// Bound by latency: policy loss of 4096 x 32768 bf16 105 us (4.8 TB/s) with a quarter of the warps there, the exponential unit 54 % busy, issue
// slots 44 %, DRAM three quarters; 87 us without the exponentials, 98 to 101 without the memory, so that neither alone is what it waits for.
// 1531 x 50257 fp32 128 us; preference, 6.2 thousand rows of 32000 bf16 (three quarters counted), 185 us, of which the statistics 72; losses
// without gradient 62 us at 4096 x 32768 bf16 and 55 at 1531 x 50257 fp32 (41 and 47 us of memory).
// Load number i of a row is chunk i, or chunk i - n beyond the first pass; slots are filled and freed in load order:
//   first pass    loads 0 .. n - 1, of which those before n - kRing are freed at once
//   second pass   loads n - kRing .. n - 1 from the ring, then loads n ..
// ------------------------------------------------------------------------------------------------
enum { kPolicy, kStats, kGrad };     // both passes with the policy loss between them; the first; the second
constexpr int kRing = 6;             // chunks of a ring
constexpr int kRowThreads = 512;     // consumer threads of an SM (768 with rings of four: the same)
constexpr int kU = 4;
template <int kT>
struct RowsSmem {
    alignas(128) uint8_t chunk[kRing][kT * kU * 16];
    float2 part[2][kT / 32];         // per warp: maximum, sum
    float4 next[2];                  // m, -g / s, g, z_y of the row
    alignas(8) uint64_t full[kRing];
    uint64_t empty[kRing];
};

template <int kT>
__device__ __forceinline__ void consumers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kT) : "memory"); }

__device__ __forceinline__ float piece_max(uint4 r, float m, float) {
    return fmaxf(fmaxf(fmaxf(m, __uint_as_float(r.x)), fmaxf(__uint_as_float(r.y), __uint_as_float(r.z))), __uint_as_float(r.w));
}
__device__ __forceinline__ float piece_max(uint4 r, float m, bf16) {
    const auto as2 = [](uint32_t v) { return *reinterpret_cast<const __nv_bfloat162*>(&v); };
    const __nv_bfloat162 b = __hmax2(__hmax2(as2(r.x), as2(r.y)), __hmax2(as2(r.z), as2(r.w)));
    return fmaxf(fmaxf(m, __low2float(b)), __high2float(b));
}

// A thread's pieces of one chunk into its running maximum and sum (two halves); kFull: all of them are there.
template <typename T, int kT, bool kFull>
__device__ __forceinline__ void chunk_stat(const uint8_t* chunk, int tid, int have, float& m, float2& s2) {
    uint4 raw[kU];
    float cm = m;
#pragma unroll
    for (int j = 0; j < kU; ++j)
        if (kFull || j < have) {
            raw[j] = *reinterpret_cast<const uint4*>(chunk + (tid + j * kT) * 16);
            cm = piece_max(raw[j], cm, T());
        }
    if (cm > m) {
        if (m != -INFINITY) s2 = mul2(s2, both(rescale(m, cm)));
        m = cm;
    }
    const Base b = base_of(m);
#pragma unroll
    for (int j = 0; j < kU; ++j)
        if (kFull || j < have) {
            float2 z[kPairs<T>];
            unpack(raw[j], z, T());
#pragma unroll
            for (int e = 0; e < kPairs<T>; ++e) s2 = add2(s2, exp_at(z[e], b));
        }
}
// Its pieces of the gradient, to `out` (the chunk's first element in memory).
template <typename T, int kT, bool kFull>
__device__ __forceinline__ void chunk_grad(const uint8_t* chunk, T* out, int tid, int have, Base b, float mul, bool zero, bool ok) {
#pragma unroll
    for (int j = 0; j < kU; ++j)
        if (kFull || j < have) {
            uint4 raw = *reinterpret_cast<const uint4*>(chunk + (tid + j * kT) * 16);
            float2 z[kPairs<T>];
            unpack(raw, z, T());
#pragma unroll
            for (int e = 0; e < kPairs<T>; ++e) z[e] = mul2(exp_at(z[e], b), both(mul));
            raw = zero ? make_uint4(0u, 0u, 0u, 0u) : pack(z, T());
            if (ok) reinterpret_cast<uint4*>(out)[tid + j * kT] = raw;
        }
}

struct RowArgs {
    PolicyArgs p;
    PrefArgs q;
};

template <typename T, int kT, int kMode>
__global__ void __launch_bounds__(kT + 32, kRowThreads / kT) k_rows(const __grid_constant__ RowArgs a) {
    constexpr int kWarps = kT / 32, kChunk = kT * kU * 16;
    extern __shared__ __align__(128) uint8_t smem_raw[];
    RowsSmem<kT>& s = *reinterpret_cast<RowsSmem<kT>*>(smem_raw);
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const T* logits = static_cast<const T*>(kMode == kPolicy ? a.p.logits : a.q.logits);
    T* dlogits = static_cast<T*>(kMode == kPolicy ? a.p.dlogits : kMode == kGrad ? a.q.dlogits : nullptr);
    const size_t ld = kMode == kPolicy ? a.p.ld : a.q.ld, ld_d = kMode == kPolicy ? a.p.ld_d : a.q.ld_d;
    const size_t rows = kMode == kPolicy ? a.p.T : a.q.T, G = gridDim.x;
    const int V = kMode == kPolicy ? a.p.V : a.q.V;
    const int32_t* labels = kMode == kPolicy ? a.p.labels : a.q.labels;
    const bool second = kMode == kGrad || (kMode == kPolicy && dlogits != nullptr);
    if (tid == 0) {
        for (int i = 0; i < kRing; ++i) {
            mbar_init(&s.full[i], 1);
            mbar_init(&s.empty[i], kWarps);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    pdl_wait();
    pdl_trigger();

    // the gradient pass goes through the rows from the last to the first: the last ones read are the ones still in L2
    auto row_of = [&](size_t k) { return kMode == kGrad ? rows - 1 - k : k; };
    auto live_row = [&](size_t t) {                  // rows that are not are neither read nor waited for
        if (kMode == kGrad) return a.q.g[t] != 0.f;
        const int y = labels[t];
        return y >= 0 && y < V && (kMode != kPolicy || a.p.weight[t] != 0.f);
    };

    if (warp == kWarps) {
        if (lane == 0) {                             // ---- producer
            int slot = 0;
            uint32_t round = 0;
            bool ok = true;
            bool live = blockIdx.x < rows && live_row(row_of(blockIdx.x));
            for (size_t k = blockIdx.x; k < rows && ok; k += G) {
                const bool now = live;
                live = k + G < rows && live_row(row_of(k + G));
                if (!now) continue;
                const T* row = logits + row_of(k) * ld;
                const RowCut c = cut_row(row, V);
                const uint32_t bytes = (uint32_t)c.pieces * 16u;
                const int n = (int)((bytes + kChunk - 1) / kChunk);
                const int loads = kMode == kPolicy && second && n > kRing ? 2 * n - kRing : n;
                for (int i = 0; i < loads && ok; ++i) {
                    const uint32_t at = (uint32_t)(i < n ? i : i - n) * kChunk, len = min((uint32_t)kChunk, bytes - at);
                    if (round > 0 && !mbar_wait(&s.empty[slot], (round - 1) & 1)) { ok = false; break; }
                    mbar_expect_tx(&s.full[slot], len);
                    bulk_load(s.chunk[slot], reinterpret_cast<const uint8_t*>(row + c.head) + at, len, &s.full[slot]);
                    if (++slot == kRing) { slot = 0; ++round; }
                }
            }
            if (!ok) {
                report_timeout();
                for (int i = 0; i < kRing; ++i) mbar_wait(&s.full[i], (round + (i < slot ? 0 : 1)) & 1, 4096u);   // copies in flight
            }
        }
        return;
    }

    // ---- consumers
    int slot = 0;
    uint32_t phase = 0;
    bool ok = true;
    double sums[3] = {0.0, 0.0, 0.0};                // thread 0: the policy loss's sums
    int parity = 0;
    // the next row's numbers are fetched while the current row is worked on
    struct {
        int y;
        float w, g, m, s;            // policy: w; gradient pass: g, m, s
        TokenIn in;                  // policy, thread 0
    } now{}, next{};
    auto fetch = [&](size_t k) {
        if (k >= rows) return;
        const size_t t = row_of(k);
        next.y = labels[t];
        if (kMode == kPolicy) {
            next.w = a.p.weight[t];
            if (tid == 0) next.in = token_in(a.p, t);
        }
        if (kMode == kGrad) {
            next.g = a.q.g[t];
            next.m = a.q.m[t];
            next.s = a.q.s[t];
        }
    };
    fetch(blockIdx.x);
    for (size_t k = blockIdx.x; k < rows; k += G) {
        now = next;
        fetch(k + G);
        const size_t t = row_of(k);
        const T* row = logits + t * ld;
        const int y = now.y;
        const RowCut c = cut_row(row, V);
        const int extra = tid < c.head ? tid : tid < c.head + c.tail ? V - c.tail + tid - c.head : -1;
        float m = -INFINITY, mul = 0.f, g = 0.f, zy = 0.f;
        const bool live = kMode == kGrad ? now.g != 0.f : y >= 0 && y < V && (kMode != kPolicy || now.w != 0.f);
        float ex = 0.f;
        if (live && extra >= 0) ex = to_f(row[extra]);
        const int n = (int)(((uint32_t)c.pieces * 16u + kChunk - 1) / kChunk);
        const int slot0 = slot;
        if (kMode == kGrad) {
            g = now.g;
            m = now.m;
            mul = -g / now.s;
            if (live) zy = to_f(row[y]);
        }
        if (kMode != kGrad && live) {
            if (tid == 0) zy = to_f(row[y]);
            const int keep_from = second ? n - kRing : n;
            float2 s2 = both(0.f);
            for (int i = 0; i < n; ++i) {
                if (!mbar_wait(&s.full[slot], phase, ok ? kSpinLimit : 1u)) ok = false;
                const int left = c.pieces - i * (kT * kU);
                if (left >= kT * kU) chunk_stat<T, kT, true>(s.chunk[slot], tid, kU, m, s2);
                else chunk_stat<T, kT, false>(s.chunk[slot], tid, (left - tid + kT - 1) / kT, m, s2);
                if (i < keep_from) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&s.empty[slot]);
                }
                if (++slot == kRing) { slot = 0; phase ^= 1u; }
            }
            RowStat st{m, sum2(s2)};
            if (extra >= 0) {
                float z[1] = {ex};
                stat_add(st, z);
            }
            // one pair per warp, joined by every warp that needs it
            const float wm = warp_max(st.m);
            float ws = at_max(st, wm);
#pragma unroll
            for (int o = 16; o; o >>= 1) ws += __shfl_xor_sync(0xffffffffu, ws, o);
            if (lane == 0) s.part[parity][warp] = make_float2(wm, ws);
            consumers_sync<kT>();
            if (warp == 0) {
                const float2 p = lane < kWarps ? s.part[parity][lane] : make_float2(-INFINITY, 0.f);
                RowStat all{p.x, 0.f};
                all.m = warp_max(all.m);
                all.s = at_max(RowStat{p.x, p.y}, all.m);
#pragma unroll
                for (int o = kWarps / 2; o; o >>= 1) all.s += __shfl_xor_sync(0xffffffffu, all.s, o);
                if (lane == 0) {
                    const bool some = all.m != -INFINITY || all.s != 0.f;
                    const float logp = some ? zy - all.m - log_sum(all) : 0.f;
                    if (kMode == kPolicy) {
                        if (some) {
                            const float w = now.w;
                            const TokenLoss l = token_loss(a.p, now.in, logp);
                            g = w * l.slope;
                            sums[0] += (double)w * l.loss;
                            sums[1] += (double)w * l.kl;
                            sums[2] += (double)w * l.clipped;
                        }
                        if (ok) a.p.logp[t] = logp;
                        s.next[parity] = make_float4(all.m, some ? -g / all.s : 0.f, g, zy);
                    } else if (ok) {
                        a.q.m[t] = all.m;
                        a.q.s[t] = all.s;
                        a.q.logp[t] = logp;
                        a.q.g[t] = 0.f;
                    }
                }
            }
            if (kMode == kPolicy && second) {
                consumers_sync<kT>();
                const float4 x = s.next[parity];
                m = x.x; mul = x.y; g = x.z; zy = x.w;
            }
            parity ^= 1;
        } else if (kMode != kGrad && tid == 0 && ok) {
            if (kMode == kPolicy) a.p.logp[t] = 0.f;
            else {
                a.q.m[t] = -INFINITY;
                a.q.s[t] = 0.f;
                a.q.logp[t] = 0.f;
                a.q.g[t] = 0.f;
            }
        }
        if (!second) continue;
        T* out = dlogits + t * ld_d;
        if (!live) {
            const RowCut o = cut_row(out, V);
            for (int i = tid; i < o.pieces; i += kT) *reinterpret_cast<uint4*>(out + o.head + i * kVec<T>) = make_uint4(0u, 0u, 0u, 0u);
            if (tid < o.head + o.tail) out[tid < o.head ? tid : V - o.tail + tid - o.head] = from_f<T>(0.f);
            continue;
        }
        // g ([v = y] - exp(z_v - m) / s): the label's element is written once more by the thread that wrote its piece
        const bool zero = g == 0.f;
        const Base base = base_of(m);
        const int resident = kMode == kGrad ? 0 : min(n, kRing);
        int at = kMode == kGrad || n >= kRing ? slot : slot0;
        for (int i = 0; i < n; ++i) {
            const int chunk = kMode == kGrad ? i : i < resident ? n - resident + i : i - resident;
            if (i >= resident) {
                if (!mbar_wait(&s.full[slot], phase, ok ? kSpinLimit : 1u)) ok = false;
                at = slot;
                if (++slot == kRing) { slot = 0; phase ^= 1u; }
            }
            const int left = c.pieces - chunk * (kT * kU);
            T* to = out + c.head + (size_t)chunk * (kT * kU * kVec<T>);
            if (left >= kT * kU) chunk_grad<T, kT, true>(s.chunk[at], to, tid, kU, base, mul, zero, ok);
            else chunk_grad<T, kT, false>(s.chunk[at], to, tid, (left - tid + kT - 1) / kT, base, mul, zero, ok);
            __syncwarp();
            if (lane == 0) mbar_arrive(&s.empty[at]);
            if (++at == kRing) at = 0;
        }
        if (extra >= 0 && ok) out[extra] = from_f<T>(zero ? 0.f : exp_at(ex, base) * mul);
        const int in_body = y - c.head;
        const int owner = in_body >= 0 && in_body < c.pieces * kVec<T> ? (in_body / kVec<T>) % kT : y < c.head ? y : y - (V - c.tail) + c.head;
        if (tid == owner && !zero && ok) out[y] = from_f<T>(exp_at(zy, base) * mul + g);
    }
    if (kMode == kGrad && blockIdx.x == 0 && warp == 0) pref_total(a.q);
    if (kMode == kPolicy && tid == 0)
        for (int i = 0; i < 3; ++i) a.p.part[(size_t)blockIdx.x * 3 + i] = sums[i];
    if (!ok) report_timeout();
}

// ------------------------------------------------------------------------------------------------
// Short rows: one warp each, its exponentials (kP 16-byte pieces a lane) in registers, so that each is formed once.  A warp
// keeps the next rows' pieces in flight in a ring of its own (bulk copies that lane 0 issues); nothing synchronises warps.  With
// a CTA per row (k_rows) the chain of a row's reductions bounded the rate: 65536 rows of 1000 bf16, policy loss 96 us, this way 76.
// ------------------------------------------------------------------------------------------------
constexpr int kWarpRow = 4096;               // bytes of the longest row that a warp takes: eight pieces a lane
constexpr int kWarpCta = 4;                  // warps of a CTA
constexpr int kWarpStages = 4;
constexpr int warp_rows_ctas(int pieces) { return pieces == 1 ? 8 : pieces == 4 ? 5 : 4; }     // CTAs of an SM, by the registers

template <typename T, int kP, int kMode>
__global__ void __launch_bounds__(kWarpCta * 32, warp_rows_ctas(kP)) k_warp_rows(const __grid_constant__ RowArgs a, int stages, uint32_t stage_bytes) {
    constexpr int kN = kPairs<T>;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ uint64_t bars[kWarpCta][kWarpStages];
    __shared__ double acc[kWarpCta][3];
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    uint64_t* full = bars[warp];
    uint8_t* ring = smem + (size_t)warp * stages * stage_bytes;
    const T* logits = static_cast<const T*>(kMode == kPolicy ? a.p.logits : a.q.logits);
    T* dlogits = static_cast<T*>(kMode == kPolicy ? a.p.dlogits : kMode == kGrad ? a.q.dlogits : nullptr);
    const size_t ld = kMode == kPolicy ? a.p.ld : a.q.ld, ld_d = kMode == kPolicy ? a.p.ld_d : a.q.ld_d;
    const size_t rows = kMode == kPolicy ? a.p.T : a.q.T, G = (size_t)gridDim.x * kWarpCta;
    const int V = kMode == kPolicy ? a.p.V : a.q.V;
    const int32_t* labels = kMode == kPolicy ? a.p.labels : a.q.labels;
    if (lane == 0) {
        for (int i = 0; i < stages; ++i) mbar_init(&full[i], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    pdl_wait();
    pdl_trigger();

    // a row's numbers, fetched ahead
    struct Row {
        int y;
        float w, g, m, s;            // policy: w; gradient pass: g, m, s
        TokenIn in;                  // policy
        bool live;                   // others are neither read nor waited for
    };
    auto fetch = [&](size_t t) {
        Row r{};
        if (t >= rows) return r;
        r.y = labels[t];
        r.live = r.y >= 0 && r.y < V;
        if (kMode == kPolicy) {
            r.w = a.p.weight[t];
            r.in = token_in(a.p, t);
            r.live = r.live && r.w != 0.f;
        }
        if (kMode == kGrad) {
            r.g = a.q.g[t];
            r.m = a.q.m[t];
            r.s = a.q.s[t];
            r.live = r.g != 0.f;
        }
        return r;
    };
    auto load = [&](int stage, size_t t) {           // lane 0; the row is live
        const T* row = logits + t * ld;
        const RowCut c = cut_row(row, V);
        if (c.pieces == 0) return;
        mbar_expect_tx(&full[stage], (uint32_t)c.pieces * 16u);
        bulk_load(ring + (size_t)stage * stage_bytes, row + c.head, (uint32_t)c.pieces * 16u, &full[stage]);
    };
    const size_t t0 = (size_t)blockIdx.x * kWarpCta + warp;
    bool ok = true;
    int stage = 0;
    uint32_t phases = 0;
    double sums[3] = {0.0, 0.0, 0.0};
    Row next = fetch(t0);
    // the row whose copy is issued next: its numbers are fetched a row ahead and looked at when it is its turn
    int y_later = -1;
    float w_later = 0.f;
    auto fetch_later = [&](size_t t) {
        const bool in = t < rows;
        y_later = in ? labels[t] : -1;
        if (kMode == kPolicy) w_later = in ? a.p.weight[t] : 0.f;
        if (kMode == kGrad) w_later = in ? a.q.g[t] : 0.f;
    };
    auto later_live = [&] { return (kMode == kGrad || (y_later >= 0 && y_later < V)) && (kMode == kStats || w_later != 0.f); };
    for (int i = 0; i < stages; ++i) {
        fetch_later(t0 + i * G);
        if (lane == 0 && later_live()) load(i, t0 + i * G);
    }
    fetch_later(t0 + stages * G);
    float zy_next = next.live ? to_f(logits[t0 * ld + next.y]) : 0.f;
    for (size_t t = t0; t < rows; t += G) {
        const Row now = next;
        const float zy = zy_next;
        const T* row = logits + t * ld;
        T* out = dlogits + t * ld_d;
        const RowCut c = cut_row(row, V);
        const int extra = lane < c.head ? lane : lane < c.head + c.tail ? V - c.tail + lane - c.head : -1;
        const float ex = now.live && extra >= 0 ? to_f(row[extra]) : -INFINITY;
        next = fetch(t + G);
        const bool write = kMode == kGrad || (kMode == kPolicy && dlogits != nullptr);
        float2 e[kP][kN];
        float m = now.m, mul = 0.f, g = now.g;
        Base b{};
        if (now.live) {
            if (c.pieces > 0) {
                if (!mbar_wait(&full[stage], (phases >> stage) & 1u, ok ? kSpinLimit : 1u)) ok = false;
                phases ^= 1u << stage;
            }
            const uint4* src = reinterpret_cast<const uint4*>(ring + (size_t)stage * stage_bytes) + lane;
            if (kMode != kGrad) {
                m = ex;              // -inf where there is none
#pragma unroll
                for (int j = 0; j < kP; ++j)
                    if (lane + 32 * j < c.pieces) m = piece_max(src[32 * j], m, T());
                m = warp_max(m);
            } else mul = -g / now.s;
            b = base_of(m);
            float2 s2 = both(0.f);
            uint4* o = reinterpret_cast<uint4*>(out + c.head) + lane;
#pragma unroll
            for (int j = 0; j < kP; ++j)
                if (lane + 32 * j < c.pieces) {
                    unpack(src[32 * j], e[j], T());
#pragma unroll
                    for (int k = 0; k < kN; ++k) {
                        e[j][k] = exp_at(e[j][k], b);
                        if (kMode != kGrad) s2 = add2(s2, e[j][k]);
                        else e[j][k] = mul2(e[j][k], both(mul));
                    }
                    if (kMode == kGrad && ok) o[32 * j] = pack(e[j], T());
                }
            if (kMode != kGrad) {
                float s = sum2(s2) + (extra >= 0 ? exp_at(ex, b) : 0.f);
#pragma unroll
                for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                const bool some = m != -INFINITY || s != 0.f;
                const float logp = some ? zy - m - log_sum(RowStat{m, s}) : 0.f;
                if (kMode == kPolicy) {
                    TokenLoss l{};
                    if (some) l = token_loss(a.p, now.in, logp);
                    g = now.w * l.slope;
                    mul = some ? -g / s : 0.f;
                    if (lane == 0) {
                        if (ok) a.p.logp[t] = logp;
                        sums[0] += (double)now.w * l.loss;
                        sums[1] += (double)now.w * l.kl;
                        sums[2] += (double)now.w * l.clipped;
                    }
                } else if (lane == 0 && ok) {
                    a.q.m[t] = m;
                    a.q.s[t] = s;
                    a.q.logp[t] = logp;
                    a.q.g[t] = 0.f;
                }
            }
        } else if (kMode != kGrad && lane == 0) {
            if (kMode == kPolicy) a.p.logp[t] = 0.f;
            else {
                a.q.m[t] = -INFINITY;
                a.q.s[t] = 0.f;
                a.q.logp[t] = 0.f;
                a.q.g[t] = 0.f;
            }
        }
        __syncwarp();                                // everybody has read the stage
        if (lane == 0 && later_live()) load(stage, t + (size_t)stages * G);
        fetch_later(t + (size_t)(stages + 1) * G);
        if (++stage == stages) stage = 0;
        zy_next = next.live ? to_f(logits[(t + G) * ld + next.y]) : 0.f;
        if (!write || !ok) continue;
        const bool zero = !now.live || g == 0.f;
        uint4* o = reinterpret_cast<uint4*>(out + c.head) + lane;
        if (kMode != kGrad || zero)
#pragma unroll
            for (int j = 0; j < kP; ++j)
                if (lane + 32 * j < c.pieces) {
#pragma unroll
                    for (int k = 0; k < kN; ++k) e[j][k] = mul2(e[j][k], both(mul));
                    o[32 * j] = zero ? make_uint4(0u, 0u, 0u, 0u) : pack(e[j], T());
                }
        if (extra >= 0) out[extra] = from_f<T>(zero ? 0.f : exp_at(ex, b) * mul);
        // the label's element, once more, by the lane that wrote its piece
        const int in_body = now.y - c.head;
        const bool inside = in_body >= 0 && now.y < V - c.tail;
        if (!zero && (inside ? lane == in_body / kVec<T> % 32 : extra == now.y)) out[now.y] = from_f<T>(exp_at(zy, b) * mul + g);
    }
    if (kMode == kGrad && blockIdx.x == 0 && warp == 0) pref_total(a.q);
    if (kMode == kPolicy) {
        if (lane == 0)
            for (int i = 0; i < 3; ++i) acc[warp][i] = sums[i];
        __syncthreads();
        if (threadIdx.x < 3) {
            double s = 0.0;
            for (int w = 0; w < kWarpCta; ++w) s += acc[w][threadIdx.x];
            a.p.part[(size_t)blockIdx.x * 3 + threadIdx.x] = s;
        }
    }
    if (!ok) report_timeout();
}

// ------------------------------------------------------------------------------------------------
// The policy loss with a row's exponentials kept in registers.  A row is taken by a cluster of C CTAs (C = 1 where one CTA
// can own it), kT threads each, a thread owning up to eight 16-byte pieces: exp(z - m) is formed once, when the element
// arrives, and scaled when the row's sum is known.  (Forming it twice makes the exponential unit as busy as the memory:
// 104 us for 4096 rows of 32768 bf16.)  A CTA's slices of the next rows are copied into shared memory meanwhile, so that the
// memory stays busy through the row's chain -- reductions, the exchange of the cluster's partial sums, the token's loss.
// No warp of its own issues the copies: registers are given to whole groups of four warps, and the exponentials need them.
// The CTAs of a cluster exchange (maximum, sum) by st.async into each other's shared memory.
// Few rows: larger clusters, so that all SMs have a part.
// ------------------------------------------------------------------------------------------------
constexpr int kOwnPieces = 8;
constexpr int kClusterMax = 8;
constexpr int kStagesMax = 8;
constexpr int kSliceThreads = 512;           // threads of an SM

struct SliceCtl {
    float2 part[2][16];              // per warp: maximum, sum
    float2 peer[2][kClusterMax];     // per CTA of the cluster
    float4 next[2];                  // m, -g / s, g, z_y of the row
    float zy[2];
    alignas(8) uint64_t full[kStagesMax];
    uint64_t peers[2];
};
constexpr size_t kSliceCtl = (sizeof(SliceCtl) + 127) / 128 * 128;

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// 8 bytes to the same variable of CTA `rank`, counted on the same barrier there.
__device__ __forceinline__ void send(float2* var, uint64_t* bar, uint32_t rank, float2 v) {
    uint32_t a, b;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(var)), "r"(rank));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(b) : "r"(smem_u32(bar)), "r"(rank));
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b64 [%0], %1, [%2];" ::"r"(a), "l"(as_u64(v)), "r"(b) : "memory");
}
__device__ __forceinline__ bool mbar_wait_cluster(uint64_t* bar, uint32_t parity, uint32_t limit) {
    for (uint32_t it = 0; it < limit; ++it) {
        uint32_t ok;
        asm volatile(
            "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
            : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
        if (ok) return true;
    }
    return false;
}

template <typename T, int kT>
__global__ void __launch_bounds__(kT, kSliceThreads / kT) k_policy_slices(const __grid_constant__ PolicyArgs a, int C, int stages, uint32_t stage_bytes) {
    constexpr int kWarps = kT / 32, kN = kPairs<T>;
    extern __shared__ __align__(128) uint8_t smem[];
    SliceCtl& s = *reinterpret_cast<SliceCtl*>(smem);
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int rank = C > 1 ? (int)cluster_rank() : 0;
    const size_t row0 = blockIdx.x / C, G = gridDim.x / C;
    if (tid == 0) {
        for (int i = 0; i < stages; ++i) mbar_init(&s.full[i], 1);
        mbar_init(&s.peers[0], 1);
        mbar_init(&s.peers[1], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (C > 1) cluster_sync(); else __syncthreads();

    // this CTA's pieces of a row
    struct Slice {
        RowCut cut;
        int first, pieces;
    };
    auto slice_of = [&](const T* row) {
        Slice q;
        q.cut = cut_row(row, a.V);
        const int per = (q.cut.pieces + C - 1) / C;
        q.first = min(rank * per, q.cut.pieces);
        q.pieces = min(per, q.cut.pieces - q.first);
        return q;
    };
    auto counted = [&](int y, float w) { return y >= 0 && y < a.V && w != 0.f; };   // other rows are neither read nor waited for
    auto load = [&](int stage, size_t t) {           // thread 0; the row is counted
        const T* row = static_cast<const T*>(a.logits) + t * a.ld;
        const Slice q = slice_of(row);
        if (q.pieces <= 0) return;
        mbar_expect_tx(&s.full[stage], (uint32_t)q.pieces * 16u);
        bulk_load(smem + kSliceCtl + (size_t)stage * stage_bytes, reinterpret_cast<const uint8_t*>(row + q.cut.head) + (size_t)q.first * 16,
                  (uint32_t)q.pieces * 16u, &s.full[stage]);
    };
    bool ok = true;
    int stage = 0, parity = 0;
    uint32_t phases = 0, peer_phase = 0;             // a bit per barrier
    double sums[3] = {0.0, 0.0, 0.0};                // thread 0
    // the numbers of the next row, and (thread 0) of the row whose copy is issued next, are fetched ahead
    int y_next = 0, y_load = 0;
    float w_next = 0.f, w_load = 0.f;
    TokenIn in_next{};                               // thread 0
    auto fetch = [&](size_t t) {
        if (t >= a.T) return;
        y_next = a.labels[t];
        w_next = a.weight[t];
        if (tid == 0) in_next = token_in(a, t);
    };
    auto fetch_load = [&](size_t t) {
        if (tid != 0) return;
        w_load = 0.f;
        if (t < a.T) {
            y_load = a.labels[t];
            w_load = a.weight[t];
        }
    };
    fetch(row0);
    if (tid == 0)
        for (int i = 0; i < stages; ++i) {
            const size_t t = row0 + i * G;
            if (t < a.T && counted(a.labels[t], a.weight[t])) load(i, t);
        }
    fetch_load(row0 + (size_t)stages * G);

    for (size_t t = row0; t < a.T; t += G) {
        const int y = y_next;
        const float w = w_next;
        const TokenIn in = in_next;
        fetch(t + G);
        const T* row = static_cast<const T*>(a.logits) + t * a.ld;
        T* out = static_cast<T*>(a.dlogits) + t * a.ld_d;
        const Slice q = slice_of(row);
        const int ends = rank == 0 ? q.cut.head + q.cut.tail : 0;
        const int extra = tid >= ends ? -1 : tid < q.cut.head ? tid : a.V - q.cut.tail + tid - q.cut.head;
        const int have = (q.pieces - tid + kT - 1) / kT;             // pieces of this thread: tid, tid + kT, ..
        auto refill = [&] {                          // the stage has been read by everybody
            if (tid == 0 && counted(y_load, w_load)) load(stage, t + (size_t)stages * G);
            fetch_load(t + (size_t)(stages + 1) * G);
            if (++stage == stages) stage = 0;
        };
        if (!counted(y, w)) {
            if (tid == 0 && rank == 0) a.logp[t] = 0.f;
            if (a.dlogits) {
                uint4* o = reinterpret_cast<uint4*>(out + q.cut.head) + q.first + tid;
                for (int i = 0; i < have; ++i) o[i * kT] = make_uint4(0u, 0u, 0u, 0u);
                if (extra >= 0) out[extra] = from_f<T>(0.f);
            }
            refill();
            continue;
        }
        const float ex = extra >= 0 ? to_f(row[extra]) : -INFINITY;
        float zy = 0.f;
        if (tid == 0) zy = to_f(row[y]);
        if (q.pieces > 0) {
            if (!mbar_wait(&s.full[stage], (phases >> stage) & 1u, ok ? kSpinLimit : 1u)) ok = false;
            phases ^= 1u << stage;
        }
        float2 e[kOwnPieces][kN], s2 = both(0.f);
        float m = -INFINITY, ms[kOwnPieces / 2];     // running maximum, and what it was for each two pieces
        const uint4* src = reinterpret_cast<const uint4*>(smem + kSliceCtl + (size_t)stage * stage_bytes) + tid;
#pragma unroll
        for (int j = 0; j < kOwnPieces; j += 2) {
            if (j < have) {
                uint4 raw[2];
                raw[0] = src[j * kT];
                float cm = piece_max(raw[0], m, T());
                if (j + 1 < have) {
                    raw[1] = src[(j + 1) * kT];
                    cm = piece_max(raw[1], cm, T());
                }
                if (cm > m) {
                    if (m != -INFINITY) s2 = mul2(s2, both(rescale(m, cm)));
                    m = cm;
                }
                const Base b = base_of(m);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (j + i < have) {
                        float2 z[kN];
                        unpack(raw[i], z, T());
#pragma unroll
                        for (int k = 0; k < kN; ++k) {
                            e[j + i][k] = exp_at(z[k], b);
                            s2 = add2(s2, e[j + i][k]);
                        }
                    }
            }
            ms[j / 2] = m;
        }
        RowStat st{m, sum2(s2)};
        if (extra >= 0) {
            const float z[1] = {ex};
            stat_add(st, z);
        }
        const float wm = warp_max(st.m);
        float ws = at_max(st, wm);
#pragma unroll
        for (int o = 16; o; o >>= 1) ws += __shfl_xor_sync(0xffffffffu, ws, o);
        if (lane == 0) s.part[parity][warp] = make_float2(wm, ws);
        __syncthreads();
        refill();
        if (warp == 0) {
            // the warps' pairs, then the CTAs': one lane each, joined by shuffles
            auto join = [&](float2 p) {
                RowStat all{p.x, 0.f};
                all.m = warp_max(all.m);
                all.s = at_max(RowStat{p.x, p.y}, all.m);
#pragma unroll
                for (int o = 8; o; o >>= 1) all.s += __shfl_xor_sync(0xffffffffu, all.s, o);
                return all;
            };
            const float2 none = make_float2(-INFINITY, 0.f);
            RowStat all = join(lane < kWarps ? s.part[parity][lane] : none);
            if (C > 1) {
                if (lane == 0) {
                    s.zy[parity] = zy;               // the logit is read before a peer can overwrite it (dlogits in place of logits)
                    mbar_expect_tx(&s.peers[parity], (uint32_t)C * 8u);
                }
                __syncwarp();
                if (lane < C) send(&s.peer[parity][rank], &s.peers[parity], (uint32_t)lane, make_float2(all.m, all.s));
                if (!mbar_wait_cluster(&s.peers[parity], (peer_phase >> parity) & 1u, ok ? kSpinLimit : 1u)) ok = false;
                peer_phase ^= 1u << parity;
                all = join(lane < C ? s.peer[parity][lane] : none);
            }
            if (lane == 0) {
                const bool some = all.m != -INFINITY || all.s != 0.f;
                const float logp = some ? zy - all.m - log_sum(all) : 0.f;
                float g = 0.f;
                TokenLoss l{};
                if (some) {
                    l = token_loss(a, in, logp);
                    g = w * l.slope;
                }
                s.next[parity] = make_float4(all.m, some ? -g / all.s : 0.f, g, zy);
                if (ok && rank == 0) a.logp[t] = logp;
                sums[0] += (double)w * l.loss;
                sums[1] += (double)w * l.kl;
                sums[2] += (double)w * l.clipped;
            }
        }
        if (a.dlogits) {
            __syncthreads();
            const float4 x = s.next[parity];
            const float mul = x.y, g = x.z;
            const Base b = base_of(x.x);
            const bool zero = g == 0.f;
            if (ok) {
                uint4* o = reinterpret_cast<uint4*>(out + q.cut.head) + q.first + tid;
#pragma unroll
                for (int j = 0; j < kOwnPieces; ++j)
                    if (j < have) {
                        const float at = ms[j / 2], f = at == -INFINITY ? mul : mul * rescale(at, x.x);
                        float2 v[kN];
#pragma unroll
                        for (int k = 0; k < kN; ++k) v[k] = mul2(e[j][k], both(f));
                        o[j * kT] = zero ? make_uint4(0u, 0u, 0u, 0u) : pack(v, T());
                    }
                if (extra >= 0) out[extra] = from_f<T>(zero ? 0.f : exp_at(ex, b) * mul);
                // the label's element, once more, by the thread that wrote its piece
                const int in_body = y - q.cut.head, piece = in_body / kVec<T> - q.first;
                const bool inside = in_body >= 0 && y < a.V - q.cut.tail;
                if (!zero && (inside ? piece >= 0 && piece < q.pieces && tid == piece % kT : extra == y)) out[y] = from_f<T>(exp_at(x.w, b) * mul + g);
            }
        }
        parity ^= 1;
    }
    if (tid == 0 && rank == 0)
        for (int i = 0; i < 3; ++i) a.part[row0 * 3 + i] = sums[i];
    if (!ok) report_timeout();
    if (C > 1) cluster_sync();       // no CTA leaves while another may still write to its shared memory
}

constexpr int kPlainWarpRow = 1024;  // the plain kernels take rows up to this length by one warp each

// Consumer threads of a CTA of k_rows for rows of this many bytes: the smallest whose ring holds the row.
int rows_threads(size_t bytes) { return bytes <= (size_t)kRing * 64 * kU * 16 ? 64 : bytes <= (size_t)kRing * 128 * kU * 16 ? 128 : 256; }
// Rows t of both matrices start at the same offset from a 16-byte boundary, for every t.
bool aligned_alike(const void* a, size_t ld_a, const void* b, size_t ld_b, size_t es) {
    return (((uintptr_t)a - (uintptr_t)b) & 15) == 0 && ((ld_a - ld_b) * es & 15) == 0;
}

template <typename T, int kT, int kMode>
cudaError_t launch_rows_of(const RowArgs& a, size_t rows, int sms, int* grid, cudaStream_t s) {
    const size_t smem = sizeof(RowsSmem<kT>), most = (size_t)sms * (kRowThreads / kT);
    *grid = (int)(rows < most ? rows : most);
    const cudaError_t e = allow_smem<k_rows<T, kT, kMode>>();
    return e != cudaSuccess ? e : launch_kernel(k_rows<T, kT, kMode>, *grid, kT + 32, smem, s, true, a);
}
template <typename T, int kMode>
cudaError_t launch_rows(const RowArgs& a, size_t rows, int V, int sms, int* grid, cudaStream_t s) {
    switch (rows_threads((size_t)V * sizeof(T))) {
        case 64: return launch_rows_of<T, 64, kMode>(a, rows, sms, grid, s);
        case 128: return launch_rows_of<T, 128, kMode>(a, rows, sms, grid, s);
        default: return launch_rows_of<T, 256, kMode>(a, rows, sms, grid, s);
    }
}

// k_policy_slices: CTAs of a cluster, threads of a CTA, slices in flight.  As few CTAs as can own the row; more where rows
// are few, down to slices of 8 KB.
struct SlicePlan {
    int cluster, threads, stages;    // cluster 0: more than a cluster can own
    uint32_t stage_bytes;
};
SlicePlan slice_plan(size_t T, size_t pieces, int sms) {
    SlicePlan p{1, 0, 0, 0};
    while (p.cluster < kClusterMax && (size_t)p.cluster * kSliceThreads * kOwnPieces < pieces) p.cluster *= 2;
    if ((size_t)p.cluster * kSliceThreads * kOwnPieces < pieces) return SlicePlan{};
    while (p.cluster < kClusterMax && T * p.cluster * 2 <= (size_t)sms && pieces / (2 * p.cluster) >= 512) p.cluster *= 2;
    const size_t own = (pieces + p.cluster - 1) / p.cluster;
    p.threads = own <= 64 * kOwnPieces ? 64 : own <= 128 * kOwnPieces ? 128 : own <= 256 * kOwnPieces ? 256 : 512;
    p.stage_bytes = (uint32_t)((own * 16 + 127) / 128 * 128);
    const size_t room = 216 * 1024 / (kSliceThreads / p.threads) - kSliceCtl;     // three slices of the largest that the threads own
    const size_t fit = room / p.stage_bytes;
    p.stages = (int)(fit < (size_t)kStagesMax ? fit : (size_t)kStagesMax);
    return p;
}
template <typename T, int kT>
cudaError_t launch_slices_of(const PolicyArgs& a, SlicePlan p, int sms, int* parts, cudaStream_t s) {
    const size_t smem = kSliceCtl + (size_t)p.stages * p.stage_bytes, most = (size_t)sms * (kSliceThreads / kT) / p.cluster;
    *parts = (int)(a.T < most ? a.T : most);
    const cudaError_t e = allow_smem<k_policy_slices<T, kT>>();
    return e != cudaSuccess ? e : launch_cluster(k_policy_slices<T, kT>, *parts * p.cluster, p.cluster, kT, smem, s, a, p.cluster, p.stages, p.stage_bytes);
}
template <typename T>
cudaError_t launch_slices(const PolicyArgs& a, SlicePlan p, int sms, int* parts, cudaStream_t s) {
    switch (p.threads) {
        case 64: return launch_slices_of<T, 64>(a, p, sms, parts, s);
        case 128: return launch_slices_of<T, 128>(a, p, sms, parts, s);
        case 256: return launch_slices_of<T, 256>(a, p, sms, parts, s);
        default: return launch_slices_of<T, 512>(a, p, sms, parts, s);
    }
}

template <typename T, int kP, int kMode>
cudaError_t launch_warps_of(const RowArgs& a, size_t rows, int V, int sms, int* grid, cudaStream_t s) {
    const uint32_t stage_bytes = (uint32_t)((V * sizeof(T) + 15) / 16 * 16);
    const size_t most = (size_t)sms * warp_rows_ctas(kP), want = (rows + kWarpCta - 1) / kWarpCta;
    const size_t fit = (size_t)200 * 1024 / (warp_rows_ctas(kP) * kWarpCta) / stage_bytes;      // at least three rows of 4 KB
    const int stages = (int)(fit < (size_t)kWarpStages ? fit : (size_t)kWarpStages);
    *grid = (int)(want < most ? want : most);
    const cudaError_t e = allow_smem<k_warp_rows<T, kP, kMode>>();
    return e != cudaSuccess ? e : launch_kernel(k_warp_rows<T, kP, kMode>, *grid, kWarpCta * 32, (size_t)kWarpCta * stages * stage_bytes, s, true, a, stages, stage_bytes);
}
template <typename T, int kMode>
cudaError_t launch_warps(const RowArgs& a, size_t rows, int V, int sms, int* grid, cudaStream_t s) {
    const size_t bytes = V * sizeof(T);
    return bytes <= 512 ? launch_warps_of<T, 1, kMode>(a, rows, V, sms, grid, s) : bytes <= 2048 ? launch_warps_of<T, 4, kMode>(a, rows, V, sms, grid, s)
                                                                                              : launch_warps_of<T, 8, kMode>(a, rows, V, sms, grid, s);
}

// Which kernel takes the rows: logits and dlogits that are not aligned alike go to the plain ones, which read the row twice
// from memory; short rows to a warp each; few long rows of the policy loss to a cluster each; the rest to k_rows.
template <typename T>
cudaError_t launch_policy(const PolicyArgs& a, float* stats, int sms, cudaStream_t s) {
    const bool alike = !a.dlogits || aligned_alike(a.logits, a.ld, a.dlogits, a.ld_d, sizeof(T));
    int parts = 0;           // CTAs or clusters that leave partial sums
    cudaError_t e = cudaSuccess;
    if (a.T > 0) {
        const RowArgs r{a, PrefArgs{}};
        const SlicePlan p = alike && a.V * sizeof(T) > kWarpRow && a.T * 2 <= (size_t)sms ? slice_plan(a.T, (size_t)a.V / kVec<T>, sms) : SlicePlan{};
        if (!alike) {
            const bool warp_rows = a.V <= kPlainWarpRow;
            const size_t want = warp_rows ? (a.T + 7) / 8 : a.T;
            parts = (int)(want < (size_t)(4 * sms) ? want : (size_t)(4 * sms));
            e = warp_rows ? launch_kernel(k_policy_rows<T, 32, 8>, parts, 256, 0, s, true, a) : launch_kernel(k_policy_rows<T, 512, 1>, parts, 512, 0, s, true, a);
        } else if (a.V * sizeof(T) <= kWarpRow) e = launch_warps<T, kPolicy>(r, a.T, a.V, sms, &parts, s);
        else if (p.cluster) e = launch_slices<T>(a, p, sms, &parts, s);
        else e = launch_rows<T, kPolicy>(r, a.T, a.V, sms, &parts, s);
    }
    if (e != cudaSuccess) return e;
    return launch_kernel(k_policy_stats, 1, 96, 0, s, true, (const double*)a.part, parts, stats);
}

template <typename T>
cudaError_t launch_pref(const PrefArgs& a, int sms, cudaStream_t s) {
    const bool alike = a.dlogits && aligned_alike(a.logits, a.ld, a.dlogits, a.ld_d, sizeof(T));
    const RowArgs r{PolicyArgs{}, a};
    int grid = 0;
    cudaError_t e = cudaSuccess;
    if (a.T > 0)
        e = a.V * sizeof(T) <= kWarpRow ? launch_warps<T, kStats>(r, a.T, a.V, sms, &grid, s) : launch_rows<T, kStats>(r, a.T, a.V, sms, &grid, s);
    if (e != cudaSuccess) return e;
    if (a.pairs > 0) {
        e = launch_kernel(k_pref_pairs, (int)(a.pairs < (size_t)sms ? a.pairs : (size_t)sms), 1024, 0, s, true, a);
        if (e != cudaSuccess) return e;
    }
    if (alike && a.T > 0)
        return a.V * sizeof(T) <= kWarpRow ? launch_warps<T, kGrad>(r, a.T, a.V, sms, &grid, s) : launch_rows<T, kGrad>(r, a.T, a.V, sms, &grid, s);
    const bool warp_rows = a.V <= kPlainWarpRow;
    const size_t want = !a.dlogits ? 1 : warp_rows ? (a.T + 7) / 8 : a.T;
    grid = (int)(want < 1 ? 1 : want < (size_t)(4 * sms) ? want : (size_t)(4 * sms));
    return warp_rows ? launch_kernel(k_pref_grad<T, 32, 8>, grid, 256, 0, s, true, a) : launch_kernel(k_pref_grad<T, 512, 1>, grid, 512, 0, s, true, a);
}

bool misaligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// A row's bytes and its chunks of up to 16 KB are counted in 32 bits; a row's columns, and the rows of an answer in steps of 512, in 31.
constexpr uint64_t kRowBytesMax = (1ull << 32) - (1ull << 16);
constexpr uint64_t kTokensMax = (1ull << 31) - 513;
bool too_wide(uint64_t V, uint32_t dtype) { return V > kRowBytesMax / (dtype == ABS_F32 ? 4 : 2); }

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

namespace abs_sgd {
cudaError_t take_status_loss(int* status, cudaStream_t s) { return take_status(status, s); }
}  // namespace abs_sgd

using namespace abs_sgd;

extern "C" size_t abs_policy_loss_workspace(void) { return up256(sizeof(double) * 3 * kStatCtasMax); }

extern "C" int abs_policy_loss(const void* logits, uint32_t dtype, uint64_t tokens, uint64_t vocab, uint64_t ld, const int32_t* labels,
                               const float* logp_old, const float* logp_ref, const float* advantage, const float* weight,
                               float clip_low, float clip_high, float kl_coef, float* stats, float* logp, void* dlogits,
                               uint64_t ld_d, void* workspace, size_t workspace_bytes, void* stream) {
    if (const char* why = check_logits(logits, dtype, tokens, vocab, ld, labels, dlogits, ld_d)) return thread_error(ABS_EINVAL, why);
    if (too_wide(vocab, dtype)) return thread_error(ABS_ELIMIT, "vocab: a row of logits exceeds 2^32 - 2^16 bytes");
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
    if (too_wide(vocab, dtype)) return thread_error(ABS_ELIMIT, "vocab: a row of logits exceeds 2^32 - 2^16 bytes");
    if (tokens > kTokensMax) return thread_error(ABS_ELIMIT, "tokens exceeds 2^31 - 513");
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
