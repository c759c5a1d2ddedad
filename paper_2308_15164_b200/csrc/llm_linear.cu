// Linear layer with bias, activation and residual, and its gradients (abs_linear*).
//
//     forward   y = act(x w + bias) + residual          A = x  [T, in]  K-major      B = w  [in, out]  N-major
//     dgrad     dx = (dy w^T) act'(z) + residual        A = dy [T, out] K-major      B = w^T           K-major
//     wgrad     dw (+)= x^T dy                          A = x^T         M-major      B = dy [T, out]   N-major
// One kernel, k_linear, for the three: C[M, N] = A[M, K] B[K, N] with the operands read as they lie (an operand whose contraction
// index runs along its rows is "K-major", the others "MN-major"; TMA boxes of 64 columns, 128-byte swizzled rows, either way), and
// the layer's elementwise work on the sums while they are still in registers.
#include <math.h>

#include <algorithm>
#include <initializer_list>

#include "abs_internal.h"
#include "abs_llm.h"
#include "llm_host.h"
#include "llm_status.cuh"
#include "row_ring.cuh"
#include "tcgen05.cuh"

namespace abs_sgd {
namespace {

enum { kForward, kDgrad, kWgrad };

struct LinArgs {
    int M, N, K;
    int tiles_m, tiles_n, whole, rest, splits, kb_per_split;   // tiles: whole ones, then `rest` cut into `splits` runs; kb: 64 of K
    float* part;                     // [splits][rest][kTM][kTN]
    void* out;
    size_t ld;
    const float* bias;
    const void* res;                 // type of the output
    size_t ld_res;
    const bf16* z_in;                // dgrad
    bf16* z_out;                     // forward
    size_t ld_z;
    int accumulate;
    int join;                        // tiles that are cut, or not, go through k_linear_join
    int wide;                        // what the rows of out, res and z are aligned to: 32, 16 bytes, or 0: less
};

// ---- activations, two numbers at a time
// |v|, at most `most`; a NaN stays one.
__device__ __forceinline__ float2 limited(float2 v, float most) {
    float2 w;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(w.x) : "f"(fabsf(v.x)), "f"(most));
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(w.y) : "f"(fabsf(v.y)), "f"(most));
    return w;
}
__device__ __forceinline__ float2 minus(float2 v) { return make_float2(-v.x, -v.y); }
__device__ __forceinline__ float2 reciprocal(float2 d) {
    float2 r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(d.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(d.y));
    return r;
}
// v = -h k rounded, k = kHi + kLo, and what that leaves out, where h is `more` larger.
template <bool kFine>
__device__ __forceinline__ float2 exponent(float2 h, float2 more, float kHi, float kLo, float2& v) {
    v = mul2(minus(h), both(kHi));
    if (!kFine) return both(0.f);
    float2 left = fma2(minus(h), both(kHi), minus(v));
    left = fma2(more, both(-kHi), left);
    return fma2(minus(h), both(kLo), left);
}
// Both activations fall, and rise, by the same function of |z|; kFine: results of 32 bits, with what the rounding of an exponential's argument leaves out.
// bf16 ones, rounded to 2^-9, do without (SiLU 8e-7 at |z| = 12; GELU 3e-6 at 8, 8e-6 at 12): the gradient through GELU alone, 8192 x 8192, takes 86 us
// with it and 74 without.
//
// Phi(-|z|) = exp(-z^2 / 2) P(1 / (1 + 0.35 |z|)) with P of degree 7 fitted to the smallest relative error over 0 <= |z| <= 13.5, so that the lower tail
// keeps its precision: 3e-7, in fp32 6e-7, with the exponential 1.4e-6 at most.  The exponential as the square of exp(-z^2 / 4), which stays within the unit's
// range as far as there is something to see.  E: the exponential, q: Phi(-|z|), w: |z| up to 16, where both are zero.
template <bool kFine>
__device__ __forceinline__ void normal_tail(float2 z, float2& E, float2& q, float2& w) {
    constexpr double k = 0.36067376022224085;                // log2(e) / 4
    w = limited(z, 16.f);
    const float2 t = reciprocal(fma2(w, both(0.35f), both(1.f))), h = mul2(w, w);
    float2 v;
    const float2 left = exponent<kFine>(h, kFine ? fma2(w, w, minus(h)) : h, (float)k, (float)(k - (double)(float)k), v), e = exp2_of(v);
    E = mul2(e, e);
    if (kFine) E = fma2(mul2(left, both(1.3862943611198906f)), E, E);
    float2 p;
    p = fma2(t, both(0.04894255149557414f), both(-0.20211968521483073f));
    p = fma2(p, t, both(0.24064142309471856f));
    p = fma2(p, t, both(-0.017023902126677096f));
    p = fma2(p, t, both(0.15596167730976151f));
    p = fma2(p, t, both(0.1333550587912772f));
    p = fma2(p, t, both(0.14027034589594403f));
    p = fma2(p, t, both(-2.731542404448325e-05f));
    q = mul2(p, E);
}
// t = sigmoid(-|z|) and r = sigmoid(|z|); t falls to zero where the exponential does, |z| > 87.  w: |z| up to 126.
template <bool kFine>
__device__ __forceinline__ void sigmoids(float2 z, float2& t, float2& r, float2& w) {
    constexpr double k = 1.4426950408889634;                 // log2(e)
    w = limited(z, 126.f);
    float2 v;
    const float2 left = exponent<kFine>(w, both(0.f), (float)k, (float)(k - (double)(float)k), v);
    float2 e = exp2_of(v);
    if (kFine) e = fma2(mul2(left, both(0.6931471805599453f)), e, e);
    r = reciprocal(add2(e, both(1.f)));
    t = mul2(e, r);
}
template <uint32_t kAct, bool kFine>
__device__ __forceinline__ float2 activate(float2 z) {
    if (kAct == ABS_ACT_RELU) return make_float2(z.x > 0.f ? z.x : z.x == z.x ? 0.f : z.x, z.y > 0.f ? z.y : z.y == z.y ? 0.f : z.y);
    const float2 top = make_float2(fmaxf(z.x, 0.f), fmaxf(z.y, 0.f));
    float2 E, q, w;
    if (kAct == ABS_ACT_GELU) {                  // max(z, 0) - |z| Phi(-|z|)
        normal_tail<kFine>(z, E, q, w);
        return fma2(minus(w), q, top);
    }
    if (kAct == ABS_ACT_SILU) {                  // max(z, 0) - |z| sigmoid(-|z|)
        sigmoids<kFine>(z, q, E, w);
        return fma2(minus(w), q, top);
    }
    return z;
}
template <uint32_t kAct, bool kFine>
__device__ __forceinline__ float2 slope(float2 z) {
    if (kAct == ABS_ACT_RELU) return make_float2(z.x > 0.f ? 1.f : z.x == z.x ? 0.f : z.x, z.y > 0.f ? 1.f : z.y == z.y ? 0.f : z.y);
    float2 E, q, w, u;                           // u: the slope at -|z|; at |z| it is 1 - u
    if (kAct == ABS_ACT_GELU) {                  // Phi(-|z|) - |z| phi(|z|)
        normal_tail<kFine>(z, E, q, w);
        u = fma2(minus(w), mul2(E, both(0.3989422804014327f)), q);
    } else if (kAct == ABS_ACT_SILU) {           // t - |z| t r
        sigmoids<kFine>(z, q, E, w);
        u = fma2(minus(mul2(w, E)), q, q);
    } else {
        return both(1.f);
    }
    return make_float2(z.x > 0.f ? 1.f - u.x : u.x, z.y > 0.f ? 1.f - u.y : u.y);
}

// kC consecutive elements of a row; `to32`: 32-byte aligned, otherwise 16-byte.
template <typename T, int kC>
struct Piece {
    static constexpr int kN = kC / kVec<T>;
    uint4 w[kN];
    __device__ __forceinline__ void load(const T* p, bool to32) {
        if (kN % 2 == 0 && to32) {
#pragma unroll
            for (int h = 0; h + 1 < kN; h += 2)
                asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                             : "=r"(w[h].x), "=r"(w[h].y), "=r"(w[h].z), "=r"(w[h].w), "=r"(w[h + 1].x), "=r"(w[h + 1].y), "=r"(w[h + 1].z), "=r"(w[h + 1].w)
                             : "l"(p + h * kVec<T>) : "memory");
        } else {
#pragma unroll
            for (int h = 0; h < kN; ++h) w[h] = *reinterpret_cast<const uint4*>(p + h * kVec<T>);
        }
    }
    __device__ __forceinline__ void store(T* p, bool to32) const {
        if (kN % 2 == 0 && to32) {
#pragma unroll
            for (int h = 0; h + 1 < kN; h += 2)
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p + h * kVec<T>), "r"(w[h].x), "r"(w[h].y), "r"(w[h].z), "r"(w[h].w),
                             "r"(w[h + 1].x), "r"(w[h + 1].y), "r"(w[h + 1].z), "r"(w[h + 1].w) : "memory");
        } else {
#pragma unroll
            for (int h = 0; h < kN; ++h) *reinterpret_cast<uint4*>(p + h * kVec<T>) = w[h];
        }
    }
    __device__ __forceinline__ void get(float2 (&v)[kC / 2]) const {
#pragma unroll
        for (int h = 0; h < kN; ++h) {
            float2 u[kPairs<T>];
            unpack(w[h], u, T());
#pragma unroll
            for (int i = 0; i < kPairs<T>; ++i) v[h * kPairs<T> + i] = u[i];
        }
    }
    __device__ __forceinline__ void put(const float2 (&v)[kC / 2]) {
#pragma unroll
        for (int h = 0; h < kN; ++h) {
            float2 u[kPairs<T>];
#pragma unroll
            for (int i = 0; i < kPairs<T>; ++i) u[i] = v[h * kPairs<T> + i];
            w[h] = pack(u, T());
        }
    }
};

// The layer's work on kC sums of a row, all of them inside the matrix: what it reads, then what it makes of the sums.
template <int kEpi, uint32_t kAct, typename T, int kC>
struct Finish {
    Piece<T, kC> r;                  // residual, or what dw holds
    Piece<bf16, kC> z;
    __device__ __forceinline__ void load(const LinArgs& a, int row, int col) {
        if (kEpi == kWgrad ? a.accumulate != 0 : a.res != nullptr)
            r.load(kEpi == kWgrad ? static_cast<const T*>(a.out) + (size_t)row * a.ld + col : static_cast<const T*>(a.res) + (size_t)row * a.ld_res + col, a.wide == 32);
        if (kEpi == kDgrad && kAct != ABS_ACT_NONE) z.load(a.z_in + (size_t)row * a.ld_z + col, a.wide == 32);
    }
    __device__ __forceinline__ void operator()(const LinArgs& a, int row, int col, float2 (&v)[kC / 2]) {
        float2 w[kC / 2];
        if (kEpi == kForward) {
            if (a.bias) {
                const float* b = a.bias + col;
#pragma unroll
                for (int i = 0; i < kC / 2; ++i) v[i] = add2(v[i], make_float2(__ldg(b + 2 * i), __ldg(b + 2 * i + 1)));
            }
            if (a.z_out) {
                Piece<bf16, kC> o;
                o.put(v);
                o.store(a.z_out + (size_t)row * a.ld_z + col, a.wide == 32);
            }
#pragma unroll
            for (int i = 0; i < kC / 2; ++i) v[i] = activate<kAct, sizeof(T) == 4>(v[i]);
        }
        if (kEpi == kDgrad && kAct != ABS_ACT_NONE) {
            z.get(w);
#pragma unroll
            for (int i = 0; i < kC / 2; ++i) v[i] = mul2(v[i], slope<kAct, sizeof(T) == 4>(w[i]));
        }
        if (kEpi == kWgrad ? a.accumulate != 0 : a.res != nullptr) {
            r.get(w);
#pragma unroll
            for (int i = 0; i < kC / 2; ++i) v[i] = add2(v[i], w[i]);
        }
        Piece<T, kC> o;
        o.put(v);
        o.store(static_cast<T*>(a.out) + (size_t)row * a.ld + col, a.wide == 32);
    }
};
// The same for single ones.
template <int kEpi, uint32_t kAct, typename T>
struct FinishOne {
    float r, z;
    __device__ __forceinline__ void load(const LinArgs& a, int row, int col) {
        if (kEpi == kWgrad) r = a.accumulate ? to_f(static_cast<const T*>(a.out)[(size_t)row * a.ld + col]) : 0.f;
        else r = a.res ? to_f(static_cast<const T*>(a.res)[(size_t)row * a.ld_res + col]) : 0.f;
        if (kEpi == kDgrad && kAct != ABS_ACT_NONE) z = __bfloat162float(a.z_in[(size_t)row * a.ld_z + col]);
    }
    __device__ __forceinline__ void operator()(const LinArgs& a, int row, int col, float bias, float v) {
        if (kEpi == kForward) {
            v += bias;
            if (a.z_out) a.z_out[(size_t)row * a.ld_z + col] = __float2bfloat16_rn(v);
            v = activate<kAct, sizeof(T) == 4>(both(v)).x;
        }
        if (kEpi == kDgrad && kAct != ABS_ACT_NONE) v *= slope<kAct, sizeof(T) == 4>(both(z)).x;
        static_cast<T*>(a.out)[(size_t)row * a.ld + col] = from_f<T>(v + r);
    }
};

// ------------------------------------------------------------------------------------------------
// Two CTAs (two SMs) share an output tile of 256 x 256: each holds the operand's 128 rows of A and 128 columns of B, 32 KB for a run of
// 64 along K.  Roles in each CTA:
//   warp 0      TMA producer, up to kStages runs ahead
//   warp 1      (first CTA only) MMA issuer: four tcgen05.mma.cta_group::2 (M 256, N 256, K 16) per run into one of two TMEM accumulators
//   the others  epilogue, four warps for the rows, a row a thread, 16 columns at a time with the reads of the next ones under way (through a
//               staging tile in shared memory the results took a tenth of its bandwidth from the product: 266 -> 254 us)
//                 kSum    eight warps of 128 columns add up an item's segments (kSegmentRuns) in registers
//                 else    bf16 results of whole tiles of one segment straight from TMEM, sixteen warps of 64 columns (8192 x 256 x 8192: 57 us,
//                         through registers with eight warps 97)
// Items are dealt out round-robin to the pairs: the whole tiles, as many as fill all pairs equally often, then the rest, each cut along K
// into `splits` parts so that they too keep all pairs busy; k_linear_join adds those up in order and does the elementwise work.
// Launched in plain stream order, and starts no successor early (see llm_ckpt8.cu).  Every wait on a barrier is bounded.
// Bound by the tensor core and what feeds it where there is enough to do (the results' way out takes a tenth of it), and by the power limit in a loop.  A
// library's bf16 product of the same operands alone took (us, this kernel / the library, few calls after a pause): 8192 x 2048 x 8192 197 / 175, with GELU 220,
// and z kept 229, as fp32 204; 8192 x 8192 x 8192 759 / 659; gradient of the input 8192 x 8192 x 2048 199 / 182; of the weight, 2048 x 8192 of 8192 tokens,
// 198 / 181.  Few tokens: 8 us for one tile of one run (launch in plain order, tensor memory, first copies, epilogue), 16 runs of K 4 more.
// ------------------------------------------------------------------------------------------------
constexpr int kTM = 256, kTN = 256, kTK = 64;    // of a pair
constexpr int kStages = 5;
constexpr int kHalf = kTK * 128 * 2;             // bytes of an operand's share of a CTA and run
constexpr int kPitch = 20;                       // floats of a staged row of 16: 16-byte pieces, eight rows on different banks
// Sums are taken out of TMEM every kSegmentRuns runs and added up in fp32, since the tensor core drops low bits at each of its additions: without, the
// error grows with K (positive terms, K 16384: up to 8e-5).  Weight gradient of 8192 tokens, error of the result's norm / us of 8192 x 8192 x 2048: 12 runs
// 7e-7 / 215, 24 1.5e-6 / 210, 32 2.1e-6 / 208, never 8.6e-6 / 206.  bf16 results, which are rounded to 2^-9, take 16 runs: with 12, a K of 1024 would need
// two segments (7 x 1024 x 1024 with GELU 15.4 us, in two 18.4; 8192 x 2048 x 8192 211 and 214, in one of any length 200).
template <typename T>
constexpr int kSegmentRuns = sizeof(T) == 4 ? 12 : 16;
template <bool kSum>
constexpr int kEpiWarps = kSum ? 8 : 16;
template <bool kSum>
constexpr int kFirstEpi = kSum ? 4 : 2;                          // the epilogue's first warp
template <bool kSum>
constexpr int kWarpCols = kTN / (kEpiWarps<kSum> / 4);           // columns of an epilogue warp
template <bool kSum>
constexpr int kThreads = (kFirstEpi<kSum> + kEpiWarps<kSum>) * 32;
constexpr int kSms = 148;
constexpr uint64_t kSizeMax = 0x7fffffc0ull;
constexpr int kMinRuns = 12;     // runs of 64 that a part of a cut tile has at least: shorter ones do not pay for the join (some 7 us)
// Where rows of the output, residual or z are not 16-byte aligned the epilogue moves single elements; if it has to read some, they are read
// in many small parts.  Up to kFewTiles tiles, a quarter of what keeps all SMs busy, that is left to k_linear_join, on all of them, and K is cut down to
// kMinRunsJoin runs.  us with / without: forward with residual, K 1024, 4 tiles 24.6 / 26.6, 16 tiles 24.6 / 26.7, 24 tiles 30.7 / 28.0; input gradient through
// GELU 20.5 / 26.6, 22.6 / 26.6, 28.7 / 26.6; weight gradient of 1024 tokens added to what is there 22.5 / 27.6, 23.6 / 28.6, 26.7 / 28.7; K 256, 512 and 2048
// alike.  With 8 runs instead of 4: 515 x 1000 x 1111 26.6 instead of 24.6.
constexpr int kFewTiles = 18, kMinRunsJoin = 4;

struct LinSmem {
    alignas(1024) uint8_t a[kStages][kHalf];
    alignas(1024) uint8_t b[kStages][kHalf];
    alignas(16) float out[16][32 * kPitch];
    alignas(8) uint64_t full[kStages];       // first CTA: both CTAs' copies of a run have landed
    uint64_t empty[kStages];                 // the run's MMAs have read both CTAs' operands
    uint64_t acc_full[2];
    uint64_t acc_empty[2];                   // first CTA: both CTAs have read the accumulator
    uint32_t tmem_base;
    uint32_t failed;
};

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// tma_load_2d whose bytes are counted on the same barrier of the cluster's first CTA.
__device__ __forceinline__ void tma_load_2d_first(void* dst, const CUtensorMap* tm, int x, int y, uint64_t* bar) {
    uint32_t b;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(b) : "r"(smem_u32(bar)));
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];"
        ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(tm)), "r"(x), "r"(y), "r"(b) : "memory");
}
// One arrival on the same barrier of the cluster's first CTA; what it announces is ordered by tcgen05.fence.
__device__ __forceinline__ void arrive_first(uint64_t* bar) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(smem_u32(bar)));
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(a) : "memory");
}
__device__ __forceinline__ void umma2_bf16(uint32_t tmem_d, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
        " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n"
        ::"r"(tmem_d), "l"(da), "l"(db), "r"(idesc), "r"(accumulate) : "memory");
}
// Arrives on this barrier of both CTAs when the MMAs issued so far are done.
__device__ __forceinline__ void umma2_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
}

// First row and column of a tile.  Eight rows of tiles at a time, column by column: the tiles that run together then share as few parts of
// the operands as they can (8192 x 8192 x 8192 row by row read one operand 14 times).
__device__ __forceinline__ void place(const LinArgs& a, int tile, int& m0, int& n0) {
    constexpr int kBand = 8;
    const int band = tile / (kBand * a.tiles_n), r = tile - band * kBand * a.tiles_n, high = min(kBand, a.tiles_m - band * kBand);
    m0 = (band * kBand + r % high) * kTM;
    n0 = r / high * kTN;
}

// This CTA's share of an operand, 128 rows (or columns) from `mn` and 64 of K from `k`.
template <bool kMn>
__device__ __forceinline__ void load_operand(uint8_t* dst, const CUtensorMap* tm, int mn, int k, uint64_t* bar) {
    if constexpr (kMn) {
        tma_load_2d_first(dst, tm, mn, k, bar);
        tma_load_2d_first(dst + kHalf / 2, tm, mn + 64, k, bar);
    } else {
        tma_load_2d_first(dst, tm, k, mn, bar);
    }
}
// Its descriptor for the k16-th step of 16.
template <bool kMn>
__device__ __forceinline__ uint64_t operand_desc(uint32_t at, int k16) {
    return kMn ? umma_desc_mn_sw128(at + k16 * 2048, kHalf / 2) : umma_desc_k_sw128(at + k16 * 32);
}

// This CTA has given up: its rows of the pair's partial sums are missing.  A call of its own, out of the way of the kernel's registers.
__device__ __noinline__ void gave_up(const LinArgs& a) {
    if (threadIdx.x == 0) report_timeout();
    if (!a.join) return;
    float* const first = a.part + (size_t)cluster_rank() * 128 * kTN;
    for (int it = blockIdx.x / 2; it < a.whole + a.rest * a.splits; it += gridDim.x / 2)
        for (int k = threadIdx.x; k < 128 * kTN && it >= a.whole; k += blockDim.x) first[(size_t)(it - a.whole) * kTM * kTN + k] = __uint_as_float(kUnformed);
}

template <int kEpi, uint32_t kAct, typename T, bool kSum>
__global__ void __launch_bounds__(kThreads<kSum>, 1) k_linear(const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_b,
                                                        const __grid_constant__ LinArgs a) {
    constexpr bool kAMn = kEpi == kWgrad, kBMn = kEpi != kDgrad;
    static_assert(kSum || sizeof(T) == 2, "");
    constexpr int kCols = kWarpCols<kSum>;
    extern __shared__ uint8_t smem_raw[];
    LinSmem& s = *reinterpret_cast<LinSmem*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int rank = (int)cluster_rank();
    const int pair = blockIdx.x / 2, pairs = gridDim.x / 2;
    const int items = a.whole + a.rest * a.splits;
    const int kb_total = (a.K + kTK - 1) / kTK;
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s.tmem_base)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&s.full[i], 1);
            mbar_init(&s.empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&s.acc_full[i], 1);
            mbar_init(&s.acc_empty[i], 2 * kEpiWarps<kSum>);       // the epilogue warps of each CTA
        }
        s.failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = s.tmem_base;
    volatile uint32_t* failed = &s.failed;

    struct Item {
        int m0, n0, kb0, kb1;        // first row and column of the pair's tile, runs of 64 of K
        int part;                    // index of the partial sum, -1: straight to the output
    };
    auto item_of = [&](int it) {
        Item q;
        int tile = it;
        q.part = -1;
        q.kb0 = 0;
        q.kb1 = kb_total;
        if (it >= a.whole) {
            const int r = it - a.whole;
            tile = a.whole + r % a.rest;
            if (kSum && a.join) {
                q.part = r;
                q.kb0 = min(kb_total, r / a.rest * a.kb_per_split);
                q.kb1 = min(kb_total, q.kb0 + a.kb_per_split);
            }
        }
        place(a, tile, q.m0, q.n0);
        return q;
    };

    // With sums a thread of the epilogue needs more registers than there are for all: of 384 x 168 at launch, 128 x 72 + 256 x 208.
    if (warp < kFirstEpi<kSum>) {
        if constexpr (kSum) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp == 0) {
            if (lane == 0) {                             // ---- TMA producer
                uint32_t st = 0, round = 0;
                for (int it = pair; it < items && !*failed; it += pairs) {
                    const Item q = item_of(it);
                    for (int kb = q.kb0; kb < q.kb1; ++kb) {
                        if (round > 0 && !mbar_wait(&s.empty[st], (round - 1) & 1)) { *failed = 1; break; }
                        if (rank == 0) mbar_expect_tx(&s.full[st], 4 * kHalf);
                        load_operand<kAMn>(s.a[st], &tm_a, q.m0 + rank * 128, kb * kTK, &s.full[st]);
                        load_operand<kBMn>(s.b[st], &tm_b, q.n0 + rank * 128, kb * kTK, &s.full[st]);
                        if (++st == kStages) { st = 0; ++round; }
                    }
                }
                if (*failed && rank == 0)                // copies in flight land before the CTAs' shared memory is released
                    for (uint32_t i = 0; i < kStages; ++i) mbar_wait(&s.full[i], (round + (i < st ? 0u : 1u)) & 1u, 4096u);
            }
        } else if (warp == 1) {
            if (lane == 0 && rank == 0) {                // ---- MMA issuer
                constexpr uint32_t idesc = umma_idesc_bf16(kTM, kTN) | (kAMn ? 1u << 15 : 0u) | (kBMn ? 1u << 16 : 0u);
                uint32_t st = 0, phase = 0;
                int i = 0;                               // segments so far: every other one in the same accumulator
                bool ok = true;
                for (int it = pair; it < items && ok; it += pairs) {
                    const Item q = item_of(it);
                    for (int kb0 = q.kb0; kb0 < q.kb1 && ok; kb0 += kSegmentRuns<T>, ++i) {
                        const int ab = i & 1, kb1 = min(q.kb1, kb0 + kSegmentRuns<T>);
                        if (i >= 2 && !mbar_wait(&s.acc_empty[ab], ((i / 2) - 1) & 1)) { ok = false; break; }
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        for (int kb = kb0; kb < kb1; ++kb) {
                            if (!mbar_wait(&s.full[st], phase)) { ok = false; break; }
                            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                            const uint32_t a0 = smem_u32(s.a[st]), b0 = smem_u32(s.b[st]);
    #pragma unroll
                            for (int k = 0; k < kTK / 16; ++k)
                                umma2_bf16(tmem + ab * kTN, operand_desc<kAMn>(a0, k), operand_desc<kBMn>(b0, k), idesc, kb > kb0 || k > 0);
                            umma2_commit(&s.empty[st]);
                            if (++st == kStages) { st = 0; phase ^= 1u; }
                        }
                        if (ok) umma2_commit(&s.acc_full[ab]);
                    }
                }
                if (!ok) *failed = 1;
            }
            __syncwarp();
        }
    } else {                                         // ---- epilogue: four warps for the rows, kCols columns each
        if constexpr (kSum) asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        const int qd = warp % 4, part_col = (warp - kFirstEpi<kSum>) / 4 * kCols;
        float* stage = s.out[warp - kFirstEpi<kSum>];
        const int row = rank * 128 + qd * 32;        // of the tile
        const uint32_t lanes = tmem + ((uint32_t)(qd * 32) << 16) + (uint32_t)part_col;
        int i = 0;
        bool ok = true;
        for (int it = pair; it < items && ok; it += pairs) {
            const Item q = item_of(it);
            float* part = kSum && q.part >= 0 ? a.part + ((size_t)q.part * kTM + row) * kTN + part_col : nullptr;
            const int rows = min(32, a.M - (q.m0 + row)), col0 = q.n0 + part_col, cols = min(kCols, a.N - col0);
            using Work = Finish<kEpi, kAct, T, 16>;  // 16 columns at a time
            const bool mine = lane < rows;           // a thread has a row of the tile
            auto whole = [&](int c) { return a.wide && !part && c * 16 + 16 <= cols; };
            auto load = [&](Work& f, int c) {
                if (whole(c) && mine) f.load(a, q.m0 + row + lane, col0 + c * 16);
            };
            // the 16 columns of chunk c
            auto emit = [&](Work& f, int c, float2 (&v)[8]) {
                if (c * 16 >= cols) return;
                if (part) {
                    if (mine)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            *reinterpret_cast<float4*>(part + (size_t)lane * kTN + c * 16 + 4 * j) = make_float4(v[2 * j].x, v[2 * j].y, v[2 * j + 1].x, v[2 * j + 1].y);
                } else if (whole(c)) {
                    if (mine) f(a, q.m0 + row + lane, col0 + c * 16, v);
                } else {                             // a column a thread, two rows at a time, through the staging tile
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        *reinterpret_cast<float4*>(stage + lane * kPitch + 4 * j) = make_float4(v[2 * j].x, v[2 * j].y, v[2 * j + 1].x, v[2 * j + 1].y);
                    __syncwarp();
                    const int col = col0 + c * 16 + lane % 16;
                    if (c * 16 + lane % 16 < cols) {
                        const float bias = kEpi == kForward && a.bias ? __ldg(a.bias + col) : 0.f;
                        constexpr int kRows = kSum || (kEpi == kDgrad && kAct != ABS_ACT_NONE) ? 8 : 16;
#pragma unroll 1
                        for (int k0 = lane / 16; k0 < rows; k0 += 2 * kRows) {
                            FinishOne<kEpi, kAct, T> one[kRows];     // the reads of as many rows are in flight together
#pragma unroll
                            for (int k = 0; k < kRows; ++k)
                                if (k0 + 2 * k < rows) one[k].load(a, q.m0 + row + k0 + 2 * k, col);
#pragma unroll
                            for (int k = 0; k < kRows; ++k)
                                if (k0 + 2 * k < rows) one[k](a, q.m0 + row + k0 + 2 * k, col, bias, stage[(k0 + 2 * k) * kPitch + lane % 16]);
                        }
                    }
                    __syncwarp();
                }
            };
            if constexpr (kSum) {
                float2 sum[kCols / 16][8];
#pragma unroll
                for (int c = 0; c < kCols / 16; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum[c][j] = both(0.f);
                for (int kb0 = q.kb0; kb0 < q.kb1; kb0 += kSegmentRuns<T>, ++i) {
                    const int ab = i & 1;
                    ok = __all_sync(0xffffffffu, mbar_wait(&s.acc_full[ab], (i / 2) & 1) && !*failed);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                    for (int c = 0; c < kCols / 16; c += 2) {
                        uint32_t v[32];
                        tmem_ld_32(lanes + (uint32_t)(ab * kTN + c * 16), v);
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            sum[c + j / 8][j % 8] = add2(sum[c + j / 8][j % 8], make_float2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1])));
                    }
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) arrive_first(&s.acc_empty[ab]);
                }
                if (!ok) break;
                Work f, next;
                load(f, 0);
#pragma unroll
                for (int c = 0; c < kCols / 16; ++c) {
                    if (c + 1 < kCols / 16) load(next, c + 1);
                    emit(f, c, sum[c]);
                    f = next;
                }
            } else {
                const int ab = i & 1;
                Work f, next;
                load(f, 0);                       // while the product runs
                ok = __all_sync(0xffffffffu, mbar_wait(&s.acc_full[ab], (i / 2) & 1) && !*failed);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                for (int c = 0; c < kCols / 16; ++c) {
                    uint32_t u[16];
                    tmem_ld_16(lanes + (uint32_t)(ab * kTN + c * 16), u);
                    if (c == kCols / 16 - 1) {
                        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) arrive_first(&s.acc_empty[ab]);
                    } else {
                        load(next, c + 1);
                    }
                    float2 v[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = make_float2(__uint_as_float(u[2 * j]), __uint_as_float(u[2 * j + 1]));
                    emit(f, c, v);
                    f = next;
                }
                ++i;
            }
        }
        if (!ok) *failed = 1;
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    cluster_sync();                                  // no CTA leaves while the other's arrivals or MMAs may still reach it
    if constexpr (kSum) {
        if (*failed) gave_up(a);
    } else {
        if (threadIdx.x == 0 && *failed) report_timeout();
    }
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

__device__ __forceinline__ bool no_number(const float2 (&v)[4]) {
    const float2 s = add2(add2(v[0], v[1]), add2(v[2], v[3]));
    return s.x != s.x || s.y != s.y;
}
// The tiles that were cut: their partial sums added up in order; where one is missing (the sum is a NaN then) nothing is written.  A warp per row of a
// tile: eight columns a thread, or, where rows are not aligned, every 32nd one.
template <int kEpi, uint32_t kAct, typename T>
__global__ void __launch_bounds__(256) k_linear_join(const __grid_constant__ LinArgs a) {
    pdl_wait();
    pdl_trigger();
    const size_t step = (size_t)a.rest * kTM * kTN;
    const int lane = threadIdx.x % 32;
    for (int i = blockIdx.x * 8 + threadIdx.x / 32; i < a.rest * kTM; i += gridDim.x * 8) {
        int m0, n0;
        place(a, a.whole + i / kTM, m0, n0);
        const int row = m0 + i % kTM;
        if (row >= a.M) continue;
        const float* from = a.part + (size_t)i * kTN;
        if (a.wide && n0 + kTN <= a.N) {
            const int col = n0 + lane * 8;
            const float* p = from + lane * 8;
            Finish<kEpi, kAct, T, 8> f;
            f.load(a, row, col);
            float2 v[4] = {};
#pragma unroll 4
            for (int k = 0; k < a.splits; ++k) {
                const float4 lo = *reinterpret_cast<const float4*>(p + k * step), hi = *reinterpret_cast<const float4*>(p + k * step + 4);
                v[0] = add2(v[0], make_float2(lo.x, lo.y));
                v[1] = add2(v[1], make_float2(lo.z, lo.w));
                v[2] = add2(v[2], make_float2(hi.x, hi.y));
                v[3] = add2(v[3], make_float2(hi.z, hi.w));
            }
            if (no_number(v)) {
                bool missing = false;
#pragma unroll 1
                for (int k = 0; k < a.splits * 8; ++k) missing = missing || unformed(p[k / 8 * step + k % 8]);
                if (missing) continue;
            }
            f(a, row, col, v);
            continue;
        }
        const int n = min(kTN, a.N - n0);
        FinishOne<kEpi, kAct, T> one[8];
        float v[8] = {};
#pragma unroll
        for (int c = 0; c < 8; ++c)
            if (c * 32 + lane < n) one[c].load(a, row, n0 + c * 32 + lane);
        for (int k = 0; k < a.splits; ++k)
#pragma unroll
            for (int c = 0; c < 8; ++c)
                if (c * 32 + lane < n) v[c] += from[k * step + c * 32 + lane];
        uint32_t missing = 0;                        // a bit per column
        const float all = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        if (all != all)
#pragma unroll 1
            for (int k = 0; k < a.splits * 8; ++k)
                if (k % 8 * 32 + lane < n && unformed(from[k / 8 * step + k % 8 * 32 + lane])) missing |= 1u << k % 8;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const int col = n0 + c * 32 + lane;
            if (c * 32 + lane < n && !(missing >> c & 1)) one[c](a, row, col, kEpi == kForward && a.bias ? a.bias[col] : 0.f, v[c]);
        }
    }
}

// Rows that TMA cannot start at, copied to rows of `to_ld` elements (16-byte aligned), a CTA per row.
__global__ void __launch_bounds__(128) k_copy_rows(const bf16* x, size_t ld, int width, size_t to_ld, size_t rows, bf16* to) {
    pdl_wait();
    pdl_trigger();
    for (size_t t = blockIdx.x; t < rows; t += gridDim.x) {
        const uint16_t* from = reinterpret_cast<const uint16_t*>(x + t * ld);
#pragma unroll 2
        for (int c = threadIdx.x * 8; c < width; c += 1024) {
            uint32_t v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = c + k < width ? from[c + k] : 0u;
            *reinterpret_cast<uint4*>(to + t * to_ld + c) = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
        }
    }
}

// n (1 .. 8) elements of a row, zeros behind them.
__device__ __forceinline__ void load_row(Piece<bf16, 8>& w, const bf16* p, int n, bool wide) {
    if (wide && n == 8) return w.load(p, false);
    uint32_t v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < n ? reinterpret_cast<const uint16_t*>(p)[i] : 0u;
    w.w[0] = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
}
// Column sums of dy over the rows of a CTA: 256 columns, every gridDim.y-th group of eight rows.  launch_column_sums adds them up.
__global__ void __launch_bounds__(256) k_bias_part(const bf16* dy, size_t ld, int T, int N, int wide, float* part, size_t part_ld) {
    __shared__ float sh[8][264];
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, col = blockIdx.x * 256 + lane * 8, n = min(8, N - col);
    float2 sum[4] = {};
    const int64_t step = (int64_t)gridDim.y * 8;
    for (int64_t t = (int64_t)blockIdx.y * 8 + warp; t < T && n > 0; t += 8 * step) {
        Piece<bf16, 8> w[8];                         // eight rows in flight
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            w[k].w[0] = make_uint4(0, 0, 0, 0);
            if (t + k * step >= T) continue;
            load_row(w[k], dy + (size_t)(t + k * step) * ld + col, n, wide != 0);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float2 v[4];
            w[k].get(v);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = add2(sum[i], v[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<float2*>(&sh[warp][lane * 8 + 2 * i]) = sum[i];
    __syncthreads();
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= N) return;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) v += sh[w][threadIdx.x];
    part[(size_t)blockIdx.y * 2 * part_ld + c] = v;
}

// All rows, 64 columns a CTA, in one launch: up to kFewRows rows, where a second launch costs more than the rows that a thread has one after the other.
constexpr int kFewRows = 1024;
__global__ void __launch_bounds__(256) k_bias_few(const bf16* dy, size_t ld, int T, int N, int wide, float* db, int accumulate) {
    __shared__ float sh[32][72];
    pdl_wait();
    pdl_trigger();
    const int piece = threadIdx.x % 8, line = threadIdx.x / 8, col = blockIdx.x * 64 + piece * 8, n = min(8, N - col);
    float2 sum[4] = {};
    for (int t = line; t < T && n > 0; t += 8 * 32) {
        Piece<bf16, 8> w[8];                         // eight rows in flight
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            w[k].w[0] = make_uint4(0, 0, 0, 0);
            if (t + k * 32 < T) load_row(w[k], dy + (size_t)(t + k * 32) * ld + col, n, wide != 0);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float2 v[4];
            w[k].get(v);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = add2(sum[i], v[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<float2*>(&sh[line][piece * 8 + 2 * i]) = sum[i];
    __syncthreads();
    const int c = blockIdx.x * 64 + threadIdx.x;
    if (threadIdx.x >= 64 || c >= N) return;
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) v += sh[i][threadIdx.x];
    db[c] = accumulate ? db[c] + v : v;
}

template <uint32_t kAct, typename T>
__global__ void __launch_bounds__(256) k_activation_backward(const T* dy, size_t ld_dy, const bf16* z, size_t ld_z, size_t rows, int width, int wide, bf16* dz, size_t ld_dz) {
    pdl_wait();
    pdl_trigger();
    const size_t per_row = ((size_t)width + 7) / 8;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < rows * per_row; i += (size_t)gridDim.x * 256) {
        const size_t t = rows * per_row >> 32 ? i / per_row : (uint32_t)i / (uint32_t)per_row;
        const int c = (int)(i - t * per_row) * 8, n = min(8, width - c);
        const T* p = dy + t * ld_dy + c;
        const bf16* q = z + t * ld_z + c;
        bf16* o = dz + t * ld_dz + c;
        if (wide && n == 8) {
            Piece<T, 8> g;
            Piece<bf16, 8> w;
            float2 v[4], u[4];
            g.load(p, false);
            w.load(q, false);
            g.get(v);
            w.get(u);
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = mul2(v[k], slope<kAct, false>(u[k]));
            w.put(v);
            w.store(o, false);
        } else {
            for (int k = 0; k < n; ++k) o[k] = __float2bfloat16_rn(to_f(p[k]) * slope<kAct, false>(both(__bfloat162float(q[k]))).x);
        }
    }
}

// How the work is cut: whole output tiles for all pairs equally often, the rest in runs of K.
struct LinPlan {
    int tiles_m, tiles_n, whole, rest, splits, kb_per_split;
    int join_splits, join_kb;        // how K is cut where few tiles have to go through k_linear_join; 0: they have not
    bool pack_a, pack_b;
    uint64_t ld_a, ld_b;             // of the packed copies
    size_t part_bytes, a_bytes, b_bytes, bias_bytes;
    int bias_parts;
    size_t bytes() const { return part_bytes + a_bytes + b_bytes + bias_bytes; }
};
// An operand as it lies in memory: rows of `cols` elements.
struct Operand {
    const void* p;
    uint64_t ld, rows, cols;
};
bool tma_ready(const Operand& o) { return !misaligned(o.p, 16) && o.ld % 8 == 0; }
bool plan_of(uint64_t M, uint64_t N, uint64_t K, const Operand& a, const Operand& b, LinPlan* out) {
    LinPlan p{};
    p.tiles_m = (int)((M + kTM - 1) / kTM);
    p.tiles_n = (int)((N + kTN - 1) / kTN);
    const int kb = (int)((K + kTK - 1) / kTK), pairs = kSms / 2;
    const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
    if (tiles > 0x3fffffff) return false;
    p.whole = (int)(tiles / pairs * pairs);
    p.rest = (int)(tiles - p.whole);
    auto cut = [&](int min_runs, int* splits, int* per) {
        const int want = p.rest ? std::max(1, std::min(pairs / p.rest, kb / min_runs)) : 1;
        *per = std::max(1, (kb + want - 1) / want);
        *splits = std::max(1, (kb + *per - 1) / *per);
    };
    cut(kMinRuns, &p.splits, &p.kb_per_split);
    if (tiles <= kFewTiles) cut(kMinRunsJoin, &p.join_splits, &p.join_kb);
    const int parts = std::max(p.splits > 1 ? p.splits : 0, p.join_splits);
    p.part_bytes = (size_t)parts * p.rest * kTM * kTN * 4;
    p.pack_a = !tma_ready(a);
    p.pack_b = !tma_ready(b);
    p.ld_a = (a.cols + 7) / 8 * 8;
    p.ld_b = (b.cols + 7) / 8 * 8;
    p.a_bytes = p.pack_a ? up256(a.rows * p.ld_a * 2) : 0;
    p.b_bytes = p.pack_b ? up256(b.rows * p.ld_b * 2) : 0;
    *out = p;
    return true;
}
int bias_parts(uint64_t T, uint64_t N) {
    const uint64_t blocks = (N + 255) / 256, want = std::max<uint64_t>(1, 2 * kSms / blocks);
    return (int)std::max<uint64_t>(1, std::min((T + 63) / 64, want));
}

// Whole tiles of no more runs than the tensor core adds up on its own.
bool one_segment(const LinArgs& a) { return !a.join && (a.K + kTK - 1) / kTK <= kSegmentRuns<bf16>; }

cudaError_t copy_rows(const Operand& o, uint64_t to_ld, bf16* to, cudaStream_t s) {
    return launch_kernel(k_copy_rows, (int)std::min<size_t>(o.rows, kSms * 16), 128, 0, s, true, static_cast<const bf16*>(o.p), (size_t)o.ld, (int)o.cols, (size_t)to_ld,
                         (size_t)o.rows, to);
}

template <int kEpi, uint32_t kAct, typename T, bool kSum>
cudaError_t run_tiles(const CUtensorMap& ta, const CUtensorMap& tb, const LinArgs& a, cudaStream_t s) {
    const cudaError_t e = allow_smem<k_linear<kEpi, kAct, T, kSum>>();
    if (e != cudaSuccess) return e;
    const int grid = 2 * std::min(a.whole + a.rest * a.splits, kSms / 2);
    return launch_cluster(k_linear<kEpi, kAct, T, kSum>, grid, 2, kThreads<kSum>, sizeof(LinSmem) + 1024, s, ta, tb, a);
}
template <int kEpi, uint32_t kAct, typename T>
cudaError_t run_act(const CUtensorMap& ta, const CUtensorMap& tb, const LinArgs& a, cudaStream_t s) {
    cudaError_t e;
    if constexpr (sizeof(T) == 2) e = one_segment(a) ? run_tiles<kEpi, kAct, T, false>(ta, tb, a, s) : run_tiles<kEpi, kAct, T, true>(ta, tb, a, s);
    else e = run_tiles<kEpi, kAct, T, true>(ta, tb, a, s);
    if (e == cudaSuccess && a.join) e = launch_kernel(k_linear_join<kEpi, kAct, T>, std::min(a.rest * kTM / 8, kSms * 8), 256, 0, s, false, a);
    return e;
}
template <int kEpi, typename T>
cudaError_t run(uint32_t act, const CUtensorMap& ta, const CUtensorMap& tb, const LinArgs& a, cudaStream_t s) {
    switch (act) {
        case ABS_ACT_RELU: return run_act<kEpi, ABS_ACT_RELU, T>(ta, tb, a, s);
        case ABS_ACT_GELU: return run_act<kEpi, ABS_ACT_GELU, T>(ta, tb, a, s);
        case ABS_ACT_SILU: return run_act<kEpi, ABS_ACT_SILU, T>(ta, tb, a, s);
        default: return run_act<kEpi, ABS_ACT_NONE, T>(ta, tb, a, s);
    }
}

// The product and its epilogue; `kind`: kForward, kDgrad, kWgrad; workspace checked against `p`.
int product(int kind, uint32_t act, uint32_t dtype, Operand oa, Operand ob, uint64_t M, uint64_t N, uint64_t K, const LinPlan& p, LinArgs a, char* ws, cudaStream_t s) {
    cudaError_t e = cudaSuccess;
    if (p.pack_a) {
        bf16* to = reinterpret_cast<bf16*>(ws + p.part_bytes);
        e = copy_rows(oa, p.ld_a, to, s);
        oa.p = to; oa.ld = p.ld_a;
    }
    if (p.pack_b && e == cudaSuccess) {
        bf16* to = reinterpret_cast<bf16*>(ws + p.part_bytes + p.a_bytes);
        e = copy_rows(ob, p.ld_b, to, s);
        ob.p = to; ob.ld = p.ld_b;
    }
    if (e != cudaSuccess) return thread_error(ABS_ECUDA, cudaGetErrorString(e));
    CUtensorMap ta, tb;
    const uint32_t rows_a = kind == kWgrad ? kTK : 128, rows_b = kind == kDgrad ? 128 : kTK;
    if (!encode_2d(&ta, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(oa.p), oa.rows, oa.cols, rows_a, 64, oa.ld) ||
        !encode_2d(&tb, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(ob.p), ob.rows, ob.cols, rows_b, 64, ob.ld))
        return thread_error(ABS_ECUDA, "cuTensorMapEncodeTiled failed");
    a.M = (int)M; a.N = (int)N; a.K = (int)K;
    a.tiles_m = p.tiles_m; a.tiles_n = p.tiles_n; a.whole = p.whole; a.rest = p.rest; a.splits = p.splits; a.kb_per_split = p.kb_per_split;
    a.join = p.splits > 1;
    const bool reads = kind == kWgrad ? a.accumulate != 0 : a.res || a.z_in;
    if (!a.wide && reads && p.join_splits) {
        a.splits = p.join_splits;
        a.kb_per_split = p.join_kb;
        a.join = 1;
    }
    a.part = reinterpret_cast<float*>(ws);
    if (kind == kForward) e = dtype == ABS_F32 ? run<kForward, float>(act, ta, tb, a, s) : run<kForward, bf16>(act, ta, tb, a, s);
    else if (kind == kDgrad) e = dtype == ABS_F32 ? run<kDgrad, float>(act, ta, tb, a, s) : run<kDgrad, bf16>(act, ta, tb, a, s);
    else e = run_act<kWgrad, ABS_ACT_NONE, float>(ta, tb, a, s);
    return e == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(e));
}

const char* check_sizes(uint64_t tokens, uint64_t in, uint64_t out, uint32_t dtype, uint32_t act, int* code) {
    *code = ABS_EINVAL;
    if (!known_dtype(dtype)) return "dtype must be ABS_F32 or ABS_BF16";
    if (act > ABS_ACT_SILU) return "unknown activation";
    if (in == 0 || out == 0) return "in and out must be at least 1";
    if (tokens <= kSizeMax && in <= kSizeMax && out <= kSizeMax) return nullptr;
    *code = ABS_ELIMIT;
    return "a size exceeds 2^31 - 64";
}
// What the rows of these matrices are aligned to: 32, 16 bytes, or 0.
int alignment(std::initializer_list<MatrixArg> all) {
    int to = 32;
    for (const MatrixArg& m : all)
        while (to && !rows_at(m, to)) to = to == 32 ? 16 : 0;
    return to;
}
// An operand of the product must not be an output.
const char* check_operands(const void* const (&out)[2], const void* a, const void* b) {
    for (const void* o : out)
        if (o && (o == a || o == b)) return "an output must not be an operand of the product";
    return out[0] && out[0] == out[1] ? "two outputs are the same" : nullptr;
}
const char* check_workspace(const LinPlan& p, const void* workspace, size_t bytes, int* code) {
    *code = ABS_EINVAL;
    if (p.bytes() == 0) return nullptr;
    if (!workspace || misaligned(workspace, 256)) return "workspace must be non-NULL and 256-byte aligned";
    *code = ABS_ENOMEM;
    return bytes < p.bytes() ? "workspace too small" : nullptr;
}

}  // namespace

cudaError_t take_status_linear(int* status, cudaStream_t s) { return take_status(status, s); }

}  // namespace abs_sgd

using namespace abs_sgd;

extern "C" size_t abs_linear_workspace(uint64_t tokens, uint64_t in, uint64_t out, const void* x, uint64_t ld_x, const void* w, uint64_t ld_w) {
    LinPlan p;
    if (tokens == 0 || tokens > kSizeMax || in > kSizeMax || out > kSizeMax) return 0;
    return plan_of(tokens, out, in, {x, ld_x, tokens, in}, {w, ld_w, in, out}, &p) ? p.bytes() : 0;
}

extern "C" int abs_linear(const void* x, uint64_t ld_x, const void* w, uint64_t ld_w, const float* bias, uint32_t act, const void* residual, uint64_t ld_residual,
                          uint32_t dtype, uint64_t tokens, uint64_t in, uint64_t out, void* y, uint64_t ld_y, void* z, uint64_t ld_z, void* workspace,
                          size_t workspace_bytes, void* stream) {
    int code = 0;
    if (const char* why = check_sizes(tokens, in, out, dtype, act, &code)) return thread_error(code, why);
    const size_t es = size_of(dtype);
    const MatrixArg m[5] = {{x, ld_x, in, 2}, {w, ld_w, out, 2}, {residual, ld_residual, out, es}, {y, ld_y, out, es}, {z, ld_z, out, 2}};
    if (const char* why = check_matrices(m)) return thread_error(ABS_EINVAL, why);
    if (misaligned(bias, 4)) return thread_error(ABS_EINVAL, "bias must be 4-byte aligned");
    if (tokens == 0) return ABS_OK;
    if (!x || !w || !y) return thread_error(ABS_EINVAL, "x, w and y must not be NULL");
    if (const char* why = check_operands({y, z}, x, w)) return thread_error(ABS_EINVAL, why);
    if (const char* why = check_in_place(m[3], m[2], true)) return thread_error(ABS_EINVAL, why);
    if (const char* why = check_in_place(m[4], m[2], false)) return thread_error(ABS_EINVAL, why);
    LinPlan p;
    const Operand oa{x, ld_x, tokens, in}, ob{w, ld_w, in, out};
    if (!plan_of(tokens, out, in, oa, ob, &p)) return thread_error(ABS_ELIMIT, "too many output tiles");
    if (const char* why = check_workspace(p, workspace, workspace_bytes, &code)) return thread_error(code, why);
    LinArgs a{};
    a.out = y; a.ld = ld_y; a.bias = bias; a.res = residual; a.ld_res = ld_residual; a.z_out = static_cast<bf16*>(z); a.ld_z = ld_z;
    a.wide = alignment({m[2], m[3], m[4]});
    return product(kForward, act, dtype, oa, ob, tokens, out, in, p, a, static_cast<char*>(workspace), static_cast<cudaStream_t>(stream));
}

extern "C" size_t abs_linear_dgrad_workspace(uint64_t tokens, uint64_t in, uint64_t out, const void* dy, uint64_t ld_dy, const void* w, uint64_t ld_w) {
    LinPlan p;
    if (tokens == 0 || tokens > kSizeMax || in > kSizeMax || out > kSizeMax) return 0;
    return plan_of(tokens, in, out, {dy, ld_dy, tokens, out}, {w, ld_w, in, out}, &p) ? p.bytes() : 0;
}

extern "C" int abs_linear_dgrad(const void* dy, uint64_t ld_dy, const void* w, uint64_t ld_w, uint32_t act, const void* z, uint64_t ld_z, const void* residual,
                                uint64_t ld_residual, uint32_t dtype, uint64_t tokens, uint64_t in, uint64_t out, void* dx, uint64_t ld_dx, void* workspace,
                                size_t workspace_bytes, void* stream) {
    int code = 0;
    if (const char* why = check_sizes(tokens, in, out, dtype, act, &code)) return thread_error(code, why);
    const size_t es = size_of(dtype);
    const MatrixArg m[5] = {{dy, ld_dy, out, 2}, {w, ld_w, out, 2}, {z, ld_z, in, 2}, {residual, ld_residual, in, es}, {dx, ld_dx, in, es}};
    if (const char* why = check_matrices(m)) return thread_error(ABS_EINVAL, why);
    if (tokens == 0) return ABS_OK;
    if ((act != ABS_ACT_NONE) != (z != nullptr)) return thread_error(ABS_EINVAL, "z must be given exactly with an activation");
    if (!dy || !w || !dx) return thread_error(ABS_EINVAL, "dy, w and dx must not be NULL");
    if (const char* why = check_operands({dx, nullptr}, dy, w)) return thread_error(ABS_EINVAL, why);
    for (int i = 2; i < 4; ++i)
        if (const char* why = check_in_place(m[4], m[i], true)) return thread_error(ABS_EINVAL, why);
    LinPlan p;
    const Operand oa{dy, ld_dy, tokens, out}, ob{w, ld_w, in, out};
    if (!plan_of(tokens, in, out, oa, ob, &p)) return thread_error(ABS_ELIMIT, "too many output tiles");
    if (const char* why = check_workspace(p, workspace, workspace_bytes, &code)) return thread_error(code, why);
    LinArgs a{};
    a.out = dx; a.ld = ld_dx; a.res = residual; a.ld_res = ld_residual; a.z_in = static_cast<const bf16*>(z); a.ld_z = ld_z;
    a.wide = alignment({m[2], m[3], m[4]});
    return product(kDgrad, act, dtype, oa, ob, tokens, in, out, p, a, static_cast<char*>(workspace), static_cast<cudaStream_t>(stream));
}

static bool wgrad_plan(uint64_t tokens, uint64_t in, uint64_t out, const Operand& x, const Operand& dy, LinPlan* p) {
    if (!plan_of(in, out, tokens, x, dy, p)) return false;
    p->bias_parts = bias_parts(tokens, out);
    p->bias_bytes = up256((size_t)p->bias_parts * 2 * part_width(out) * 4);
    return true;
}

extern "C" size_t abs_linear_wgrad_workspace(uint64_t tokens, uint64_t in, uint64_t out, const void* x, uint64_t ld_x, const void* dy, uint64_t ld_dy) {
    LinPlan p;
    if (tokens == 0 || out == 0 || tokens > kSizeMax || in > kSizeMax || out > kSizeMax) return 0;
    return wgrad_plan(tokens, in, out, {x, ld_x, tokens, in}, {dy, ld_dy, tokens, out}, &p) ? p.bytes() : 0;
}

extern "C" int abs_linear_wgrad(const void* x, uint64_t ld_x, const void* dy, uint64_t ld_dy, uint64_t tokens, uint64_t in, uint64_t out, float* dw, uint64_t ld_dw,
                                float* db, int accumulate, void* workspace, size_t workspace_bytes, void* stream) {
    int code = 0;
    if (const char* why = check_sizes(tokens, in, out, ABS_F32, ABS_ACT_NONE, &code)) return thread_error(code, why);
    const MatrixArg m[3] = {{x, ld_x, in, 2}, {dy, ld_dy, out, 2}, {dw, ld_dw, out, 4}};
    if (const char* why = check_matrices(m)) return thread_error(ABS_EINVAL, why);
    if (!dw || misaligned(db, 4)) return thread_error(ABS_EINVAL, "dw must not be NULL, db 4-byte aligned");
    if (dw == db) return thread_error(ABS_EINVAL, "two outputs are the same");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaSuccess;
    if (tokens == 0) {
        if (!accumulate) {
            e = cudaMemset2DAsync(dw, ld_dw * 4, 0, out * 4, in, s);
            if (e == cudaSuccess && db) e = cudaMemsetAsync(db, 0, out * 4, s);
        }
        return e == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(e));
    }
    if (!x || !dy) return thread_error(ABS_EINVAL, "x and dy must not be NULL");
    if (const char* why = check_operands({dw, db}, x, dy)) return thread_error(ABS_EINVAL, why);
    LinPlan p;
    const Operand oa{x, ld_x, tokens, in}, ob{dy, ld_dy, tokens, out};
    if (!wgrad_plan(tokens, in, out, oa, ob, &p)) return thread_error(ABS_ELIMIT, "too many output tiles");
    if (const char* why = check_workspace(p, workspace, workspace_bytes, &code)) return thread_error(code, why);
    if (db) {
        float* part = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.part_bytes + p.a_bytes + p.b_bytes);
        const unsigned blocks = (unsigned)((out + 255) / 256);
        if (tokens <= (uint64_t)kFewRows)
            e = launch_kernel(k_bias_few, (unsigned)((out + 63) / 64), 256, 0, s, true, static_cast<const bf16*>(dy), (size_t)ld_dy, (int)tokens, (int)out, (int)tma_ready(ob), db,
                              accumulate);
        else
            e = launch_kernel(k_bias_part, dim3(blocks, p.bias_parts), 256, 0, s, true, static_cast<const bf16*>(dy), (size_t)ld_dy, (int)tokens, (int)out, (int)tma_ready(ob), part,
                          part_width(out));
        if (e == cudaSuccess && tokens > (uint64_t)kFewRows) e = launch_column_sums(part, p.bias_parts, (int)out, db, nullptr, accumulate, s);
        if (e != cudaSuccess) return thread_error(ABS_ECUDA, cudaGetErrorString(e));
    }
    LinArgs a{};
    a.out = dw; a.ld = ld_dw; a.accumulate = accumulate != 0; a.wide = alignment({m[2]});
    return product(kWgrad, ABS_ACT_NONE, ABS_F32, oa, ob, in, out, tokens, p, a, static_cast<char*>(workspace), s);
}

extern "C" int abs_activation_backward(const void* dy, uint64_t ld_dy, uint32_t dtype, const void* z, uint64_t ld_z, uint32_t act, uint64_t tokens, uint64_t width,
                                       void* dz, uint64_t ld_dz, void* stream) {
    int code = 0;
    if (const char* why = check_sizes(tokens, width, 1, dtype, act, &code)) return thread_error(code, why);
    const MatrixArg m[3] = {{dy, ld_dy, width, size_of(dtype)}, {z, ld_z, width, 2}, {dz, ld_dz, width, 2}};
    if (const char* why = check_matrices(m)) return thread_error(ABS_EINVAL, why);
    for (int i = 0; i < 2; ++i)
        if (const char* why = check_in_place(m[2], m[i], true)) return thread_error(ABS_EINVAL, why);
    if (tokens == 0) return ABS_OK;
    if (!dy || !z || !dz) return thread_error(ABS_EINVAL, "dy, z and dz must not be NULL");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int wide = rows_at(m[0], 16) && rows_at(m[1], 16) && rows_at(m[2], 16);
    const size_t want = ((size_t)tokens * ((width + 7) / 8) + 511) / 512;
    const int grid = (int)std::min<size_t>(want, kSms * 8);
    auto go = [&](auto kernel, auto zero) {
        return launch_kernel(kernel, grid, 256, 0, s, true, static_cast<const decltype(zero)*>(dy), (size_t)ld_dy, static_cast<const bf16*>(z), (size_t)ld_z, (size_t)tokens,
                             (int)width, wide, static_cast<bf16*>(dz), (size_t)ld_dz);
    };
    auto with = [&](auto zero) {
        using T = decltype(zero);
        return act == ABS_ACT_RELU ? go(k_activation_backward<ABS_ACT_RELU, T>, zero) : act == ABS_ACT_GELU ? go(k_activation_backward<ABS_ACT_GELU, T>, zero)
             : act == ABS_ACT_SILU ? go(k_activation_backward<ABS_ACT_SILU, T>, zero) : go(k_activation_backward<ABS_ACT_NONE, T>, zero);
    };
    const cudaError_t e = dtype == ABS_F32 ? with(0.f) : with(bf16());
    return e == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(e));
}
