// Activations held in 8 bits between the forward and the backward pass (abs_ckpt8_*).
//
// A block of 32 consecutive values of a row: int8 q and one power of two, value = q 2^(e - 127), the smallest e with
// amax <= 127 2^(e - 127).  int8 and not an 8-bit float: inside a block of 32 an activation's values are within a few
// octaves of its largest, where 7 bits of magnitude below the block's maximum are 3 to 4 times as fine (rms) as a
// 3-bit mantissa.  A power of two and not amax / 127: q 2^k is exactly a bf16 number (7 significant bits), so that the
// weight gradient feeds it to the bf16 tensor cores without a rounding of its own.
#include <algorithm>

#include "abs_internal.h"
#include "abs_llm.h"
#include "llm_status.cuh"
#include "row_ops.cuh"
#include "tcgen05.cuh"

namespace abs_sgd {
namespace {

// Exponent byte of a block from the bits of its largest magnitude (a NaN's bits are above infinity's).
__device__ __forceinline__ uint32_t block_exponent(uint32_t amax_bits) {
    const uint32_t field = amax_bits >> 23;
    if (field == 255u) return 255u;
    // amax = 1.f 2^(field - 127) <= 127 2^k = 1.984375 2^(6 + k)
    const int e = (int)field - 6 + ((amax_bits & 0x7FFFFFu) > 0x7E0000u ? 1 : 0);
    return e < 0 ? 0u : (uint32_t)e;
}
// 2^(e - 127) and its reciprocal; e = 255: NaN.
__device__ __forceinline__ float pow2_of(uint32_t e) {
    return __uint_as_float(e == 0u ? 0x00400000u : e == 255u ? 0x7FC00000u : e << 23);
}
__device__ __forceinline__ float inv_pow2_of(uint32_t e) { return __uint_as_float((254u - e) << 23); }   // e <= 249

// n / d and n % d by a multiplication, for n < 2^31 (d >= 1); larger ranges take the division.
struct Divide {
    uint32_t d, mul, shift;
    int small;               // all n that are asked for are below 2^31
};
__device__ __forceinline__ size_t divide(size_t n, const Divide& v, uint32_t* rest) {
    if (v.small) {
        const uint32_t m = (uint32_t)n, q = v.d == 1u ? m : __umulhi(m, v.mul) >> v.shift;
        *rest = m - q * v.d;
        return q;
    }
    const size_t q = n / v.d;
    *rest = (uint32_t)(n - q * v.d);
    return q;
}

struct PackArgs {
    size_t ld, T;
    int D;
    int pieces;              // of eight values in a stored row: W / 8
    Divide per_row;          // by the units of a row
    size_t units;
};
constexpr int kUnroll = 4;   // units whose loads are issued together

__device__ __forceinline__ uint4 bits_of(const float* v) { return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])); }
__device__ __forceinline__ uint4 bits_of(const bf16* v) {
    auto two = [&](int k) { return (uint32_t)__bfloat16_as_ushort(v[k]) | (uint32_t)__bfloat16_as_ushort(v[k + 1]) << 16; };
    return make_uint4(two(0), two(2), two(4), two(6));
}
// Bits of the largest magnitude of a piece, as those of an fp32 (integers order magnitudes; NaN comes out on top).
__device__ __forceinline__ uint32_t magnitude(uint4 r, float) {
    return max(max(r.x & 0x7FFFFFFFu, r.y & 0x7FFFFFFFu), max(r.z & 0x7FFFFFFFu, r.w & 0x7FFFFFFFu));
}
__device__ __forceinline__ uint32_t magnitude(uint4 r, bf16) {
    const uint32_t m = __vmaxu2(__vmaxu2(r.x & 0x7FFF7FFFu, r.y & 0x7FFF7FFFu), __vmaxu2(r.z & 0x7FFF7FFFu, r.w & 0x7FFF7FFFu));
    return max(m << 16, m & 0xFFFF0000u);
}

// A unit is eight values; the four lanes of a block are neighbours.  kWide: the rows allow 16-byte loads.  A block's maximum by
// two exchanges, its exponent from the maximum's bits; kUnroll units of a thread are loaded before the first is used.  Bound by
// memory: 16384 x 4096 bf16 36 us (203 MB, 31 us of memory), 8192 x 4096 fp32 27 (26); rows that no 16-byte load can start at 49.
template <typename T, bool kWide>
__global__ void __launch_bounds__(256) k_ckpt8_quantize(const T* x, const __grid_constant__ PackArgs a, uint2* q, uint8_t* e) {
    pdl_wait();
    pdl_trigger();
    // units is a multiple of 4: a block's lanes are all in or all out; all lanes of a warp stay in the loop for the exchange
    constexpr int kPacks = 8 / kVec<T>;              // 16-byte pieces of a unit
    for (size_t i0 = (size_t)blockIdx.x * 256 * kUnroll; i0 < a.units; i0 += (size_t)gridDim.x * 256 * kUnroll) {
        uint4 raw[kUnroll][kPacks];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const size_t i = i0 + u * 256 + threadIdx.x;
            uint32_t piece;
            const size_t t = divide(i < a.units ? i : 0, a.per_row, &piece);
            const int c = i < a.units ? (int)piece * 8 : a.D;
            const T* p = x + t * a.ld + c;
            if (kWide && c + 8 <= a.D) {
#pragma unroll
                for (int k = 0; k < kPacks; ++k) raw[u][k] = reinterpret_cast<const uint4*>(p)[k];
            } else {
                T v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = c + k < a.D ? p[k] : from_f<T>(0.f);
#pragma unroll
                for (int k = 0; k < kPacks; ++k) raw[u][k] = bits_of(v + k * kVec<T>);
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const size_t i = i0 + u * 256 + threadIdx.x;
            uint32_t m = 0;
#pragma unroll
            for (int k = 0; k < kPacks; ++k) m = max(m, magnitude(raw[u][k], T()));
            m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
            m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
            const uint32_t code = block_exponent(m);
            const float2 inv = both(code == 255u ? 0.f : inv_pow2_of(code));
            // the sum with 1.5 2^23 is rounded to an integer (to nearest even), whose low byte is q
            uint32_t w[2], b[8];
#pragma unroll
            for (int k = 0; k < kPacks; ++k) {
                float2 v[kPairs<T>];
                unpack(raw[u][k], v, T());
#pragma unroll
                for (int j = 0; j < kPairs<T>; ++j) {
                    const float2 r = add2(mul2(v[j], inv), both(12582912.f));
                    b[k * kVec<T> + 2 * j] = __float_as_uint(r.x);
                    b[k * kVec<T> + 2 * j + 1] = __float_as_uint(r.y);
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
                w[h] = code == 255u ? 0u : __byte_perm(__byte_perm(b[4 * h], b[4 * h + 1], 0x0040), __byte_perm(b[4 * h + 2], b[4 * h + 3], 0x0040), 0x5410);
            if (i < a.units) {
                q[i] = make_uint2(w[0], w[1]);
                if (i % 4 == 0) e[i / 4] = (uint8_t)code;
            }
        }
    }
}

// The values of kV stored bytes (raw) with exponent byte `code`, as a 16-byte piece.
template <typename T>
__device__ __forceinline__ void unpack8(const uint32_t (&raw)[kVec<T> / 4], uint32_t code, float2 (&v)[kPairs<T>]) {
    const float s = pow2_of(code);
#pragma unroll
    for (int k = 0; k < kPairs<T>; ++k) {
        const uint32_t w = raw[k / 2] ^ 0x80808080u;     // the byte q + 128 as the low mantissa byte of 2^23
        const float2 f = make_float2(__uint_as_float(__byte_perm(w, 0x4B000000u, 0x7540 + 2 * (k % 2))),
                                     __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7541 + 2 * (k % 2))));
        v[k] = mul2(add2(f, both(-8388736.f)), both(s));
    }
}

// Rows on 16-byte boundaries: a unit is one 16-byte piece of a row.  16384 x 4096 bf16: 36 us (203 MB, 31 us of memory), 8192 x 4096 fp32 32 (26).
template <typename T>
__global__ void __launch_bounds__(256) k_ckpt8_dequantize(const uint8_t* q, const uint8_t* e, T* x, const __grid_constant__ PackArgs a) {
    constexpr int kV = kVec<T>;
    const size_t width = (size_t)a.pieces * 8;           // of a stored row
    pdl_wait();
    pdl_trigger();
    for (size_t i0 = (size_t)blockIdx.x * 256 * kUnroll + threadIdx.x; i0 < a.units; i0 += (size_t)gridDim.x * 256 * kUnroll) {
        uint32_t raw[kUnroll][kV / 4], code[kUnroll], piece[kUnroll];
        size_t t[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const size_t i = i0 + u * 256;
            t[u] = divide(i < a.units ? i : 0, a.per_row, &piece[u]);
            const size_t at = t[u] * width + (size_t)piece[u] * kV;
            code[u] = e[at / 32];
            if (kV == 8) {
                const uint2 r = *reinterpret_cast<const uint2*>(q + at);
                raw[u][0] = r.x;
                raw[u][kV / 4 - 1] = r.y;
            } else raw[u][0] = *reinterpret_cast<const uint32_t*>(q + at);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            if (i0 + u * 256 >= a.units) break;
            float2 v[kPairs<T>];
            unpack8<T>(raw[u], code[u], v);
            const int c = (int)piece[u] * kV;
            T* p = x + t[u] * a.ld + c;
            if (c + kV <= a.D) *reinterpret_cast<uint4*>(p) = pack(v, T());
            else {
#pragma unroll
                for (int k = 0; k < kV; ++k)
                    if (c + k < a.D) p[k] = from_f<T>(k % 2 ? v[k / 2].y : v[k / 2].x);
            }
        }
    }
}

// Rows that start anywhere: a unit is the part of a row that kLanes lanes make together, a piece each.  The pieces are put
// down in shared memory at the offset that the part has from a 16-byte boundary in memory, and leave from there in whole
// 16-byte pieces, the ends as single elements (element stores straight from the registers took four times as long).
template <typename T, int kLanes>
__global__ void __launch_bounds__(256) k_ckpt8_dequantize_any(const uint8_t* q, const uint8_t* e, T* x, const __grid_constant__ PackArgs a) {
    constexpr int kV = kVec<T>, kGroups = 256 / kLanes, kBuf = kLanes * 16 + 16;
    __shared__ __align__(16) uint8_t buf[kGroups * kBuf];
    const int lane = threadIdx.x % kLanes;
    uint8_t* mine = buf + (threadIdx.x / kLanes) * kBuf;
    const size_t width = (size_t)a.pieces * 8;
    pdl_wait();
    pdl_trigger();
    // all lanes of a warp stay in the loop
    for (size_t g0 = (size_t)blockIdx.x * kGroups * kUnroll; g0 < a.units; g0 += (size_t)gridDim.x * kGroups * kUnroll) {
        uint32_t raw[kUnroll][kV / 4], code[kUnroll], step[kUnroll];
        size_t t[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const size_t i = g0 + u * kGroups + threadIdx.x / kLanes;
            t[u] = divide(i < a.units ? i : 0, a.per_row, &step[u]);
            const int c = ((int)step[u] * kLanes + lane) * kV;
            const size_t at = t[u] * width + (size_t)c;
#pragma unroll
            for (int k = 0; k < kV / 4; ++k) raw[u][k] = 0u;
            code[u] = 0u;
            if (c < a.D) {
                code[u] = e[at / 32];
                if (kV == 8) {
                    const uint2 r = *reinterpret_cast<const uint2*>(q + at);
                    raw[u][0] = r.x;
                    raw[u][kV / 4 - 1] = r.y;
                } else raw[u][0] = *reinterpret_cast<const uint32_t*>(q + at);
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            float2 v[kPairs<T>];
            unpack8<T>(raw[u], code[u], v);
            const uint4 out = pack(v, T());
            const uint32_t w[4] = {out.x, out.y, out.z, out.w};
            const int c0 = (int)step[u] * kLanes * kV, c1 = min(a.D, c0 + kLanes * kV);      // the part of the row
            const uintptr_t to = reinterpret_cast<uintptr_t>(x + t[u] * a.ld + c0);
            const uint32_t off = (uint32_t)(to & 15);
            uint8_t* put = mine + off + lane * 16;
            if (sizeof(T) == 4 || off % 4 == 0) {
#pragma unroll
                for (int k = 0; k < 4; ++k) reinterpret_cast<uint32_t*>(put)[k] = w[k];
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k) reinterpret_cast<uint16_t*>(put)[k] = (uint16_t)(w[k / 2] >> (16 * (k % 2)));
            }
            __syncwarp();
            if (g0 + u * kGroups + threadIdx.x / kLanes < a.units) {
                const uint32_t end = off + (uint32_t)(c1 - c0) * sizeof(T);              // in the buffer
                T* base = reinterpret_cast<T*>(to - off);
                const T* have = reinterpret_cast<const T*>(mine);
                for (uint32_t g = (uint32_t)lane * 16; g < end; g += kLanes * 16)        // at most two
                    if (g >= off && g + 16 <= end) reinterpret_cast<uint4*>(base)[g / 16] = reinterpret_cast<const uint4*>(mine)[g / 16];
                const uint32_t head = min(off ? 16u : 0u, end) / (uint32_t)sizeof(T);
                for (uint32_t k = off / sizeof(T) + lane; k < head; k += kLanes) base[k] = have[k];
                const uint32_t tail = max(end & ~15u, off ? 16u : 0u) / (uint32_t)sizeof(T);
                for (uint32_t k = tail + lane; k < end / sizeof(T); k += kLanes) base[k] = have[k];
            }
            __syncwarp();
        }
    }
}

// ------------------------------------------------------------------------------------------------
// dw[i, o] = sum_t x^[t, i] dy[t, o].  Both operands lie with the contraction index t along the rows, i.e. "MN-major": a
// TMA box of 64 columns x 64 tokens is 64 swizzled 128-byte rows, one per token.
// Two CTAs (two SMs) share an output tile of 256 x 256: each holds the operand columns of its 128 rows and of half of
// the tile's columns, so that a run of 64 tokens costs an SM 24 KB of copies for 512 cycles of the tensor core (one CTA with
// a 128 x 256 tile would need 40 KB, more than the L2 gives it).  Roles in each CTA:
//   warp 0      TMA producer, up to kStages runs ahead: 128 columns of q (8 KB), 128 columns of dy (two boxes, 16 KB)
//   warp 1      (first CTA only) MMA issuer: four tcgen05.mma.cta_group::2 (M 256, N 256, K 16) per run into one of two TMEM
//               accumulators
//   warps 2-5   epilogue: TMEM -> registers -> dw (or a partial sum), coalesced through a padded staging tile.  In
//               k_wgrad<false> eight warps (2-9), which keep the tile's sums in registers and add a finished accumulator to
//               them every kSegmentRuns runs: the tensor core drops low bits at each of its additions, so that its error grows
//               with their number (of the result's norm at 8192 tokens 2.8e-6 without, 2.0e-7 every 16 runs, 1.6e-7 every 12; half
//               as much again where a few tokens are much larger than the others; every 8: 1.2e-7, 2 to 7 % slower).  k_wgrad<true>
//               has no registers for that; where an item has more than kFusedRuns runs it adds a finished accumulator to what the
//               same threads wrote before (16384 tokens, 18944 x 256: error 7.0e-6 -> 4.5e-7 for 147 -> 161 us; 8192 tokens, 9728 x 512:
//               2.7e-6 -> 4.4e-7, 93 -> 100).  The code for it is an instantiation of its own: in the others' epilogue it cost 1 to 2 us
//   warps 6-21  q -> bf16 operand tile, two groups of eight warps on alternate runs: thread = (token, block of 32), the two
//               16-byte pieces of q become four of bf16.  The exponents come by plain loads, kAhead of a group's runs ahead.
// Every tile of a row of tiles converts the same operand again.  Beyond kFusedOut output columns the operand is therefore
// converted once, to bf16 in the workspace (three more bytes of memory traffic per value), and k_wgrad<false> takes both
// operands by TMA, without converter warps.  Measured, converted in the kernel / before it, us: 512 output columns 8192 x 1000 27.0 / 27.5,
// 8192 x 4096 57 / 60, 3000 x 512 24.8 / 24.0; 300 columns 32768 x 512 58 / 70; 256 columns 4096 x 4096 28 / 33, 16384 x 128 24.9 / 23.5; 640 columns
// 8192 x 4096 82 / 68, 2048 x 4096 30.7 / 24.9, 515 x 4096 18.7 / 15.7, 16 x 4096 14.5 / 12.6; 1111 columns 515 x 600 19.9 / 18.2; 4096 columns
// 3000 x 4096 125 / 92, 1024 x 4096 57.7 / 41.3, 128 x 4096 36.6 / 28.9.
// 8192 x 4096 x 4096 210 (in a loop that the power limit slows 255; a library bf16 product of operands already in bf16: 182): bound by the
// tensor core (pipe 74 % busy); on few tokens by the launch, the first copies and the epilogue: 40 x 128 x 128 10.4 us, 515 x 1000 x 1111 18.4, of which
// 5 for dy's odd rows.
// The kernel is launched in plain stream order and starts no successor early: chained by programmatic dependent launch, calls in a
// row hung, for a reason that is not known.  Every wait on a barrier is bounded, so it was not one of those; nor can a call's TMEM
// allocation have waited for the call ahead on the same SM, where the shared memory of two such CTAs has no room.
// Items are dealt out round-robin to the pairs: the whole tiles, as many as fill all pairs equally often, then the rest, each
// cut along the tokens into `splits` runs so that they too keep all pairs busy; k_wgrad_join adds those up in order.
// ------------------------------------------------------------------------------------------------
constexpr int kTM = 256, kTN = 256, kTK = 64;    // of a pair
constexpr int kRawBytes = kTK * 128, kABytes = kTK * 128 * 2, kBBytes = kTK * 128 * 2;
constexpr int kAhead = 4;
constexpr int kPitch = 33;
constexpr int kSegmentRuns = 12;
constexpr int kFusedRuns = 32;

template <bool kFused>
struct WgSmem {
    static constexpr int kStages = 5, kASlots = kFused ? 4 : kStages;
    static constexpr int kEpiWarps = kFused ? 4 : 8;
    alignas(1024) uint8_t raw[kFused ? kStages : 1][kFused ? kRawBytes : 1024];
    alignas(1024) uint8_t b[kStages][kBBytes];
    alignas(1024) uint8_t a[kASlots][kABytes];
    float out[kEpiWarps][32 * kPitch];
    alignas(8) uint64_t full[kStages];       // fused: this CTA's copies of a run have landed; else, first CTA: both CTAs' have
    uint64_t empty[kStages];                 // the run's MMAs have read both CTAs' operands
    uint64_t ready[kASlots];                 // fused, first CTA: both CTAs' operands of a run are there
    uint64_t acc_full[2];
    uint64_t acc_empty[2];                   // first CTA: both CTAs have read the accumulator
    uint32_t tmem_base;
    uint32_t failed;
};

struct WgArgs {
    const uint8_t* e;
    size_t e_ld;             // W / 32
    int T, D, N;
    int tiles_n, whole, rest, splits, kb_per_split;   // tiles: whole ones, then `rest` cut into `splits` runs; kb: 64 tokens
    float* dw;
    size_t ld;
    float* part;             // [splits][rest][kTM][kTN]
    int accumulate;
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
// One arrival on the same barrier of the cluster's first CTA.  What it announces -- operand tiles written and fenced for the
// async proxy, accumulators read and fenced by tcgen05.fence -- is ordered by those fences; a release at cluster scope would
// make the warp wait for the exponents that it has in flight (617 instead of 350 us when this form was chosen).
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

template <bool kFused>
constexpr int kWgThreads = kFused ? 704 : 320;

// tm_x: q, or the operand in bf16.  kLong (with kFused): items may have more than kFusedRuns runs.
template <bool kFused, bool kLong>
__global__ void __launch_bounds__(kWgThreads<kFused>, 1) k_wgrad(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_dy,
                                                                 const __grid_constant__ WgArgs a) {
    constexpr int kStages = WgSmem<kFused>::kStages, kASlots = WgSmem<kFused>::kASlots;
    extern __shared__ uint8_t smem_raw[];
    WgSmem<kFused>& s = *reinterpret_cast<WgSmem<kFused>*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int rank = (int)cluster_rank();
    const int pair = blockIdx.x / 2, pairs = gridDim.x / 2;
    const int items = a.whole + a.rest * a.splits;
    const int kb_total = (a.T + kTK - 1) / kTK;
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s.tmem_base)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&s.full[i], 1);
            mbar_init(&s.empty[i], 1);
        }
        for (int i = 0; i < kASlots; ++i) mbar_init(&s.ready[i], 16);    // eight warps of each CTA
        for (int i = 0; i < 2; ++i) {
            mbar_init(&s.acc_full[i], 1);
            mbar_init(&s.acc_empty[i], 2 * WgSmem<kFused>::kEpiWarps);   // the epilogue warps of each CTA
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
        int m0, n0, kb0, kb1;        // first row and column of the pair's tile, runs of 64 tokens
        int part;                    // index of the partial sum, -1: straight to dw
    };
    constexpr int kSegment = !kFused ? kSegmentRuns : kLong ? kFusedRuns : 1 << 30;    // runs that the tensor core adds up on its own
    auto item_of = [&](int it) {
        Item q;
        int tile = it;
        q.part = -1;
        q.kb0 = 0;
        q.kb1 = kb_total;
        if (it >= a.whole) {
            const int r = it - a.whole;
            tile = a.whole + r % a.rest;
            if (a.splits > 1) {
                q.part = r;
                q.kb0 = min(kb_total, r / a.rest * a.kb_per_split);
                q.kb1 = min(kb_total, q.kb0 + a.kb_per_split);
            }
        }
        q.m0 = tile / a.tiles_n * kTM;
        q.n0 = tile % a.tiles_n * kTN;
        return q;
    };

    if (warp == 0) {
        if (lane == 0) {                             // ---- TMA producer
            uint32_t st = 0, round = 0;
            for (int it = pair; it < items && !*failed; it += pairs) {
                const Item q = item_of(it);
                for (int kb = q.kb0; kb < q.kb1; ++kb) {
                    if (round > 0 && !mbar_wait(&s.empty[st], (round - 1) & 1)) { *failed = 1; break; }
                    const int m = q.m0 + rank * 128, n = q.n0 + rank * 128, t = kb * kTK;
                    if constexpr (kFused) {
                        mbar_expect_tx(&s.full[st], kRawBytes + kBBytes);
                        tma_load_2d(s.raw[st], &tm_x, m, t, &s.full[st]);
                        tma_load_2d(s.b[st], &tm_dy, n, t, &s.full[st]);
                        tma_load_2d(s.b[st] + 8192, &tm_dy, n + 64, t, &s.full[st]);
                    } else {
                        if (rank == 0) mbar_expect_tx(&s.full[st], 2 * (kABytes + kBBytes));
                        tma_load_2d_first(s.a[st], &tm_x, m, t, &s.full[st]);
                        tma_load_2d_first(s.a[st] + 8192, &tm_x, m + 64, t, &s.full[st]);
                        tma_load_2d_first(s.b[st], &tm_dy, n, t, &s.full[st]);
                        tma_load_2d_first(s.b[st] + 8192, &tm_dy, n + 64, t, &s.full[st]);
                    }
                    if (++st == kStages) { st = 0; ++round; }
                }
            }
            if (*failed && (kFused || rank == 0))    // copies in flight land before the CTAs' shared memory is released
                for (uint32_t i = 0; i < kStages; ++i) mbar_wait(&s.full[i], (round + (i < st ? 0u : 1u)) & 1u, 4096u);
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {                // ---- MMA issuer
            constexpr uint32_t idesc = umma_idesc_bf16(kTM, kTN) | (1u << 15) | (1u << 16);   // both operands MN-major
            uint32_t st = 0, sl = 0, sl_phase = 0;
            int i = 0;                               // segments so far: every other one in the same accumulator
            bool ok = true;
            for (int it = pair; it < items && ok; it += pairs) {
                const Item q = item_of(it);
                for (int kb0 = q.kb0; kb0 < q.kb1 && ok; kb0 += min(kSegment, q.kb1 - kb0), ++i) {
                    const int ab = i & 1, kb1 = min(q.kb1 - kb0, kSegment) + kb0;
                    if (i >= 2 && !mbar_wait(&s.acc_empty[ab], ((i / 2) - 1) & 1)) { ok = false; break; }
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    for (int kb = kb0; kb < kb1; ++kb) {
                        if (!mbar_wait(kFused ? &s.ready[sl] : &s.full[sl], sl_phase)) { ok = false; break; }
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint32_t a0 = smem_u32(s.a[sl]), b0 = smem_u32(s.b[st]);
#pragma unroll
                        for (int k = 0; k < kTK / 16; ++k)
                            umma2_bf16(tmem + ab * kTN, umma_desc_mn_sw128(a0 + k * 2048, 8192), umma_desc_mn_sw128(b0 + k * 2048, 8192), idesc,
                                       kb > kb0 || k > 0);
                        umma2_commit(&s.empty[st]);
                        if (++st == kStages) st = 0;
                        if (++sl == kASlots) { sl = 0; sl_phase ^= 1u; }
                    }
                    if (ok) umma2_commit(&s.acc_full[ab]);
                }
            }
            if (!ok) *failed = 1;
        }
        __syncwarp();
    } else if constexpr (!kFused) {                  // ---- epilogue: warps 2-5 the first 128 columns, 6-9 the others
        const int qd = warp % 4, half = (warp - 2) / 4;
        float* stage = s.out[warp - 2];
        const int row = rank * 128 + qd * 32;        // of the tile
        int i = 0;
        bool ok = true;
        for (int it = pair; it < items && ok; it += pairs) {
            const Item q = item_of(it);
            float2 sum[4][16];
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int j = 0; j < 16; ++j) sum[c][j] = both(0.f);
            for (int kb0 = q.kb0; kb0 < q.kb1; kb0 += kSegment, ++i) {
                const int ab = i & 1;
                ok = __all_sync(0xffffffffu, mbar_wait(&s.acc_full[ab], (i / 2) & 1) && !*failed);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                for (int c = 0; c < 8; ++c) {            // 16 columns: the sums and 32 loaded ones do not fit the registers
                    uint32_t v[16];
                    tmem_ld_16(tmem + ((uint32_t)(qd * 32) << 16) + (uint32_t)(ab * kTN + half * 128 + c * 16), v);
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        sum[c / 2][c % 2 * 8 + j] = add2(sum[c / 2][c % 2 * 8 + j], make_float2(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1])));
                }
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) arrive_first(&s.acc_empty[ab]);
            }
            if (!ok) {
                *failed = 1;
                break;
            }
            const bool part = q.part >= 0;
            float* base = part ? a.part + ((size_t)q.part * kTM + row) * kTN : a.dw + (size_t)(q.m0 + row) * a.ld + q.n0;
            const size_t ld = part ? (size_t)kTN : a.ld;
            const int rows = min(32, a.D - (q.m0 + row)), cols = a.N - q.n0 - half * 128;
            const bool add = a.accumulate && !part;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if (c * 32 >= cols) continue;
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    stage[lane * kPitch + 2 * j] = sum[c][j].x;
                    stage[lane * kPitch + 2 * j + 1] = sum[c][j].y;
                }
                __syncwarp();
                float* p = base + half * 128 + c * 32 + lane;
                if (c * 32 + lane < cols) {
                    if (add) {
#pragma unroll 8
                        for (int r = 0; r < rows; ++r) p[(size_t)r * ld] += stage[r * kPitch + lane];
                    } else {
#pragma unroll 8
                        for (int r = 0; r < rows; ++r) p[(size_t)r * ld] = stage[r * kPitch + lane];
                    }
                }
                __syncwarp();
            }
        }
    } else if (warp < 6) {                           // ---- epilogue
        const int qd = warp % 4;
        float* stage = s.out[warp - 2];
        int i = 0;
        for (int it = pair, done = 0; it < items; ++i) {     // done: runs of the item in the segments before
            const Item q = item_of(it);
            const int ab = i & 1;
            const bool ok = mbar_wait(&s.acc_full[ab], (i / 2) & 1) && !*failed;
            if (!__all_sync(0xffffffffu, ok)) {
                *failed = 1;
                break;
            }
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const int row = rank * 128 + qd * 32;    // of the tile
            const bool part = q.part >= 0;
            float* base = part ? a.part + ((size_t)q.part * kTM + row) * kTN : a.dw + (size_t)(q.m0 + row) * a.ld + q.n0;
            const size_t ld = part ? (size_t)kTN : a.ld;
            const int rows = min(32, a.D - (q.m0 + row)), cols = a.N - q.n0;
            const bool add = a.accumulate && !part, more = kLong && done > 0;
            for (int c = 0; c < kTN / 32; ++c) {
                uint32_t v[32];
                tmem_ld_32(tmem + ((uint32_t)(qd * 32) << 16) + (uint32_t)(ab * kTN + c * 32), v);
                if (c == kTN / 32 - 1) {
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) arrive_first(&s.acc_empty[ab]);
                }
                if (c * 32 >= cols) continue;
#pragma unroll
                for (int j = 0; j < 32; ++j) stage[lane * kPitch + j] = __uint_as_float(v[j]);
                __syncwarp();
                float* p = base + c * 32 + lane;
                if (c * 32 + lane < cols) {
                    if (more) {                      // to this thread's own sums of the segments before, in order and with no load to wait for
#pragma unroll 8
                        for (int r = 0; r < rows; ++r)
                            asm volatile("red.global.add.f32 [%0], %1;" ::"l"(p + (size_t)r * ld), "f"(stage[r * kPitch + lane]) : "memory");
                    } else if (add) {
#pragma unroll 8
                        for (int r = 0; r < rows; ++r) p[(size_t)r * ld] += stage[r * kPitch + lane];
                    } else {
#pragma unroll 8
                        for (int r = 0; r < rows; ++r) p[(size_t)r * ld] = stage[r * kPitch + lane];
                    }
                }
                __syncwarp();
            }
            done += kSegment;
            if (!kLong || done >= q.kb1 - q.kb0) {
                done = 0;
                it += pairs;
            }
        }
    } else {                                         // ---- q -> bf16 operand tile
        const int tid = (threadIdx.x - 192) % 256, group = (threadIdx.x - 192) / 256;
        const int r = tid % kTK, blk = tid / kTK;    // token of the run, block of 32 columns
        const uint32_t sw = (uint32_t)(r & 7);
        int n = 0;                                   // runs so far, of both groups
        bool ok = true;
        for (int it = pair; it < items && ok; it += pairs) {
            const Item q = item_of(it);
            const size_t ecol = (size_t)((q.m0 + rank * 128) / 32 + blk);
            const uint8_t* ep = a.e + (size_t)r * a.e_ld + ecol;
            const bool have = ecol < a.e_ld;
            auto exponent = [&](int kb) -> uint32_t {   // of this thread's block; beyond the matrix q is filled with zeros
                return have && kb < q.kb1 && kb * kTK + r < a.T ? ep[(size_t)kb * kTK * a.e_ld] : 0u;
            };
            const int first = q.kb0 + ((group - n) & 1);     // this group's runs: every other one
            uint32_t e[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) e[u] = exponent(first + 2 * u);
            for (int kb0 = first; kb0 < q.kb1 && ok; kb0 += 2 * kAhead) {
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const int kb = kb0 + 2 * u;
                    if (kb >= q.kb1 || !ok) continue;
                    const int run = n + (kb - q.kb0);
                    const int st = run % kStages, sl = run % kASlots;
                    const float scale = pow2_of(e[u]);
                    e[u] = exponent(kb + 2 * kAhead);
                    // the MMAs of the run kASlots back have read this slot of the operand tile
                    if (run >= kASlots && !mbar_wait(&s.empty[(run - kASlots) % kStages], ((run - kASlots) / kStages) & 1)) { ok = false; continue; }
                    if (!mbar_wait(&s.full[st], (run / kStages) & 1)) { ok = false; continue; }
                    const uint8_t* src = s.raw[st] + r * 128;
                    uint8_t* dst = s.a[sl] + (blk / 2) * 8192 + r * 128;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint4 v = *reinterpret_cast<const uint4*>(src + ((uint32_t)(blk * 2 + h) ^ sw) * 16);
                        const uint32_t w[4] = {v.x ^ 0x80808080u, v.y ^ 0x80808080u, v.z ^ 0x80808080u, v.w ^ 0x80808080u};
#pragma unroll
                        for (int p = 0; p < 2; ++p) {
                            uint32_t o[4];
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const uint32_t word = w[2 * p + j / 2];
                                // the byte q + 128 as the low mantissa byte of 2^23: subtracting 2^23 + 128 leaves q exactly
                                float2 f = make_float2(__uint_as_float(__byte_perm(word, 0x4B000000u, 0x7540 + 2 * (j % 2))),
                                                       __uint_as_float(__byte_perm(word, 0x4B000000u, 0x7541 + 2 * (j % 2))));
                                f = mul2(add2(f, both(-8388736.f)), both(scale));
                                const __nv_bfloat162 b2 = __float22bfloat162_rn(f);
                                o[j] = *reinterpret_cast<const uint32_t*>(&b2);
                            }
                            const uint32_t chunk = (uint32_t)((blk % 2) * 4 + h * 2 + p);
                            *reinterpret_cast<uint4*>(dst + (chunk ^ sw) * 16) = make_uint4(o[0], o[1], o[2], o[3]);
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) arrive_first(&s.ready[sl]);
                }
            }
            n += q.kb1 - q.kb0;
        }
        if (!ok) *failed = 1;
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    cluster_sync();                                  // no CTA leaves while the other's arrivals or MMAs may still reach it
    if (threadIdx.x == 0 && *failed) report_timeout();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

// dw (+)= the partial sums of the tiles that were cut, in order.
__global__ void __launch_bounds__(256) k_wgrad_join(const __grid_constant__ WgArgs a) {
    pdl_wait();
    pdl_trigger();
    const size_t step = (size_t)a.rest * kTM * kTN;
    constexpr int kRows = 4;                         // rows of tiles at a time
    for (int i0 = blockIdx.x * kRows; i0 < a.rest * kTM; i0 += gridDim.x * kRows) {
        float s[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) s[r] = 0.f;
        const float* p = a.part + (size_t)i0 * kTN + threadIdx.x;    // kTM is a multiple of kRows
#pragma unroll 2
        for (int k = 0; k < a.splits; ++k)
#pragma unroll
            for (int r = 0; r < kRows; ++r) s[r] += p[k * step + (size_t)r * kTN];
        const int tile = a.whole + i0 / kTM, m = tile / a.tiles_n * kTM + i0 % kTM, n = tile % a.tiles_n * kTN + threadIdx.x;
        if (n >= a.N) continue;
        float* o = a.dw + (size_t)m * a.ld + n;
#pragma unroll
        for (int r = 0; r < kRows; ++r)
            if (m + r < a.D) o[(size_t)r * a.ld] = a.accumulate ? o[(size_t)r * a.ld] + s[r] : s[r];
    }
}

// dy with rows that TMA cannot start at, copied to rows of `ld8` elements (16-byte aligned).
__global__ void __launch_bounds__(256) k_pack_rows(const bf16* x, size_t ld, int N, int ld8, size_t n, bf16* out) {
    pdl_wait();
    pdl_trigger();
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) {
        const size_t t = i / ld8;
        const int c = (int)(i - t * ld8);
        out[i] = c < N ? x[t * ld + c] : __float2bfloat16_rn(0.f);
    }
}

bool misaligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

int grid_for(size_t n, int per_cta) {
    const size_t want = (n + per_cta - 1) / per_cta;
    return (int)std::min<size_t>(want, 148 * 16);
}

constexpr int kSms = 148;
constexpr uint64_t kSizeMax = 0x7fffffc0ull;     // tokens, width, out: what is rounded up to a tile stays an int
constexpr int kFusedOut = 512;   // output columns up to which the operand is converted in the kernel
constexpr int kMinRuns = 12;     // runs of 64 tokens that a part of a cut tile has at least: shorter ones do not pay for the join

// How the work is cut: whole output tiles for all pairs of SMs equally often, the rest in runs of tokens.
struct WgPlan {
    int tiles_m, tiles_n, whole, rest, splits, kb_per_split;
    bool repack, fused;
    size_t ld8, part_bytes, pack_bytes, x_bytes;
    size_t bytes() const { return part_bytes + pack_bytes + x_bytes; }
};
bool plan_of(uint64_t T, uint64_t D, uint64_t N, const void* dy, uint64_t ld_dy, WgPlan* out) {
    WgPlan p{};
    p.tiles_m = (int)((D + kTM - 1) / kTM);
    p.tiles_n = (int)((N + kTN - 1) / kTN);
    const int kb = (int)((T + kTK - 1) / kTK), pairs = kSms / 2;
    const int64_t tiles = (int64_t)p.tiles_m * p.tiles_n;
    if (tiles > 0x3fffffff) return false;
    p.whole = (int)(tiles / pairs * pairs);
    p.rest = (int)(tiles - p.whole);
    p.fused = N <= (uint64_t)kFusedOut;
    int splits = p.rest ? std::min(pairs / p.rest, kb / kMinRuns) : 1;
    if (splits < 1) splits = 1;
    p.kb_per_split = std::max(1, (kb + splits - 1) / splits);
    p.splits = std::max(1, (kb + p.kb_per_split - 1) / p.kb_per_split);
    p.repack = misaligned(dy, 16) || ld_dy % 8 != 0;
    p.ld8 = (N + 7) / 8 * 8;
    p.part_bytes = p.splits > 1 ? (size_t)p.splits * p.rest * kTM * kTN * 4 : 0;
    p.pack_bytes = p.repack ? up256((size_t)T * p.ld8 * 2) : 0;
    p.x_bytes = p.fused ? 0 : up256((size_t)T * ((D + 31) / 32 * 32) * 2);
    *out = p;
    return true;
}

}  // namespace
}  // namespace abs_sgd

using namespace abs_sgd;

namespace abs_sgd {
namespace {
// The arguments for rows of `per_row` units.
PackArgs pack_args(uint64_t tokens, uint64_t width, uint64_t ld, uint32_t per_row) {
    PackArgs a{};
    a.ld = (size_t)ld;
    a.T = (size_t)tokens;
    a.D = (int)width;
    a.pieces = (int)((width + 31) / 32 * 4);
    a.units = a.T * per_row;
    Divide& v = a.per_row;
    v.d = per_row;
    v.small = a.units < 0x7fffffffull;
    uint32_t log = 0;
    while ((1ull << log) < per_row) ++log;
    if (log) {               // mul = ceil(2^(31 + log) / d) < 2^32; exact for n < 2^31
        v.mul = (uint32_t)(((1ull << (31 + log)) + per_row - 1) / per_row);
        v.shift = log - 1;
    }
    return a;
}
int pack_grid(size_t units, int per_cta) {
    const size_t want = (units + (size_t)per_cta * kUnroll - 1) / ((size_t)per_cta * kUnroll);
    return (int)std::min<size_t>(want, kSms * 8);
}
const char* check_ckpt(const void* x, uint64_t ld, uint32_t dtype, uint64_t tokens, uint64_t width, const void* q, const void* e, int* code) {
    *code = ABS_EINVAL;
    if (dtype != ABS_F32 && dtype != ABS_BF16) return "dtype must be ABS_F32 or ABS_BF16";
    if (width == 0 || ld < width) return "width must be at least 1 and ld_x at least width";
    if (width > 0x7fffff00ull) {
        *code = ABS_ELIMIT;
        return "width exceeds 2^31 - 256";
    }
    if (tokens && (!x || !q || !e)) return "x, q and e must not be NULL";
    if (misaligned(x, dtype == ABS_F32 ? 4 : 2) || misaligned(q, 16)) return "x must be aligned to its elements, q to 16 bytes";
    return nullptr;
}
template <typename T>
cudaError_t quantize(const void* x, uint64_t ld, uint64_t tokens, uint64_t width, int8_t* q, uint8_t* e, cudaStream_t s) {
    const bool wide = !misaligned(x, 16) && ld * sizeof(T) % 16 == 0;
    const PackArgs a = pack_args(tokens, width, ld, (uint32_t)((width + 31) / 32 * 4));
    return launch_kernel(wide ? k_ckpt8_quantize<T, true> : k_ckpt8_quantize<T, false>, pack_grid(a.units, 256), 256, 0, s, true, static_cast<const T*>(x), a,
                         reinterpret_cast<uint2*>(q), e);
}
template <typename T, int kLanes>
cudaError_t dequantize_any(const int8_t* q, const uint8_t* e, void* x, uint64_t ld, uint64_t tokens, uint64_t width, uint32_t pieces, cudaStream_t s) {
    const PackArgs a = pack_args(tokens, width, ld, (pieces + kLanes - 1) / kLanes);
    return launch_kernel(k_ckpt8_dequantize_any<T, kLanes>, pack_grid(a.units, 256 / kLanes), 256, 0, s, true, reinterpret_cast<const uint8_t*>(q), e,
                         static_cast<T*>(x), a);
}
template <typename T>
cudaError_t dequantize(const int8_t* q, const uint8_t* e, void* x, uint64_t ld, uint64_t tokens, uint64_t width, cudaStream_t s) {
    const uint32_t pieces = (uint32_t)((width + kVec<T> - 1) / kVec<T>);
    if (!misaligned(x, 16) && ld * sizeof(T) % 16 == 0) {
        const PackArgs a = pack_args(tokens, width, ld, pieces);
        return launch_kernel(k_ckpt8_dequantize<T>, pack_grid(a.units, 256), 256, 0, s, true, reinterpret_cast<const uint8_t*>(q), e, static_cast<T*>(x), a);
    }
    // lanes of a row's part: as many as the row has pieces, within a warp
    return pieces <= 4 ? dequantize_any<T, 4>(q, e, x, ld, tokens, width, pieces, s) : pieces <= 8 ? dequantize_any<T, 8>(q, e, x, ld, tokens, width, pieces, s)
         : pieces <= 16 ? dequantize_any<T, 16>(q, e, x, ld, tokens, width, pieces, s) : dequantize_any<T, 32>(q, e, x, ld, tokens, width, pieces, s);
}
template <bool kFused, bool kLong>
cudaError_t launch_wgrad(const CUtensorMap& tx, const CUtensorMap& td, const WgArgs& a, int grid, cudaStream_t s) {
    const cudaError_t e = allow_smem<k_wgrad<kFused, kLong>>();
    return e != cudaSuccess ? e : launch_cluster(k_wgrad<kFused, kLong>, grid, 2, kWgThreads<kFused>, sizeof(WgSmem<kFused>) + 1024, s, tx, td, a);
}
}  // namespace
}  // namespace abs_sgd

extern "C" int abs_ckpt8_quantize(const void* x, uint64_t ld_x, uint32_t dtype, uint64_t tokens, uint64_t width, int8_t* q, uint8_t* e,
                                  void* stream) {
    int code = 0;
    if (const char* why = check_ckpt(x, ld_x, dtype, tokens, width, q, e, &code)) return thread_error(code, why);
    if (tokens == 0) return ABS_OK;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t r = dtype == ABS_F32 ? quantize<float>(x, ld_x, tokens, width, q, e, s) : quantize<bf16>(x, ld_x, tokens, width, q, e, s);
    return r == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(r));
}

extern "C" int abs_ckpt8_dequantize(const int8_t* q, const uint8_t* e, uint64_t tokens, uint64_t width, void* x, uint64_t ld_x, uint32_t dtype,
                                    void* stream) {
    int code = 0;
    if (const char* why = check_ckpt(x, ld_x, dtype, tokens, width, q, e, &code)) return thread_error(code, why);
    if (tokens == 0) return ABS_OK;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const cudaError_t r = dtype == ABS_F32 ? dequantize<float>(q, e, x, ld_x, tokens, width, s) : dequantize<bf16>(q, e, x, ld_x, tokens, width, s);
    return r == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(r));
}

extern "C" size_t abs_ckpt8_wgrad_workspace(uint64_t tokens, uint64_t width, uint64_t out, const void* dy, uint64_t ld_dy) {
    if (tokens > kSizeMax || width > kSizeMax || out > kSizeMax) return 0;
    WgPlan p;
    return plan_of(tokens, width, out, dy, ld_dy, &p) ? p.bytes() : 0;
}

extern "C" int abs_ckpt8_wgrad(const int8_t* q, const uint8_t* e, const void* dy, uint64_t ld_dy, uint64_t tokens, uint64_t width,
                               uint64_t out, float* dw, uint64_t ld_dw, int accumulate, void* workspace, size_t workspace_bytes, void* stream) {
    if (width == 0 || out == 0 || ld_dy < out || ld_dw < out) return thread_error(ABS_EINVAL, "width and out must be at least 1, ld_dy and ld_dw at least out");
    if (tokens > kSizeMax || width > kSizeMax || out > kSizeMax) return thread_error(ABS_ELIMIT, "a size exceeds 2^31 - 64");
    if (!dw || misaligned(dw, 4)) return thread_error(ABS_EINVAL, "dw must be non-NULL and 4-byte aligned");
    if (tokens && (!q || !e || !dy)) return thread_error(ABS_EINVAL, "q, e and dy must not be NULL");
    if (misaligned(q, 16) || misaligned(dy, 2)) return thread_error(ABS_EINVAL, "q must be aligned to 16 bytes, dy to its elements");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t r = cudaSuccess;
    if (tokens == 0) {
        if (!accumulate) r = cudaMemset2DAsync(dw, ld_dw * 4, 0, out * 4, width, s);
        return r == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(r));
    }
    WgPlan p;
    if (!plan_of(tokens, width, out, dy, ld_dy, &p)) return thread_error(ABS_ELIMIT, "too many output tiles");
    if (p.bytes()) {
        if (!workspace || misaligned(workspace, 256)) return thread_error(ABS_EINVAL, "workspace must be non-NULL and 256-byte aligned");
        if (workspace_bytes < p.bytes()) return thread_error(ABS_ENOMEM, "workspace too small");
    }
    float* part = static_cast<float*>(workspace);
    if (p.repack) {
        bf16* packed = reinterpret_cast<bf16*>(static_cast<char*>(workspace) + p.part_bytes);
        const size_t n = (size_t)tokens * p.ld8;
        r = launch_kernel(k_pack_rows, grid_for(n, 1024), 256, 0, s, true, static_cast<const bf16*>(dy), (size_t)ld_dy, (int)out, (int)p.ld8, n, packed);
        if (r != cudaSuccess) return thread_error(ABS_ECUDA, cudaGetErrorString(r));
        dy = packed;
        ld_dy = p.ld8;
    }
    const uint64_t W = (width + 31) / 32 * 32;
    CUtensorMap tx, td;
    bf16* x = reinterpret_cast<bf16*>(static_cast<char*>(workspace) + p.part_bytes + p.pack_bytes);
    if (!p.fused) {
        r = dequantize<bf16>(q, e, x, W, tokens, W, s);
        if (r != cudaSuccess) return thread_error(ABS_ECUDA, cudaGetErrorString(r));
    }
    if (!(p.fused ? encode_2d(&tx, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, const_cast<int8_t*>(q), tokens, W, kTK, 128)
                  : encode_2d(&tx, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, x, tokens, W, kTK, 64)) ||
        !encode_2d(&td, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(dy), tokens, out, kTK, 64, ld_dy))
        return thread_error(ABS_ECUDA, "cuTensorMapEncodeTiled failed");
    WgArgs a{};
    a.e = e; a.e_ld = W / 32; a.T = (int)tokens; a.D = (int)width; a.N = (int)out;
    a.tiles_n = p.tiles_n; a.whole = p.whole; a.rest = p.rest; a.splits = p.splits; a.kb_per_split = p.kb_per_split;
    a.dw = dw; a.ld = ld_dw; a.part = part; a.accumulate = accumulate != 0;
    const int grid = 2 * std::min(p.whole + p.rest * p.splits, kSms / 2);
    const int most = p.whole > 0 || p.splits == 1 ? (a.T + kTK - 1) / kTK : a.kb_per_split;      // runs of the longest item
    r = !p.fused          ? launch_wgrad<false, false>(tx, td, a, grid, s)
        : most > kFusedRuns ? launch_wgrad<true, true>(tx, td, a, grid, s)
                            : launch_wgrad<true, false>(tx, td, a, grid, s);
    if (r == cudaSuccess && p.splits > 1) r = launch_kernel(k_wgrad_join, std::min(p.rest * kTM / 4, kSms * 8), 256, 0, s, false, a);
    return r == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(r));
}

extern "C" int abs_llm_check(void* stream) {
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    int any = 0;
    for (const auto take : {&take_status, &take_status_norm, &take_status_loss, &take_status_layer_norm, &take_status_linear, &take_status_recurrence}) {
        int st = 0;
        const cudaError_t r = take(&st, s);
        if (r != cudaSuccess) return thread_error(ABS_ECUDA, cudaGetErrorString(r));
        any |= st;
    }
    return any == 0 ? ABS_OK : thread_error(ABS_ETIMEOUT, "a bounded wait inside a kernel ran out");
}
