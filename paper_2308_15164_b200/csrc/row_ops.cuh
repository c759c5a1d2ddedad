// Device-side helpers of the kernels that work on rows of activations or logits: element types, 16-byte pieces,
// reductions over a group of threads.
#pragma once

#include <cuda_bf16.h>
#include <stddef.h>
#include <stdint.h>

namespace abs_sgd {

using bf16 = __nv_bfloat16;

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(bf16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_f(float v);
template <>
__device__ __forceinline__ float from_f<float>(float v) { return v; }
template <>
__device__ __forceinline__ bf16 from_f<bf16>(float v) { return __float2bfloat16_rn(v); }

// N consecutive elements as floats; the address is a multiple of N elements' bytes (N = 1: of one element's).
template <typename T, int N>
struct Pack;
template <typename T>
struct Pack<T, 1> {
    static __device__ __forceinline__ void load(const T* p, float (&v)[1]) { v[0] = to_f(*p); }
    static __device__ __forceinline__ void store(T* p, const float (&v)[1]) { *p = from_f<T>(v[0]); }
};
template <>
struct Pack<float, 4> {
    static __device__ __forceinline__ void load(const float* p, float (&v)[4]) {
        const float4 a = *reinterpret_cast<const float4*>(p);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    }
    static __device__ __forceinline__ void store(float* p, const float (&v)[4]) {
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    }
};
template <>
struct Pack<bf16, 8> {
    static __device__ __forceinline__ void load(const bf16* p, float (&v)[8]) {
        const uint4 a = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ void store(bf16* p, const float (&v)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&b);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);   // elements of a 16-byte piece

// Pairs of fp32 in one 64-bit register (fma.rn.f32x2 and its kin round like the scalar instructions).
__device__ __forceinline__ uint64_t as_u64(float2 v) { return *reinterpret_cast<uint64_t*>(&v); }
__device__ __forceinline__ float2 as_f2(uint64_t v) { return *reinterpret_cast<float2*>(&v); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(as_u64(a)), "l"(as_u64(b)), "l"(as_u64(c)));
    return as_f2(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(as_u64(a)), "l"(as_u64(b)));
    return as_f2(r);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(as_u64(a)), "l"(as_u64(b)));
    return as_f2(r);
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
__device__ __forceinline__ float sum2(float2 v) { return v.x + v.y; }

// A 16-byte piece as kVec / 2 pairs.
template <typename T>
constexpr int kPairs = kVec<T> / 2;
__device__ __forceinline__ void unpack(uint4 a, float2 (&v)[2], float) {
    v[0] = make_float2(__uint_as_float(a.x), __uint_as_float(a.y));
    v[1] = make_float2(__uint_as_float(a.z), __uint_as_float(a.w));
}
__device__ __forceinline__ void unpack(uint4 a, float2 (&v)[4], bf16) {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
}
__device__ __forceinline__ uint4 pack(const float2 (&v)[2], float) {
    return make_uint4(__float_as_uint(v[0].x), __float_as_uint(v[0].y), __float_as_uint(v[1].x), __float_as_uint(v[1].y));
}
__device__ __forceinline__ uint4 pack(const float2 (&v)[4], bf16) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __float22bfloat162_rn(v[i]);
        w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// 2^v by the approximate unit (relative error 2^-22; results below the normal range become 0).
__device__ __forceinline__ float exp2_of(float v) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float2 exp2_of(float2 v) { return make_float2(exp2_of(v.x), exp2_of(v.y)); }

// A row cut into single elements up to the first 16-byte boundary, 16-byte pieces, and single elements behind the last.
struct RowCut {
    int head, pieces, tail;
};
template <typename T>
__device__ __forceinline__ RowCut cut_row(const T* p, int n) {
    RowCut c;
    c.head = min(n, (int)(((16u - ((uint32_t)reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) / (uint32_t)sizeof(T)));
    c.pieces = (n - c.head) / kVec<T>;
    c.tail = n - c.head - c.pieces * kVec<T>;
    return c;
}

// Sum over a group of kThreads consecutive threads (32: a warp; more: the whole CTA of kThreads threads, `sh` holds
// kN * kThreads / 32 floats).  Every thread gets the sums; the order is fixed.
template <int kThreads, int kN>
__device__ __forceinline__ void group_sum(float (&v)[kN], float* sh) {
#pragma unroll
    for (int k = 0; k < kN; ++k)
#pragma unroll
        for (int o = 16; o; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
    if (kThreads == 32) return;
    constexpr int kWarps = kThreads / 32;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    __syncthreads();                       // `sh` may still be read from the previous call
    if (lane == 0)
#pragma unroll
        for (int k = 0; k < kN; ++k) sh[k * kWarps + warp] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kN; ++k) {
        float a = lane < kWarps ? sh[k * kWarps + lane] : 0.f;
#pragma unroll
        for (int o = 16; o; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
        v[k] = a;
    }
}

}  // namespace abs_sgd
