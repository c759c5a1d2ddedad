// Rows of activations through a ring of row images in shared memory: the copies of the next rows are in flight while a CTA, or a
// warp of it, works on the current one.  Used by the norms' kernels.
#pragma once

#include <cuda_runtime.h>

#include "bulk_copy.cuh"
#include "llm_host.h"
#include "llm_status.cuh"
#include "row_ops.cuh"

namespace abs_sgd {

constexpr int kRingMax = 8;
constexpr int kRingSmem = 216 * 1024;   // shared memory of an SM that the ring kernels' CTAs share (1 KB per CTA is the system's)
constexpr int kRowWarps = 8;            // warps of a CTA where each has rows of its own

// Columns of a row of partial sums: 16-byte pieces.
constexpr __host__ __device__ size_t part_width(size_t D) { return (D + 3) / 4 * 4; }

struct RingCtl {
    alignas(16) float red[3][6][16]; // [reduction][number][warp]
    alignas(8) uint64_t full[kRingMax];
    unsigned done;                   // warps that have read the current row
    unsigned gave_up;                // a wait for a row's image has run out
};
constexpr size_t kRingCtl = (sizeof(RingCtl) + 15) / 16 * 16;

// Sums over a row's threads: the warp (kWarp), or the CTA with one synchronisation, where `sh` (zero beyond the CTA's warps) must
// not be the buffer of the reduction just before.
template <bool kWarp, int kN>
__device__ __forceinline__ void row_sum(float (&v)[kN], float (*sh)[16], int warps) {
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    if (kN <= 2) {
#pragma unroll
        for (int k = 0; k < kN; ++k) {
#pragma unroll
            for (int o = 16; o; o >>= 1) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
            if (!kWarp && lane == 0) sh[k][warp] = v[k];
        }
        if (kWarp) return;
    } else {                         // up to eight: a step halves the numbers of a lane, number k ends in lanes 16 k0 + 8 k1 + 4 k2
        float w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = k < kN ? v[k < kN ? k : 0] : 0.f;
#pragma unroll
        for (int o = 16, n = 4; n; o >>= 1, n >>= 1)
#pragma unroll
            for (int k = 0; k < n; ++k) {
                const bool up = lane & o;
                const float give = up ? w[2 * k] : w[2 * k + 1], keep = up ? w[2 * k + 1] : w[2 * k];
                w[k] = keep + __shfl_xor_sync(0xffffffffu, give, o);
            }
        w[0] += __shfl_xor_sync(0xffffffffu, w[0], 2);
        w[0] += __shfl_xor_sync(0xffffffffu, w[0], 1);
        if (kWarp) {
#pragma unroll
            for (int k = 0; k < kN; ++k) v[k] = __shfl_sync(0xffffffffu, w[0], (k & 1) << 4 | (k & 2) << 2 | (k & 4));
            return;
        }
        const int k = (lane >> 4 & 1) | (lane >> 2 & 2) | (lane & 4);
        if (k < kN && (lane & 3) == 0) sh[k][warp] = w[0];
    }
    __syncthreads();
    if (warps == 1 && kN <= 2) return;
#pragma unroll
    for (int k = 0; k < kN; ++k) v[k] = 0.f;
    for (int w = 0; w < warps; w += 4)
#pragma unroll
        for (int k = 0; k < kN; ++k) {
            const float4 f = *reinterpret_cast<const float4*>(&sh[k][w]);
            v[k] += (f.x + f.y) + (f.z + f.w);
        }
}

__device__ __forceinline__ void copy_piece(void* to, const void* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}

// A CTA's rows (kWarp: a warp's): how they are cut, which of them are in flight, which is the current one.
template <typename T, int kIn, int kP, bool kWarp>
struct Ring {
    using Element = T;
    static constexpr int kInputs = kIn;
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

    static __device__ __forceinline__ int tid() { return kWarp ? threadIdx.x % 32 : threadIdx.x; }
    static __device__ __forceinline__ int step() { return kWarp ? 32 : blockDim.x; }
    // Rows of n elements, the first of this CTA (warp) at row0; room_bytes: a multiple of 16 that holds a row.
    __device__ __forceinline__ void begin(uint8_t* smem, size_t all_rows, int n, int ring_stages, uint32_t room_bytes, const T* row0) {
        ctl = reinterpret_cast<RingCtl*>(smem);
        row_bytes = room_bytes;
        stages = ring_stages;
        base = smem + kRingCtl + (kWarp ? (size_t)(threadIdx.x / 32) * stages * kIn * row_bytes : 0);
        rows = all_rows;
        cut = cut_row(row0, n);
        bytes = (uint32_t)cut.pieces * 16u;
        const int tid = Ring::tid();
        extra = tid < cut.head ? tid : tid < cut.head + cut.tail ? n - cut.tail + tid - cut.head : -1;
        if (!kWarp) {
            for (int i = tid; i < 18 * 16; i += blockDim.x) (&ctl->red[0][0][0])[i] = 0.f;
            if (tid == 0) {
                ctl->done = ctl->gave_up = 0;
                for (int i = 0; i < stages; ++i) mbar_init(&ctl->full[i], 1);
                asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            }
            __syncthreads();
        }
    }
    // One thread; kWarp: every lane its own pieces, one group of copies for each row.
    __device__ __forceinline__ void load(int stage, size_t t) {
        if (kWarp) {
            if (t < rows)
#pragma unroll
                for (int i = 0; i < kIn; ++i)
                    if (in[i])
#pragma unroll
                        for (int j = 0; j < kP; ++j)
                            if (has(j)) copy_piece(base + (size_t)(stage * kIn + i) * row_bytes + (tid() + j * 32) * 16, in[i] + t * ld[i] + column(j));
            asm volatile("cp.async.commit_group;" ::: "memory");
            return;
        }
        if (t >= rows || bytes == 0) return;
        uint32_t total = 0;
#pragma unroll
        for (int i = 0; i < kIn; ++i) total += in[i] ? bytes : 0;
        mbar_expect_tx(&ctl->full[stage], total);
#pragma unroll
        for (int i = 0; i < kIn; ++i)
            if (in[i]) bulk_load(base + (size_t)(stage * kIn + i) * row_bytes, in[i] + t * ld[i] + cut.head, bytes, &ctl->full[stage]);
    }
    // Everybody has passed the first synchronisation of the current row, t, the k-th: the image of the row before it is free.
    __device__ __forceinline__ void refill(size_t t, size_t G, int k) {
        if (threadIdx.x == 0 && k > 0) load((st == 0 ? stages : st) - 1, t + (size_t)(stages - 1) * G);
    }
    // This warp has read the image of the current row, t, for the last time; the last of the CTA's warps fills it again.  (No warp
    // is a row ahead: there is a synchronisation of the CTA in every row.)
    __device__ __forceinline__ void release(size_t t, size_t G, int warps) {
        if (kWarp) return load(st, t + (size_t)stages * G);          // a lane reads its own copies only
        __syncwarp();
        if (threadIdx.x % 32 != 0) return;
        __threadfence_block();
        if (atomicInc(&ctl->done, (unsigned)warps - 1) != (unsigned)warps - 1) return;
        __threadfence_block();
        load(st, t + (size_t)stages * G);
    }
    __device__ __forceinline__ void load_extra(size_t t, float (&v)[kIn]) const {
        if (extra < 0 || t >= rows) return;
#pragma unroll
        for (int i = 0; i < kIn; ++i) v[i] = in[i] ? to_f(in[i][t * ld[i] + extra]) : 0.f;
    }
    __device__ __forceinline__ void wait() {
        if (kWarp) {                 // a group per row: all but the last stages - 1 have arrived
            if (stages == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
            else if (stages == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
            else asm volatile("cp.async.wait_group 3;" ::: "memory");
            return;
        }
        if (bytes != 0 && !mbar_wait(&ctl->full[st], phase, ok ? kSpinLimit : 1u)) {
            ok = false;
            ctl->gave_up = 1;
        }
    }
    // Behind the last row: the CTA's sums over its rows cannot be formed (the rows' own synchronisations have made it known).  Marks them so.
    __device__ __forceinline__ bool without(float* sums, int n) const {
        if constexpr (!kWarp) {
            if (*(volatile unsigned*)&ctl->gave_up) {
                for (int i = threadIdx.x; i < n; i += blockDim.x) sums[i] = __uint_as_float(kUnformed);
                if (threadIdx.x == 0) report_timeout();
                return true;
            }
        }
        return false;
    }
    __device__ __forceinline__ void next() {
        if (++st == stages) { st = 0; phase ^= 1u; }
    }
    // Piece j of this thread of input i, in the current row's image.
    __device__ __forceinline__ void piece(int i, int j, float2 (&v)[kPairs<T>]) const {
        unpack(*reinterpret_cast<const uint4*>(base + (size_t)(st * kIn + i) * row_bytes + (tid() + j * step()) * 16), v, T());
    }
    __device__ __forceinline__ bool has(int j) const { return tid() + j * step() < cut.pieces; }
    __device__ __forceinline__ int column(int j) const { return cut.head + (tid() + j * step()) * kVec<T>; }
    __device__ __forceinline__ void store(T* row, int j, const float2 (&v)[kPairs<T>]) const {
        if (ok) *reinterpret_cast<uint4*>(row + column(j)) = pack(v, T());
    }
    // This thread's columns of a weight vector, times those of a second one if there is one; its single element is returned.
    __device__ __forceinline__ float weights(const float* p, const float* q, float2 (&w)[kP][kPairs<T>]) const {
        auto at = [&](int c) { return q ? p[c] * q[c] : p[c]; };
#pragma unroll
        for (int j = 0; j < kP; ++j)
#pragma unroll
            for (int i = 0; i < kPairs<T>; ++i) w[j][i] = has(j) ? make_float2(at(column(j) + 2 * i), at(column(j) + 2 * i + 1)) : both(0.f);
        return extra >= 0 ? at(extra) : 0.f;
    }
};

// ---- host side: how the matrices of a call lie
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

// first[c] (+)= the sum over i < n of part[i][0][c], second (may be NULL) of part[i][1][c]; rows of part_width(D).  llm_norm.cu
cudaError_t launch_column_sums(const float* part, int n, int D, float* first, float* second, int accumulate, cudaStream_t s);

}  // namespace abs_sgd
