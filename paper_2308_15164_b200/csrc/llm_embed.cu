// Scaled embedding lookup and its gradient (abs_embed*).
//
// Forward: a gather of rows, bound by memory.  Backward: the tokens are sorted by id (a stable radix sort, so that a row's tokens
// stay in their order), the sorted list is cut into chunks of equal length, each summed row by row; a row whose tokens pass a
// chunk's border leaves partial sums that a last kernel adds up in order.  No atomics: equal inputs give equal bits, and a token
// that fills half the micro-batch costs no more than the others.
#include <math.h>

#include <algorithm>

#include "abs_internal.h"
#include "abs_llm.h"
#include "llm_host.h"
#include "row_ops.cuh"

namespace abs_sgd {
namespace {

constexpr int kSms = 148;
constexpr uint64_t kSizeMax = 0x7fffffc0ull, kWidthMax = 1 << 23;     // tokens and vocab; width

// kE consecutive elements: of the activations (16 bytes, or single ones) and as fp32.
template <int kE>
__device__ __forceinline__ void load_f(const float* p, float (&v)[kE]) {
    if constexpr (kE == 1) v[0] = *p;
    else
#pragma unroll
        for (int i = 0; i < kE; i += 4) {
            const float4 f = *reinterpret_cast<const float4*>(p + i);
            v[i] = f.x; v[i + 1] = f.y; v[i + 2] = f.z; v[i + 3] = f.w;
        }
}
template <int kE>
__device__ __forceinline__ void store_f(float* p, const float (&v)[kE]) {
    if constexpr (kE == 1) *p = v[0];
    else
#pragma unroll
        for (int i = 0; i < kE; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
}

// Threads of a row: a power of two, so that a CTA of 256 threads takes 256 / lanes rows.
struct Lanes {
    int log;                 // lanes = 1 << log
    int pieces;              // of a row, kE elements each
};
Lanes lanes_for(uint64_t width, int elems) {
    Lanes l{0, (int)((width + elems - 1) / elems)};
    while (l.log < 8 && (1 << l.log) < l.pieces) ++l.log;
    return l;
}

template <typename T, int kE>
__global__ void __launch_bounds__(256) k_embed(const int32_t* ids, size_t tokens, const float* table, size_t ld_table, int vocab, float scale, T* y, size_t ld_y,
                                               Lanes l) {
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & ((1 << l.log) - 1), rows = 256 >> l.log;
    for (size_t t = (size_t)blockIdx.x * rows + (threadIdx.x >> l.log); t < tokens; t += (size_t)gridDim.x * rows) {
        const int id = ids[t];
        const bool known = id >= 0 && id < vocab;
        const float* from = table + (known ? (size_t)id : 0) * ld_table;
        T* to = y + t * ld_y;
#pragma unroll 2
        for (int j = lane; j < l.pieces; j += 1 << l.log) {
            float v[kE];
            if (known) {
                load_f<kE>(from + (size_t)j * kE, v);
#pragma unroll
                for (int i = 0; i < kE; ++i) v[i] *= scale;
            } else {
#pragma unroll
                for (int i = 0; i < kE; ++i) v[i] = 0.f;
            }
            Pack<T, kE>::store(to + (size_t)j * kE, v);
        }
    }
}

// ------------------------------------------------------------------------------------------------
// Tokens sorted by id: pairs (id, token), ids outside the vocabulary as `vocab`, behind all others.  Digits of kBits bits from the
// lowest; a pass counts each block's digits, adds the counts up over digits and blocks, and places the pairs.  Within a
// block a warp owns consecutive pairs and takes 32 at a time, in order: equal digits of the 32 find one another by
// match.any, so every pair's place is known without a comparison.  Up to kBlock tokens one CTA does all passes.
// ------------------------------------------------------------------------------------------------
constexpr int kBits = 8, kDigits = 1 << kBits;
constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32, kRounds = 16;
constexpr int kBlock = kSortThreads * kRounds;           // pairs of a block and step
constexpr int kBlocksMax = 512;

struct SortArgs {
    const int32_t* ids;
    int tokens, vocab;
    int blocks, steps;                                   // steps of kBlock pairs that a block takes, one after the other
    int passes;
    uint2* buf[2];                                       // pass p writes buf[p & 1]
    uint32_t* counts;                                    // [blocks][kDigits]
};

__device__ __forceinline__ uint2 pair_at(const SortArgs& a, int pass, int i) {
    if (pass > 0) return a.buf[(pass - 1) & 1][i];
    const int id = a.ids[i];
    return make_uint2(id >= 0 && id < a.vocab ? (uint32_t)id : (uint32_t)a.vocab, (uint32_t)i);
}
__device__ __forceinline__ uint32_t digit_of(uint2 p, int pass) { return p.x >> (pass * kBits) & (kDigits - 1); }

struct SortSmem {
    uint32_t warp[kSortWarps][kDigits];                  // a warp's count of a digit, then the first place of its pairs
    uint32_t base[kDigits];                              // first place of the block's pairs of a digit
    uint32_t scan[kSortWarps];
};

// Exclusive sum over kDigits values, one for each of the first kDigits threads; all threads call.
__device__ __forceinline__ uint32_t digit_scan(uint32_t v, SortSmem& s) {
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    uint32_t sum = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t w = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += w;
    }
    __syncthreads();
    if (lane == 31) s.scan[warp] = sum;
    __syncthreads();
    uint32_t before = 0;
#pragma unroll
    for (int w = 0; w < kDigits / 32; ++w) before += w < warp ? s.scan[w] : 0;
    return before + sum - v;
}

// Places the pairs first .. first + n - 1 (n <= kBlock); s.base moves on by what was placed.
__device__ void place_block(const SortArgs& a, SortSmem& s, int pass, int first, int n) {
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    uint2 p[kRounds];
    uint32_t rank[kRounds];
    for (int d = lane; d < kDigits; d += 32) s.warp[warp][d] = 0;
    __syncwarp();
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int i = (warp * kRounds + r) * 32 + lane;
        p[r] = i < n ? pair_at(a, pass, first + i) : make_uint2(0, 0);
    }
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const bool live = (warp * kRounds + r) * 32 + lane < n;
        const uint32_t d = live ? digit_of(p[r], pass) : kDigits;
        const uint32_t same = __match_any_sync(0xffffffffu, d);
        const uint32_t below = __popc(same & ((1u << lane) - 1));
        uint32_t at = 0;
        if (live) at = s.warp[warp][d];
        __syncwarp();
        if (live && below == 0) s.warp[warp][d] = at + __popc(same);
        __syncwarp();
        rank[r] = at + below;
    }
    __syncthreads();
    for (int d = threadIdx.x; d < kDigits; d += kSortThreads) {
        uint32_t at = s.base[d];
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) {
            const uint32_t c = s.warp[w][d];
            s.warp[w][d] = at;
            at += c;
        }
        s.base[d] = at;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
        if ((warp * kRounds + r) * 32 + lane < n) a.buf[pass & 1][s.warp[warp][digit_of(p[r], pass)] + rank[r]] = p[r];
    __syncthreads();
}

// The digits of pairs first .. first + n - 1 added to s.base.
__device__ void count_digits(const SortArgs& a, SortSmem& s, int pass, int first, int n) {
    for (int i = threadIdx.x; i < n; i += kSortThreads) atomicAdd(&s.base[digit_of(pair_at(a, pass, first + i), pass)], 1u);
}

__global__ void __launch_bounds__(kSortThreads) k_sort_small(const __grid_constant__ SortArgs a) {
    __shared__ SortSmem s;
    pdl_wait();
    pdl_trigger();
    for (int pass = 0; pass < a.passes; ++pass) {
        if (threadIdx.x < kDigits) s.base[threadIdx.x] = 0;
        __syncthreads();
        count_digits(a, s, pass, 0, a.tokens);
        __syncthreads();
        const uint32_t at = digit_scan(threadIdx.x < kDigits ? s.base[threadIdx.x] : 0, s);
        if (threadIdx.x < kDigits) s.base[threadIdx.x] = at;
        __syncthreads();
        place_block(a, s, pass, 0, a.tokens);            // its writes are read by the same CTA, behind a synchronisation
    }
}

__global__ void __launch_bounds__(kSortThreads) k_sort_count(const __grid_constant__ SortArgs a, int pass) {
    __shared__ SortSmem s;
    pdl_wait();
    pdl_trigger();
    if (threadIdx.x < kDigits) s.base[threadIdx.x] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * a.steps * kBlock;
    const int64_t n = min((int64_t)a.steps * kBlock, a.tokens - first);
    if (n > 0) count_digits(a, s, pass, (int)first, (int)n);
    __syncthreads();
    if (threadIdx.x < kDigits) a.counts[blockIdx.x * kDigits + threadIdx.x] = s.base[threadIdx.x];
}

__global__ void __launch_bounds__(kSortThreads) k_sort_place(const __grid_constant__ SortArgs a, int pass) {
    __shared__ SortSmem s;
    pdl_wait();
    pdl_trigger();
    uint32_t before = 0, all = 0;
    if (threadIdx.x < kDigits)
#pragma unroll 8
        for (int b = 0; b < a.blocks; ++b) {
            const uint32_t c = a.counts[b * kDigits + threadIdx.x];
            all += c;
            before += b < (int)blockIdx.x ? c : 0;
        }
    const uint32_t at = digit_scan(all, s);
    if (threadIdx.x < kDigits) s.base[threadIdx.x] = at + before;
    __syncthreads();
    for (int k = 0; k < a.steps; ++k) {
        const int64_t first = ((int64_t)blockIdx.x * a.steps + k) * kBlock;
        if (first >= a.tokens) break;
        place_block(a, s, pass, (int)first, (int)min((int64_t)kBlock, a.tokens - first));
    }
}

// ------------------------------------------------------------------------------------------------
// Sums over the sorted list.
// ------------------------------------------------------------------------------------------------
constexpr int kChunk = 32;                               // sorted tokens that a group of threads adds up

struct SumArgs {
    const uint2* list;
    const void* dy;
    size_t ld_dy;
    int tokens, vocab, D;
    float scale;
    float* out;
    size_t ld_out;
    int accumulate;
    Lanes l;
    int chunks, zero_ctas;                               // CTAs in front that write the rows of no token
    float* part;                                         // [chunk][2][width]: of the run that began before, of the one that goes on
    size_t width;
};

// The first place in the list whose id is at least v.
__device__ __forceinline__ int lower_bound(const uint2* list, int n, uint32_t v) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (list[mid].x < v) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

template <int kE>
__device__ __forceinline__ void put_row(const SumArgs& a, uint32_t id, int j, const float (&sum)[kE]) {
    float* p = a.out + (size_t)id * a.ld_out + (size_t)j * kE;
    float v[kE];
    if (a.accumulate) {
        load_f<kE>(p, v);
#pragma unroll
        for (int i = 0; i < kE; ++i) v[i] = fmaf(a.scale, sum[i], v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < kE; ++i) v[i] = a.scale * sum[i];
    }
    store_f<kE>(p, v);
}

template <typename T, int kE>
__global__ void __launch_bounds__(256) k_embed_sums(const __grid_constant__ SumArgs a) {
    pdl_wait();
    pdl_trigger();
    if ((int)blockIdx.x < a.zero_ctas) {                 // eight rows a warp: who has a token is looked up by a lane each
        const int lane = threadIdx.x % 32, warps = a.zero_ctas * 8;
        for (int64_t v0 = ((int64_t)blockIdx.x * 8 + threadIdx.x / 32) * 8; v0 < a.vocab; v0 += (int64_t)warps * 8) {
            bool absent = false;
            if (lane < 8 && v0 + lane < a.vocab) {
                const int at = lower_bound(a.list, a.tokens, (uint32_t)(v0 + lane));
                absent = at == a.tokens || a.list[at].x != (uint32_t)(v0 + lane);
            }
            uint32_t rows = __ballot_sync(0xffffffffu, absent);
            const float zero[kE] = {};
            while (rows) {
                const int r = __ffs(rows) - 1;
                rows &= rows - 1;
                for (int j = lane; j < a.l.pieces; j += 32) store_f<kE>(a.out + (size_t)(v0 + r) * a.ld_out + (size_t)j * kE, zero);
            }
        }
        return;
    }
    const int lane = threadIdx.x & ((1 << a.l.log) - 1), groups = 256 >> a.l.log;
    const int64_t chunk = (int64_t)(blockIdx.x - a.zero_ctas) * groups + (threadIdx.x >> a.l.log);
    if (chunk >= a.chunks) return;
    const int first = (int)(chunk * kChunk), n = min(kChunk, a.tokens - first);
    const uint32_t ahead = first > 0 ? a.list[first - 1].x : 0xffffffffu, behind = first + n < a.tokens ? a.list[first + n].x : 0xffffffffu;
    const int j = blockIdx.y * (1 << a.l.log) + lane;
    if (j >= a.l.pieces) return;
    const T* dy = static_cast<const T*>(a.dy) + (size_t)j * kE;
    float* part = a.part + (size_t)chunk * 2 * a.width + (size_t)j * kE;
    float sum[kE] = {};
    uint32_t id = a.list[first].x;
    bool began = id == ahead;                            // the current run began in a chunk before
    constexpr int kAhead = 8;
    for (int i0 = 0; i0 < n; i0 += kAhead) {
        uint2 p[kAhead];
        float v[kAhead][kE];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) p[k] = i0 + k < n ? a.list[first + i0 + k] : make_uint2(0xffffffffu, 0);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (p[k].x < (uint32_t)a.vocab) Pack<T, kE>::load(dy + (size_t)p[k].y * a.ld_dy, v[k]);
            else
#pragma unroll
                for (int i = 0; i < kE; ++i) v[k][i] = 0.f;
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (i0 + k >= n) break;
            if (p[k].x != id) {
                if (id < (uint32_t)a.vocab) {
                    if (began) store_f<kE>(part, sum);
                    else put_row<kE>(a, id, j, sum);
                }
                began = false;
                id = p[k].x;
#pragma unroll
                for (int i = 0; i < kE; ++i) sum[i] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < kE; ++i) sum[i] += v[k][i];
        }
    }
    if (id >= (uint32_t)a.vocab) return;
    if (began) store_f<kE>(part, sum);
    else if (id == behind) store_f<kE>(part + a.width, sum);
    else put_row<kE>(a, id, j, sum);
}

// The rows whose tokens pass the end of a chunk: that chunk's second partial sum, then the first ones of those behind it.
template <int kE>
__global__ void __launch_bounds__(256) k_embed_join(const __grid_constant__ SumArgs a) {
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & ((1 << a.l.log) - 1), groups = 256 >> a.l.log;
    const int64_t chunk = (int64_t)blockIdx.x * groups + (threadIdx.x >> a.l.log);
    if (chunk >= a.chunks - 1) return;
    const int first = (int)(chunk * kChunk), next = first + kChunk;
    const uint32_t id = a.list[next - 1].x;
    if (id != a.list[next].x || id >= (uint32_t)a.vocab || (first > 0 && a.list[first - 1].x == id)) return;
    const int last = lower_bound(a.list, a.tokens, id + 1) - 1, ends = last / kChunk;      // the chunk with the run's last token
    const int j = blockIdx.y * (1 << a.l.log) + lane;
    if (j >= a.l.pieces) return;
    const float* part = a.part + (size_t)j * kE;
    float sum[kE];
    load_f<kE>(part + ((size_t)chunk * 2 + 1) * a.width, sum);
#pragma unroll 4
    for (int64_t k = chunk + 1; k <= ends; ++k) {
        float v[kE];
        load_f<kE>(part + (size_t)k * 2 * a.width, v);
#pragma unroll
        for (int i = 0; i < kE; ++i) sum[i] += v[i];
    }
    put_row<kE>(a, id, j, sum);
}

struct EmbedPlan {
    int blocks, steps, passes, chunks;
    size_t width, list_bytes, count_bytes, part_bytes;
    size_t bytes() const { return 2 * list_bytes + count_bytes + part_bytes; }
};
EmbedPlan embed_plan(uint64_t tokens, uint64_t vocab, uint64_t width) {
    EmbedPlan p{};
    const uint64_t steps = (tokens + kBlock - 1) / kBlock;
    p.steps = (int)((steps + kBlocksMax - 1) / kBlocksMax);
    p.blocks = p.steps ? (int)((steps + p.steps - 1) / p.steps) : 0;
    p.passes = 1;
    while (p.passes * kBits < 32 && vocab >> (p.passes * kBits)) ++p.passes;       // the largest key is `vocab`
    p.chunks = (int)((tokens + kChunk - 1) / kChunk);
    p.width = (width + 7) / 8 * 8;
    p.list_bytes = up256(tokens * sizeof(uint2));
    p.count_bytes = p.blocks > 1 ? up256((size_t)p.blocks * kDigits * 4) : 0;
    p.part_bytes = p.chunks > 1 ? up256((size_t)p.chunks * 2 * p.width * 4) : 0;
    return p;
}

template <typename T, int kE>
cudaError_t sum_rows(SumArgs a, uint64_t width, cudaStream_t s) {
    a.l = lanes_for(width, kE);
    const int groups = 256 >> a.l.log;
    const unsigned slabs = (unsigned)((a.l.pieces + (1 << a.l.log) - 1) >> a.l.log);
    if (a.accumulate == 0) a.zero_ctas = (int)std::min<int64_t>(((int64_t)a.vocab + 63) / 64, kSms * 4);
    const unsigned ctas = (unsigned)((a.chunks + groups - 1) / groups);
    // rows of no token: only the first slab's CTAs write them, whole
    cudaError_t e = cudaSuccess;
    if (slabs == 1 || a.zero_ctas == 0) {
        e = launch_kernel(k_embed_sums<T, kE>, dim3(a.zero_ctas + ctas, slabs), 256, 0, s, true, a);
    } else {
        SumArgs z = a;
        z.chunks = 0;
        e = launch_kernel(k_embed_sums<T, kE>, dim3(a.zero_ctas), 256, 0, s, true, z);
        a.zero_ctas = 0;
        if (e == cudaSuccess) e = launch_kernel(k_embed_sums<T, kE>, dim3(ctas, slabs), 256, 0, s, true, a);
    }
    if (e == cudaSuccess && a.chunks > 1) e = launch_kernel(k_embed_join<kE>, dim3(ctas, slabs), 256, 0, s, true, a);
    return e;
}

}  // namespace
}  // namespace abs_sgd

using namespace abs_sgd;

extern "C" int abs_embed(const int32_t* ids, uint64_t tokens, const float* table, uint64_t ld_table, uint64_t vocab, uint64_t width, float scale, uint32_t dtype,
                         void* y, uint64_t ld_y, void* stream) {
    if (!known_dtype(dtype)) return thread_error(ABS_EINVAL, "dtype must be ABS_F32 or ABS_BF16");
    if (width == 0 || vocab == 0) return thread_error(ABS_EINVAL, "width and vocab must be at least 1");
    if (tokens > kSizeMax || vocab > kSizeMax || width > kWidthMax) return thread_error(ABS_ELIMIT, "tokens or vocab exceeds 2^31 - 64, or width 2^23");
    if (!isfinite(scale)) return thread_error(ABS_EINVAL, "scale must be finite");
    const MatrixArg m[2] = {{table, ld_table, width, 4}, {y, ld_y, width, size_of(dtype)}};
    if (const char* why = check_matrices(m)) return thread_error(ABS_EINVAL, why);
    if (misaligned(ids, 4)) return thread_error(ABS_EINVAL, "ids must be 4-byte aligned");
    if (tokens == 0) return ABS_OK;
    if (!ids || !table || !y) return thread_error(ABS_EINVAL, "ids, table and y must not be NULL");
    if (y == table) return thread_error(ABS_EINVAL, "y must not be the table");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    auto go = [&](auto kernel, auto zero, int elems) {
        const Lanes l = lanes_for(width, elems);
        const uint64_t rows = 256 >> l.log, want = (tokens + rows - 1) / rows;
        return launch_kernel(kernel, dim3((unsigned)std::min<uint64_t>(want, kSms * 64)), 256, 0, s, true, ids, (size_t)tokens, table, (size_t)ld_table, (int)vocab, scale,
                             static_cast<decltype(zero)*>(y), (size_t)ld_y, l);
    };
    const bool wide = rows_at(m[0], 16) && rows_at(m[1], 16) && width * m[1].es % 16 == 0;
    const cudaError_t e = dtype == ABS_F32 ? (wide ? go(k_embed<float, 4>, 0.f, 4) : go(k_embed<float, 1>, 0.f, 1))
                                           : (wide ? go(k_embed<bf16, 8>, bf16(), 8) : go(k_embed<bf16, 1>, bf16(), 1));
    return e == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(e));
}

extern "C" size_t abs_embed_backward_workspace(uint64_t tokens, uint64_t vocab, uint64_t width) {
    if (tokens > kSizeMax || vocab > kSizeMax || width > kWidthMax) return 0;
    return embed_plan(tokens, vocab, width).bytes();
}

extern "C" int abs_embed_backward(const void* dy, uint64_t ld_dy, uint32_t dtype, const int32_t* ids, uint64_t tokens, uint64_t vocab, uint64_t width, float scale,
                                  float* dtable, uint64_t ld_dtable, int accumulate, void* workspace, size_t workspace_bytes, void* stream) {
    if (!known_dtype(dtype)) return thread_error(ABS_EINVAL, "dtype must be ABS_F32 or ABS_BF16");
    if (width == 0 || vocab == 0) return thread_error(ABS_EINVAL, "width and vocab must be at least 1");
    if (tokens > kSizeMax || vocab > kSizeMax || width > kWidthMax) return thread_error(ABS_ELIMIT, "tokens or vocab exceeds 2^31 - 64, or width 2^23");
    if (!isfinite(scale)) return thread_error(ABS_EINVAL, "scale must be finite");
    const MatrixArg m[2] = {{dtable, ld_dtable, width, 4}, {dy, ld_dy, width, size_of(dtype)}};
    if (const char* why = check_matrices(m)) return thread_error(ABS_EINVAL, why);
    if (misaligned(ids, 4)) return thread_error(ABS_EINVAL, "ids must be 4-byte aligned");
    if (!dtable) return thread_error(ABS_EINVAL, "dtable must not be NULL");
    if (dy == dtable) return thread_error(ABS_EINVAL, "dtable must not be dy");
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    cudaError_t e = cudaSuccess;
    if (tokens == 0) {
        if (!accumulate) e = cudaMemset2DAsync(dtable, ld_dtable * 4, 0, width * 4, vocab, s);
        return e == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(e));
    }
    if (!ids || !dy) return thread_error(ABS_EINVAL, "ids and dy must not be NULL");
    const EmbedPlan p = embed_plan(tokens, vocab, width);
    if (!workspace || misaligned(workspace, 256)) return thread_error(ABS_EINVAL, "workspace must be non-NULL and 256-byte aligned");
    if (workspace_bytes < p.bytes()) return thread_error(ABS_ENOMEM, "workspace too small");
    char* ws = static_cast<char*>(workspace);
    SortArgs a{};
    a.ids = ids; a.tokens = (int)tokens; a.vocab = (int)vocab; a.blocks = p.blocks; a.steps = p.steps; a.passes = p.passes;
    a.buf[0] = reinterpret_cast<uint2*>(ws);
    a.buf[1] = reinterpret_cast<uint2*>(ws + p.list_bytes);
    a.counts = reinterpret_cast<uint32_t*>(ws + 2 * p.list_bytes);
    if (p.blocks == 1 && p.steps == 1) {
        e = launch_kernel(k_sort_small, 1, kSortThreads, 0, s, true, a);
    } else {
        for (int pass = 0; pass < p.passes && e == cudaSuccess; ++pass) {
            e = launch_kernel(k_sort_count, p.blocks, kSortThreads, 0, s, true, a, pass);
            if (e == cudaSuccess) e = launch_kernel(k_sort_place, p.blocks, kSortThreads, 0, s, true, a, pass);
        }
    }
    if (e != cudaSuccess) return thread_error(ABS_ECUDA, cudaGetErrorString(e));
    SumArgs q{};
    q.list = a.buf[(p.passes - 1) & 1]; q.dy = dy; q.ld_dy = ld_dy; q.tokens = (int)tokens; q.vocab = (int)vocab; q.D = (int)width; q.scale = scale;
    q.out = dtable; q.ld_out = ld_dtable; q.accumulate = accumulate != 0; q.chunks = p.chunks;
    q.part = reinterpret_cast<float*>(ws + 2 * p.list_bytes + p.count_bytes); q.width = p.width;
    const bool wide = rows_at(m[0], 16) && rows_at(m[1], 16) && width * m[1].es % 16 == 0;
    e = dtype == ABS_F32 ? (wide ? sum_rows<float, 4>(q, width, s) : sum_rows<float, 1>(q, width, s))
                         : (wide ? sum_rows<bf16, 8>(q, width, s) : sum_rows<bf16, 1>(q, width, s));
    return e == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(e));
}
