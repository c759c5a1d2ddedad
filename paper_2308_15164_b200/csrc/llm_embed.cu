// Scaled embedding lookup and its gradient (abs_embed*).
//
// Forward: a gather of rows, bound by memory.  Backward: the tokens are sorted by id (a stable radix sort, so that a row's tokens
// stay in their order), the sorted list is cut into chunks of equal length, each summed row by row; a row whose tokens pass a
// chunk's border leaves partial sums that a last kernel adds up in order.  No additions whose order could change: equal inputs give
// equal bits, and a token that fills half the micro-batch costs no more than the others.
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
// match.any, so every pair's place is known without a comparison.  Up to kBlock tokens one CTA does all passes, up to kClusterMost a
// cluster of eight, in one launch (8192 tokens: 13 us, one CTA 27); more tokens take two launches a pass (65536: 24 us, one cluster 38).
// ------------------------------------------------------------------------------------------------
constexpr int kBits = 8, kDigits = 1 << kBits;
constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32, kRounds = 4;
constexpr int kBlock = kSortThreads * kRounds;           // pairs of a block and step
constexpr int kBlocksMax = 512;
constexpr int kCluster = 8, kClusterMost = kCluster * kBlock;

// Rows of the table, first .. last - 1, that are cleared meanwhile by the CTAs that do not sort: all rows are, before the sums go to those
// that have a token (8192 tokens have some 3000 of 32000).
struct Clear {
    float* out;
    size_t ld;
    int64_t first, last;
    int width, wide;                                     // wide: rows of whole 16-byte pieces, aligned
};

struct SortArgs {
    const int32_t* ids;
    int tokens, vocab;
    int blocks, steps;                                   // steps of kBlock pairs that a block takes, one after the other
    int passes;
    uint2* buf[2];                                       // pass p writes buf[p & 1]
    uint32_t* counts;                                    // [blocks][kDigits]
};

__device__ __forceinline__ uint2 pair_at(const SortArgs& a, int pass, int i) {
    if (pass > 0) return __ldcg(a.buf[(pass - 1) & 1] + i);
    const int id = a.ids[i];
    return make_uint2(id >= 0 && id < a.vocab ? (uint32_t)id : (uint32_t)a.vocab, (uint32_t)i);
}
__device__ __forceinline__ uint32_t digit_of(uint2 p, int pass) { return p.x >> (pass * kBits) & (kDigits - 1); }

struct SortSmem {
    uint32_t warp[kSortWarps][kDigits];                  // a warp's count of a digit, then the first place of its pairs
    uint32_t base[kDigits];                              // first place of the block's pairs of a digit
    uint32_t scan[kSortWarps];
};

// By the CTAs from `first_cta` on.
__device__ __forceinline__ void clear_rows(const Clear& c, int first_cta) {
    const int64_t rows = c.last - c.first, at = (int64_t)(blockIdx.x - first_cta) * kSortThreads + threadIdx.x, all = (int64_t)(gridDim.x - first_cta) * kSortThreads;
    float* from = c.out + c.first * (int64_t)c.ld;
    const bool packed = c.ld == (size_t)c.width;         // one piece of memory
    const int64_t lines = packed ? 1 : rows, length = packed ? rows * c.width : c.width;
    if (c.wide) {
        const int64_t pieces = length / 4;
        if (packed) {
#pragma unroll 4
            for (int64_t i = at; i < pieces; i += all) reinterpret_cast<float4*>(from)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        } else {
            for (int64_t i = at; i < lines * pieces; i += all) {
                const int64_t r = i / pieces;
                *reinterpret_cast<float4*>(from + r * (int64_t)c.ld + (i - r * pieces) * 4) = make_float4(0.f, 0.f, 0.f, 0.f);
            }
        }
    } else {
        for (int64_t i = at; i < lines * length; i += all) {
            const int64_t r = packed ? 0 : i / length;
            from[r * (int64_t)c.ld + (i - r * length)] = 0.f;
        }
    }
}

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

__global__ void __launch_bounds__(kSortThreads) k_sort_small(const __grid_constant__ SortArgs a, const __grid_constant__ Clear c) {
    __shared__ SortSmem s;
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x > 0) return clear_rows(c, 1);
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

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The first cluster sorts, a run of the tokens for each CTA; the others clear.
__global__ void __launch_bounds__(kSortThreads) k_sort_cluster(const __grid_constant__ SortArgs a, const __grid_constant__ Clear c) {
    __shared__ SortSmem s;
    if (blockIdx.x >= kCluster) return clear_rows(c, kCluster);
    const int per = (a.tokens + kCluster - 1) / kCluster, first = min((int)blockIdx.x * per, a.tokens), n = min(per, a.tokens - first);
    for (int pass = 0; pass < a.passes; ++pass) {
        if (threadIdx.x < kDigits) s.base[threadIdx.x] = 0;
        __syncthreads();
        count_digits(a, s, pass, first, n);
        __syncthreads();
        if (threadIdx.x < kDigits) a.counts[blockIdx.x * kDigits + threadIdx.x] = s.base[threadIdx.x];
        __threadfence();
        cluster_sync();
        uint32_t before = 0, all = 0;
        if (threadIdx.x < kDigits)
#pragma unroll
            for (int b = 0; b < kCluster; ++b) {
                const uint32_t v = __ldcg(a.counts + b * kDigits + threadIdx.x);
                all += v;
                before += b < (int)blockIdx.x ? v : 0;
            }
        const uint32_t at = digit_scan(all, s);
        if (threadIdx.x < kDigits) s.base[threadIdx.x] = at + before;
        __syncthreads();
        for (int k = 0; k < n; k += kBlock) place_block(a, s, pass, first + k, min(kBlock, n - k));
        __threadfence();
        cluster_sync();              // all pairs are placed, all counts read
    }
}

__global__ void __launch_bounds__(kSortThreads) k_sort_count(const __grid_constant__ SortArgs a, const __grid_constant__ Clear c, int pass) {
    __shared__ SortSmem s;
    pdl_wait();
    pdl_trigger();
    if ((int)blockIdx.x >= a.blocks) return clear_rows(c, a.blocks);
    if (threadIdx.x < kDigits) s.base[threadIdx.x] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * a.steps * kBlock;
    const int64_t n = min((int64_t)a.steps * kBlock, a.tokens - first);
    if (n > 0) count_digits(a, s, pass, (int)first, (int)n);
    __syncthreads();
    if (threadIdx.x < kDigits) a.counts[blockIdx.x * kDigits + threadIdx.x] = s.base[threadIdx.x];
}

__global__ void __launch_bounds__(kSortThreads) k_sort_place(const __grid_constant__ SortArgs a, const __grid_constant__ Clear c, int pass) {
    __shared__ SortSmem s;
    pdl_wait();
    pdl_trigger();
    if ((int)blockIdx.x >= a.blocks) return clear_rows(c, a.blocks);
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

struct SumArgs {
    const uint2* list;
    const void* dy;
    size_t ld_dy;
    int tokens, vocab;
    float scale;
    float* out;
    size_t ld_out;
    int accumulate;
    Lanes l;
    int chunk, chunks;                                   // sorted tokens that a group of threads adds up
    float* part;                                         // [chunk][2][width]: of the run that began before, of the one that goes on
    size_t width;
};

// A row's sum; accumulate: one addition for each element, by the memory (nobody else adds to it, so that the order is no matter; read, added and
// written by the thread, a chunk's rows wait for one another: 16 us instead of 5 for 8192 x 64).  The memory takes numbers below 2^-126 for zero, what it
// adds, what it adds to and what comes out.
template <int kE>
__device__ __forceinline__ void put_row(const SumArgs& a, uint32_t id, int j, const float (&sum)[kE]) {
    float* p = a.out + (size_t)id * a.ld_out + (size_t)j * kE;
    float v[kE];
#pragma unroll
    for (int i = 0; i < kE; ++i) v[i] = a.scale * sum[i];
    if (!a.accumulate) return store_f<kE>(p, v);
    if constexpr (kE == 1) {
        asm volatile("red.relaxed.gpu.global.add.f32 [%0], %1;" ::"l"(p), "f"(v[0]) : "memory");
    } else {
#pragma unroll
        for (int i = 0; i < kE; i += 4)
            asm volatile("red.relaxed.gpu.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(p + i), "f"(v[i]), "f"(v[i + 1]), "f"(v[i + 2]), "f"(v[i + 3]) : "memory");
    }
}

// kE elements as they lie in memory, and their sums (pairs: two fp32 additions an instruction).
template <typename T, int kE>
struct Raw {
    uint4 w;
    __device__ __forceinline__ void load(const T* p) { w = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void clear() { w = make_uint4(0, 0, 0, 0); }
};
template <typename T>
struct Raw<T, 1> {
    T w;
    __device__ __forceinline__ void load(const T* p) { w = *p; }
    __device__ __forceinline__ void clear() { w = from_f<T>(0.f); }
};
template <typename T, int kE>
struct Sums {
    float2 v[kE / 2];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < kE / 2; ++i) v[i] = both(0.f);
    }
    __device__ __forceinline__ void add(const Raw<T, kE>& r) {
        float2 u[kE / 2];
        unpack(r.w, u, T());
#pragma unroll
        for (int i = 0; i < kE / 2; ++i) v[i] = add2(v[i], u[i]);
    }
    __device__ __forceinline__ void get(float (&f)[kE]) const {
#pragma unroll
        for (int i = 0; i < kE; ++i) f[i] = i % 2 ? v[i / 2].y : v[i / 2].x;
    }
};
template <typename T>
struct Sums<T, 1> {
    float v;
    __device__ __forceinline__ void clear() { v = 0.f; }
    __device__ __forceinline__ void add(const Raw<T, 1>& r) { v += to_f(r.w); }
    __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = v; }
};

template <typename T, int kE>
__global__ void __launch_bounds__(256, 4) k_embed_sums(const __grid_constant__ SumArgs a) {
    pdl_wait();
    pdl_trigger();
    const int lane = threadIdx.x & ((1 << a.l.log) - 1), groups = 256 >> a.l.log;
    const int64_t chunk = (int64_t)blockIdx.x * groups + (threadIdx.x >> a.l.log);
    if (chunk >= a.chunks) return;
    const int first = (int)(chunk * a.chunk), n = min(a.chunk, a.tokens - first);
    const uint2* list = a.list + first;
    const uint32_t ahead = first > 0 ? list[-1].x : 0xffffffffu, behind = first + n < a.tokens ? list[n].x : 0xffffffffu;
    const int j = blockIdx.y * (1 << a.l.log) + lane;
    if (j >= a.l.pieces) return;
    const T* dy = static_cast<const T*>(a.dy) + (size_t)j * kE;
    float* part = a.part + (size_t)chunk * 2 * a.width + (size_t)j * kE;
    Sums<T, kE> sum;
    sum.clear();
    uint32_t id = list[0].x;
    bool began = id == ahead;                            // the current run began in a chunk before
    // to: where a run that is not the table's row alone goes
    auto put = [&](float* to, bool whole) {
        float v[kE];
        sum.get(v);
        if (whole) put_row<kE>(a, id, j, v);
        else store_f<kE>(to, v);
    };
    constexpr int kAhead = 8;                            // rows in flight
    for (int i0 = 0; i0 < n; i0 += kAhead) {
        uint2 p[kAhead];
        Raw<T, kE> v[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) p[k] = i0 + k < n ? list[i0 + k] : make_uint2(0xffffffffu, 0);     // beyond the list: another run
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            v[k].clear();
            if (p[k].x < (uint32_t)a.vocab) v[k].load(dy + (size_t)p[k].y * a.ld_dy);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (p[k].x != id) {
                if (id < (uint32_t)a.vocab) put(part, !began);
                began = false;
                id = p[k].x;
                sum.clear();
            }
            sum.add(v[k]);
        }
    }
    if (id >= (uint32_t)a.vocab) return;
    if (began) put(part, false);
    else put(part + a.width, id != behind);
}

// The rows whose tokens pass the end of a chunk: that chunk's second partial sum, then the first ones of those behind it, a CTA for each.
// The CTA's groups of threads take the chunks behind in turn, four loads each in flight; their sums are added up in order.
template <int kE>
__global__ void __launch_bounds__(256) k_embed_join(const __grid_constant__ SumArgs a) {
    __shared__ float sh[256][kE];
    pdl_wait();
    pdl_trigger();
    const int chunk = blockIdx.x, first = chunk * a.chunk, next = first + a.chunk;
    const uint32_t id = a.list[next - 1].x;
    if (id != a.list[next].x || id >= (uint32_t)a.vocab || (first > 0 && a.list[first - 1].x == id)) return;
    int64_t behind = 0;                                  // chunks behind that the run goes into
    for (bool all = true; all;) {
        const int64_t k = chunk + 1 + behind + threadIdx.x % 32;
        const uint32_t on = __ballot_sync(0xffffffffu, k < a.chunks && a.list[k * a.chunk].x == id);
        all = on == 0xffffffffu;
        behind += __popc(on);
    }
    const size_t step = 2 * a.width;
    const int lanes = 1 << a.l.log, lane = threadIdx.x & (lanes - 1), line = threadIdx.x >> a.l.log, lines = 256 >> a.l.log;
    for (int j0 = 0; j0 < a.l.pieces; j0 += lanes) {
        const int j = j0 + lane;
        const float* part = a.part + (size_t)chunk * step + (size_t)min(j, a.l.pieces - 1) * kE;
        float sum[kE] = {};
        if (line == 0) load_f<kE>(part + a.width, sum);
        for (int64_t k0 = 1 + line * 4; k0 <= behind; k0 += lines * 4) {
            float v[4][kE];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k0 + k <= behind) load_f<kE>(part + (size_t)(k0 + k) * step, v[k]);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (k0 + k <= behind)
#pragma unroll
                    for (int i = 0; i < kE; ++i) sum[i] += v[k][i];
        }
        if (lines > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kE; ++i) sh[threadIdx.x][i] = sum[i];
            __syncthreads();
            for (int w = 1; w < lines && line == 0; ++w)
#pragma unroll
                for (int i = 0; i < kE; ++i) sum[i] += sh[w * lanes + lane][i];
        }
        if (line == 0 && j < a.l.pieces) put_row<kE>(a, id, j, sum);
    }
}

// Few tokens: each looks for its own kind among all of them, the first of a kind adds them up; the other rows are cleared by the CTAs
// behind.  One launch instead of three.
constexpr int kFew = 128;
template <typename T, int kE>
__global__ void __launch_bounds__(256) k_embed_few(const __grid_constant__ SumArgs a, const int32_t* ids, int token_ctas) {
    __shared__ int32_t sh[kFew];
    pdl_wait();
    pdl_trigger();
    for (int t = threadIdx.x; t < kFew; t += 256) sh[t] = t < a.tokens ? ids[t] : -1;
    __syncthreads();
    if ((int)blockIdx.x >= token_ctas) {                 // four rows a warp
        const int lane = threadIdx.x % 32;
        const int64_t step = (int64_t)(gridDim.x - token_ctas) * 8 * 4;
        for (int64_t v0 = ((int64_t)(blockIdx.x - token_ctas) * 8 + threadIdx.x / 32) * 4; v0 < a.vocab; v0 += step)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                bool here = false;
#pragma unroll
                for (int t = 0; t < kFew; t += 32) here = here || sh[t + lane] == (int)(v0 + r);
                if (__any_sync(0xffffffffu, here) || v0 + r >= a.vocab) continue;
                const float zero[kE] = {};
#pragma unroll 4
                for (int j = lane; j < a.l.pieces; j += 32) store_f<kE>(a.out + (size_t)(v0 + r) * a.ld_out + (size_t)j * kE, zero);
            }
        return;
    }
    const int lane = threadIdx.x & ((1 << a.l.log) - 1), t = blockIdx.x * (256 >> a.l.log) + (threadIdx.x >> a.l.log);
    if (t >= a.tokens || sh[t] < 0 || sh[t] >= a.vocab) return;
    const int id = sh[t];
    uint32_t same[kFew / 32];
#pragma unroll
    for (int w = 0; w < kFew / 32; ++w) {
        same[w] = 0;
#pragma unroll 8
        for (int i = 0; i < 32; ++i) same[w] |= (sh[w * 32 + i] == id ? 1u : 0u) << i;
    }
#pragma unroll
    for (int w = 0; w < kFew / 32; ++w) {
        const uint32_t front = t >= w * 32 + 32 ? 0xffffffffu : t > w * 32 ? (1u << (t - w * 32)) - 1 : 0u;
        if (same[w] & front) return;                     // not the first of its kind
    }
    for (int j = lane; j < a.l.pieces; j += 1 << a.l.log) {
        const T* dy = static_cast<const T*>(a.dy) + (size_t)j * kE;
        float sum[kE] = {};
#pragma unroll
        for (int w = 0; w < kFew / 32; ++w) {
            uint32_t left = same[w];
            while (left) {
                constexpr int kAhead = 4;
                float v[kAhead][kE];
                bool have[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    have[k] = left != 0;
                    if (have[k]) Pack<T, kE>::load(dy + (size_t)(w * 32 + __ffs(left) - 1) * a.ld_dy, v[k]);
                    left &= left - 1;
                }
#pragma unroll
                for (int k = 0; k < kAhead; ++k)
                    if (have[k])
#pragma unroll
                        for (int i = 0; i < kE; ++i) sum[i] += v[k][i];
            }
        }
        put_row<kE>(a, (uint32_t)id, j, sum);
    }
}

struct EmbedPlan {
    int blocks, steps, passes, chunk, chunks;
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
    // as long as that leaves some 128 thousand threads: a run's partial sums are added up by one CTA
    const uint64_t most = (tokens << lanes_for(width, 8).log) >> 17;
    for (p.chunk = 16; p.chunk < 256 && (uint64_t)p.chunk * 2 <= most;) p.chunk *= 2;
    p.chunks = (int)((tokens + p.chunk - 1) / p.chunk);
    p.width = (width + 7) / 8 * 8;
    p.list_bytes = up256(tokens * sizeof(uint2));
    p.count_bytes = p.blocks > 1 ? up256((size_t)std::max(p.blocks, kCluster) * kDigits * 4) : 0;
    p.part_bytes = p.chunks > 1 ? up256((size_t)p.chunks * 2 * p.width * 4) : 0;
    return p;
}

template <typename T, int kE>
cudaError_t sum_rows(SumArgs a, uint64_t width, const int32_t* few, cudaStream_t s) {
    a.l = lanes_for(width, kE);
    const int groups = 256 >> a.l.log;
    if (few) {
        const unsigned tokens = (unsigned)((a.tokens + groups - 1) / groups), rows = a.accumulate ? 0 : (unsigned)std::min<int64_t>(((int64_t)a.vocab + 31) / 32, kSms * 8);
        return launch_kernel(k_embed_few<T, kE>, tokens + rows, 256, 0, s, true, a, few, (int)tokens);
    }
    const dim3 grid((unsigned)((a.chunks + groups - 1) / groups), (unsigned)((a.l.pieces + (1 << a.l.log) - 1) >> a.l.log));
    const cudaError_t e = launch_kernel(k_embed_sums<T, kE>, grid, 256, 0, s, true, a);
    if (e != cudaSuccess || a.chunks == 1) return e;
    return launch_kernel(k_embed_join<kE>, a.chunks - 1, 256, 0, s, true, a);
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
    const bool wide = rows_at(m[0], 16) && rows_at(m[1], 16) && width * m[1].es % 16 == 0;
    const bool few = tokens <= (uint64_t)kFew;
    if (!few) {
        const bool one = p.blocks == 1, cluster = !one && tokens <= (uint64_t)kClusterMost;
        const int launches = one || cluster ? 1 : 2 * p.passes;
        const int clear = accumulate ? 0 : (int)std::min<uint64_t>(vocab * width / launches / (4 * kSortThreads) + 1, 3 * kSms);
        Clear c{dtable, (size_t)ld_dtable, 0, 0, (int)width, rows_at(m[0], 16) && width % 4 == 0};
        for (int i = 0; i < launches && e == cudaSuccess; ++i) {
            c.first = c.last;
            c.last = (int64_t)(vocab * (i + 1) / launches);
            if (one) e = launch_kernel(k_sort_small, 1 + clear, kSortThreads, 0, s, true, a, c);
            else if (cluster) e = launch_cluster(k_sort_cluster, kCluster + (clear + kCluster - 1) / kCluster * kCluster, kCluster, kSortThreads, 0, s, a, c);
            else e = launch_kernel(i % 2 ? k_sort_place : k_sort_count, p.blocks + clear, kSortThreads, 0, s, true, a, c, i / 2);
        }
        if (e != cudaSuccess) return thread_error(ABS_ECUDA, cudaGetErrorString(e));
    }
    SumArgs q{};
    q.list = a.buf[(p.passes - 1) & 1]; q.dy = dy; q.ld_dy = ld_dy; q.tokens = (int)tokens; q.vocab = (int)vocab; q.scale = scale;
    q.out = dtable; q.ld_out = ld_dtable; q.accumulate = accumulate != 0; q.chunk = p.chunk; q.chunks = p.chunks;
    q.part = reinterpret_cast<float*>(ws + 2 * p.list_bytes + p.count_bytes); q.width = p.width;
    const int32_t* all = few ? ids : nullptr;
    e = dtype == ABS_F32 ? (wide ? sum_rows<float, 4>(q, width, all, s) : sum_rows<float, 1>(q, width, all, s))
                         : (wide ? sum_rows<bf16, 8>(q, width, all, s) : sum_rows<bf16, 1>(q, width, all, s));
    return e == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(e));
}
