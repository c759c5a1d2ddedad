// Gated linear recurrence over packed sequences (abs_recurrence*).
//
//     h_t = a_t h_{t-1} + b_t,   a = sigmoid(g),  b = (1 - a) x  or  x
// Composed, rows i..j act on the state in front of them as h -> A h + B with A = a_i ... a_j, and two such maps compose to
// (A2 A1, A2 B1 + B2): that is what lets a long sequence be worked on in parallel.  Backward with e_t = a_t d_t, what row t hands
// to row t - 1, is the same recurrence in reversed time: e_t = a_t e_{t+1} + a_t dy_t, d_t = dy_t + e_{t+1}.
// A sequence's first row forgets what is in front of it; as a map that is A = -0, which stays -0 in every product with later
// factors (a >= +0) and is told from an underflow by its sign, so that no infinity or NaN of one sequence reaches the next.
// Two passes: the maps of a strip's segments, then the rows from the states that follow from them; equal inputs give equal bits.  Bound by memory,
// forward 3 and backward 6 elements per position; the first pass reads 2 of them once more, but only behind the last begin of a sequence in a
// segment, and in an order that leaves what the second reads first in L2.  us, bf16: 65536 x 1024 118-127, 16384 x 4096 of 24 sequences 107-110, their
// gradients 203-212 and 152-170.  (One pass with tiles that wait for the tiles in front of them, 65536 x 1024: 296.  The tiles that run together
// all wait for the same few, and what they hold in registers is too little to hide that.)
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "abs_internal.h"
#include "abs_llm.h"
#include "llm_host.h"
#include "llm_status.cuh"
#include "row_ops.cuh"
#include "tcgen05.cuh"

namespace abs_sgd {
namespace {

constexpr int kWarps = 8, kCols = 64;    // of a tile; a lane owns two columns
constexpr int kSms = 148;
constexpr uint64_t kSizeMax = 0x7ffffc00ull;
// Rows of a warp, 16 forward and 8 backward (bf16): 32 KB of inputs for a tile, backward 16 KB in the first pass; three tiles in flight.  CTAs of an SM: as
// many as its shared memory holds.  us, 65536 x 1024 one sequence forward / 16384 x 4096 of 24 sequences backward, bf16: as here 118 / 152; forward first
// pass with two tiles in flight and three CTAs an SM 131 (the SMs that are free first take three, others are left with one); with 8 rows a warp and four CTAs
// 131; backward first pass with 16 160; backward with three CTAs an SM and two tiles in flight 193; forward with 8 rows and four CTAs 138.
template <typename T, bool kBack, bool kMaps>
constexpr int kRowsOf = (kBack ? 8 : 16) * 2 / (int)sizeof(T);
template <typename T, bool kBack, bool kMaps>
constexpr int kTileOf = kWarps * kRowsOf<T, kBack, kMaps>;
constexpr int kStages = 3;               // tiles in flight
template <bool kBack, bool kMaps>
constexpr int kCtasOf = kBack && kMaps ? 3 : 2;          // of an SM
template <bool kBack, bool kMaps>
constexpr int kStageBytes = kBack && kMaps ? 16384 : 32768;
constexpr int kTileMin = kTileOf<float, true, false>;

struct RecArgs {
    const void *x, *g, *dy, *y;          // y: of the forward pass (backward only)
    size_t ld_x, ld_g, ld_dy, ld_y;
    void *out, *out2;                    // forward: y; backward: dx, dg
    size_t ld_out, ld_out2;
    const int32_t* offsets;
    const float *h0, *before;            // before: h0, backward dlast: the state in front of a sequence in scan order
    float* after;                        // last, backward dh0
    int T, D, seqs;
    int strips;
    int segs, rows;                      // segments, rows of one (a multiple of a tile; the last may have fewer)
    int parts, part_rows;                // of a segment, in the first pass: a map for each
    int pairs;                           // a lane's two columns are aligned to two elements in every matrix
    struct Map* maps;                    // [segment][part][strip][lane]
};

// sigmoid(g) and 1 - sigmoid(g), each to its own precision.
__device__ __forceinline__ void gate_of(float2 g, float2& a, float2& rest, bf16) {
    float2 v = mul2(g, both(-1.4426950408889634f));
    asm("min.NaN.f32 %0, %0, 0f42FC0000;" : "+f"(v.x));  // 126
    asm("min.NaN.f32 %0, %0, 0f42FC0000;" : "+f"(v.y));
    const float2 e = exp2_of(v), d = add2(e, both(1.f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a.x) : "f"(d.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a.y) : "f"(d.y));
    rest = mul2(e, a);
}
__device__ __forceinline__ void gate_of(float2 g, float2& a, float2& rest, float) {
    const float2 e = make_float2(expf(g.x < -87.f ? 87.f : -g.x), expf(g.y < -87.f ? 87.f : -g.y));
    const float2 d = add2(e, both(1.f));         // at most 2^126
    float2 r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(d.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(d.y));
    // a step of Newton's method: half a unit in the last place, as a division has, instead of one (a state lives through many gates)
    a = fma2(r, fma2(make_float2(-d.x, -d.y), r, both(1.f)), r);
    rest = mul2(e, a);
}
// The maps of two columns.
struct alignas(16) Map {
    float2 A, B;
};
__device__ __forceinline__ Map identity() { return {make_float2(1.f, 1.f), make_float2(0.f, 0.f)}; }
__device__ __forceinline__ bool forgets(float A) { return __float_as_uint(A) == 0x80000000u; }
__device__ __forceinline__ bool no_number(float2 v) { return v.x != v.x || v.y != v.y; }
// A s + B.  No gate is zero, so that an infinite state stays infinite; behind so many rows that their A has fallen to zero, the product with it
// is a NaN.  kInfinite: with that in mind.  The runs of maps below are gone through without, and once more where they end in a NaN.
template <bool kInfinite>
__device__ __forceinline__ float2 along(float2 A, float2 s, float2 B) {
    float2 r = fma2(A, s, B);
    if (kInfinite && A.x == 0.f && isinf(s.x)) r.x = s.x + B.x;
    if (kInfinite && A.y == 0.f && isinf(s.y)) r.y = s.y + B.y;
    return r;
}
// m followed by `then`; kForgets: either may forget what is in front of it.
template <bool kForgets, bool kInfinite = false>
__device__ __forceinline__ Map compose(Map m, Map then) {
    Map r{mul2(m.A, then.A), along<kInfinite>(then.A, m.B, then.B)};
    if (kForgets && forgets(then.A.x)) {
        r.A.x = then.A.x;
        r.B.x = then.B.x;
    }
    if (kForgets && forgets(then.A.y)) {
        r.A.y = then.A.y;
        r.B.y = then.B.y;
    }
    return r;
}
template <bool kForgets, bool kInfinite = false>
__device__ __forceinline__ float2 apply(Map m, float2 s) {
    float2 r = along<kInfinite>(m.A, s, m.B);
    if (kForgets && forgets(m.A.x)) r.x = m.B.x;
    if (kForgets && forgets(m.A.y)) r.y = m.B.y;
    return r;
}

// Two elements from shared or aligned global memory; n of two elements at any address.
__device__ __forceinline__ float2 pair_of(const float* p) { return *reinterpret_cast<const float2*>(p); }
__device__ __forceinline__ float2 pair_of(const bf16* p) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(p);
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <typename T>
__device__ __forceinline__ float2 load2(const T* p, int n, bool aligned) {
    if (n == 2 && aligned) return pair_of(p);
    return make_float2(n > 0 ? to_f(p[0]) : 0.f, n > 1 ? to_f(p[1]) : 0.f);
}
__device__ __forceinline__ void put_pair(float* p, float2 v) { *reinterpret_cast<float2*>(p) = v; }
__device__ __forceinline__ void put_pair(bf16* p, float2 v) { *reinterpret_cast<__nv_bfloat162*>(p) = __float22bfloat162_rn(v); }
template <typename T>
__device__ __forceinline__ void store2(T* p, int n, bool aligned, float2 v) {
    if (n == 2 && aligned) return put_pair(p, v);
    if (n > 0) p[0] = from_f<T>(v.x);
    if (n > 1) p[1] = from_f<T>(v.y);
}

// Which sequence row t belongs to: the number of sequences that end at or before it.
__device__ __forceinline__ int begin_of(const RecArgs& a, int q) { return a.offsets ? min(max(a.offsets[q], 0), a.T) : q == 0 ? 0 : a.T; }
// The same row for all lanes of a warp, 32 ends looked at in a step.
__device__ __forceinline__ int sequence_of(const RecArgs& a, int t) {
    int lo = 0, hi = a.seqs;
    while (lo < hi) {
        const int step = (hi - lo + 31) / 32;
        const int64_t at = lo + (int64_t)(threadIdx.x % 32 + 1) * step - 1;
        const bool over = at < hi && begin_of(a, (int)at + 1) <= t;
        lo += __popc(__ballot_sync(0xffffffffu, over)) * step;
        hi = min(hi, lo + step - 1);
    }
    return lo;
}
// From a sequence at or before that of row t on.
__device__ __forceinline__ int sequence_from(const RecArgs& a, int q, int t) {
    for (int i = 0; i < 4 && q < a.seqs && begin_of(a, q + 1) <= t; ++i) ++q;
    int hi = a.seqs;
    while (q < hi && begin_of(a, q + 1) <= t) {
        const int mid = q + (hi - q) / 2;
        if (begin_of(a, mid + 1) <= t) q = mid + 1;
        else hi = mid;
    }
    return q;
}

template <bool kMaps>
struct RecSmem {
    Map map[2][kWarps][32];                      // of a warp's rows, by the tile's parity
    Map front[kMaps ? 1 : kWarps][kMaps ? 1 : 32];       // second pass: of the segments in front, a run of them for each warp
    alignas(8) uint64_t full[kStages];
    int failed[2];
};
template <bool kMaps>
constexpr size_t kRecSmem = (sizeof(RecSmem<kMaps>) + 127) / 128 * 128;
// Dynamic shared memory of a CTA; where the lanes read memory no tiles.
template <bool kBack, bool kMaps>
constexpr size_t smem_bytes(bool tma) { return kRecSmem<kMaps> + (tma ? kStages * kStageBytes<kBack, kMaps> : 0) + 128; }
// The CTAs that the plan counts on fit (of an SM's 228 KB, 1 KB a CTA is the system's).
template <bool kBack, bool kMaps>
constexpr bool kFits = kCtasOf<kBack, kMaps> * (smem_bytes<kBack, kMaps>(true) + 1024) <= 228 * 1024;
static_assert(kFits<false, false> && kFits<false, true> && kFits<true, false> && kFits<true, true>, "");

// A CTA takes a segment of a strip of 64 columns, tile by tile (kTileOf rows in scan order: backward from the last one).
//   kMaps   the segment's map: from its last tile to its first, or to the first in which a sequence begins (nothing in front of that
//           matters), so that what was read last is what the second pass reads first
//   else    the state in front of the segment from the maps of those in front, in order; then for each tile
//             1. a lane reads its rows of two columns, forms the gates, and the map of its warp's rows
//             2. the maps of the warps in front give the state in front of its rows, those of all warps the state of the next tile
//             3. it goes over its rows again
// kTma: the next tiles are copied to shared memory meanwhile.  Otherwise (rows that are not 16-byte aligned) the lanes read memory.
template <typename T, uint32_t kKind, bool kBack, bool kTma, bool kMaps>
__global__ void __launch_bounds__(kWarps * 32, kCtasOf<kBack, kMaps>) k_recurrence(const __grid_constant__ RecArgs a, const __grid_constant__ CUtensorMap tm_g,
                                                                            const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_dy,
                                                                            const __grid_constant__ CUtensorMap tm_y) {
    constexpr int kRows = kRowsOf<T, kBack, kMaps>, kTile = kTileOf<T, kBack, kMaps>;
    constexpr int kInput = kTile * kCols * (int)sizeof(T);       // bytes of an input's tile
    constexpr int kInputs = kBack && !kMaps ? 4 : 2;
    static_assert(kInput * kInputs == kStageBytes<kBack, kMaps>, "");
    enum { kG, kIn, kX, kY };                                    // kIn: x, backward dy; kX backward only
    extern __shared__ uint8_t raw[];
    RecSmem<kMaps>& s = *reinterpret_cast<RecSmem<kMaps>*>((reinterpret_cast<uintptr_t>(raw) + 127) & ~(uintptr_t)127);
    uint8_t* const ring = reinterpret_cast<uint8_t*>(&s) + kRecSmem<kMaps>;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int strip = blockIdx.x % a.strips, index = blockIdx.x / a.strips, seg = kMaps ? index / a.parts : index;
    // its rows in scan order, the first pass's from the segment's last part on
    const int64_t row0 = (int64_t)seg * a.rows + (kMaps ? (int64_t)(index % a.parts) * a.part_rows : 0);
    const int rows = (int)(min(kMaps ? min(row0 + a.part_rows, (int64_t)(seg + 1) * a.rows) : row0 + a.rows, (int64_t)a.T) - row0);
    const int tiles = kMaps ? max((rows + kTile - 1) / kTile, 0) : max((rows + kTile - 1) / kTile, 1);       // one at least, for sequences without rows
    auto tile_row = [&](int i) { return (int)row0 + (kMaps ? tiles - 1 - i : i) * kTile; };
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) mbar_init(&s.full[i], 1);
        s.failed[0] = s.failed[1] = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_wait();
    pdl_trigger();
    int copied = 0;                                              // thread 0: tiles whose copies are under way or done
    auto copy_next = [&]() {
        if constexpr (kTma) {
            if (copied >= tiles) return;
            const int u0 = tile_row(copied), c = strip * kCols, st = copied % kStages;
            const int t = kBack ? a.T - u0 - kTile : u0;         // a first row below 0 reads zeros
            uint8_t* to = ring + st * kStageBytes<kBack, kMaps>;
            mbar_expect_tx(&s.full[st], kInput * kInputs);
            tma_load_2d(to + kG * kInput, &tm_g, c, t, &s.full[st]);
            tma_load_2d(to + kIn * kInput, kBack ? &tm_dy : &tm_x, c, t, &s.full[st]);
            if constexpr (kInputs == 4) {
                tma_load_2d(to + kX * kInput, &tm_x, c, t, &s.full[st]);
                tma_load_2d(to + kY * kInput, &tm_y, c, t - 1, &s.full[st]);
            }
            ++copied;
        }
    };
    __syncthreads();
    if (threadIdx.x == 0)
        for (int i = 0; i < kStages; ++i) copy_next();

    const int c = strip * kCols + lane * 2, n = min(max(a.D - c, 0), 2);
    Map behind = identity();                                     // kMaps, warp 0: of the tiles so far
    float2 start = both(0.f);                                    // else: the state in front of the tile
    bool failed = false;
    if (!kMaps && seg > 0) {
        const int all = seg * a.parts, per = (all + kWarps - 1) / kWarps, k0 = warp * per, k1 = min(k0 + per, all);
        const Map* p = a.maps + (size_t)strip * 32 + lane;
        Map run = identity();
        bool missing = false;                                    // a CTA of the first pass gave up
        for (int k = k0; k < k1; k += 8) {
            Map v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < k1) v[i] = p[(size_t)(k + i) * a.strips * 32];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < k1) {
                    missing = missing || unformed(v[i].A.x);
                    run = compose<true>(run, v[i]);
                }
        }
        if (no_number(run.B)) {
            run = identity();
            for (int k = k0; k < k1; ++k) run = compose<true, true>(run, p[(size_t)k * a.strips * 32]);
        }
        s.front[warp][lane] = run;
        failed = __syncthreads_or(missing) != 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) start = apply<true>(s.front[w][lane], start);
        if (no_number(start)) {
            start = both(0.f);
            for (int w = 0; w < kWarps; ++w) start = apply<true, true>(s.front[w][lane], start);
        }
    }

    const bool plain_strip = (strip + 1) * kCols <= a.D && a.pairs;
    int from = 0, to = 0;                                        // a sequence that the warp has met
    int stage = 0;
    uint32_t phase = 0;
    for (int i = 0; i < tiles && !failed; ++i) {
        const int u0 = tile_row(i) + warp * kRows;        // first row of the warp, in scan order
        auto row = [&](int r) { return kBack ? a.T - 1 - (u0 + r) : u0 + r; };
        // rows inside one sequence, nearly all there are: none needs a look of its own.  Otherwise: which are in a sequence, and which are the
        // first and last one in scan order
        const int low = kBack ? a.T - u0 - kRows : u0;
        bool plain = low > from && low + kRows < to && plain_strip;
        int seq = 0;
        uint32_t member = 0, first = 0, final = 0;
        if (!plain) {
            int b = a.T, e = a.T;
            bool m = false, f = false, l = false;
            const int q0 = sequence_of(a, max(low, 0));
            if (lane < kRows && u0 + lane < a.T) {
                const int t = row(lane);
                seq = sequence_from(a, q0, t);
                if (seq < a.seqs) {
                    b = begin_of(a, seq);
                    e = begin_of(a, seq + 1);
                }
                m = t >= b && t < e;
                f = m && t == b;
                l = m && t == e - 1;
            }
            member = __ballot_sync(0xffffffffu, m);
            first = __ballot_sync(0xffffffffu, kBack ? l : f);
            final = __ballot_sync(0xffffffffu, kBack ? f : l);
            constexpr int kNext = kMaps ? 0 : kRows - 1;         // towards the next tile
            from = __shfl_sync(0xffffffffu, b, kNext);
            to = __shfl_sync(0xffffffffu, e, kNext);
            plain = low > from && low + kRows < to && plain_strip;
        }
        // two columns of the r-th row of an input; not for rows of no sequence
        auto fetch = [&](int which, int r) {
            if constexpr (kTma) {
                const int at = kBack ? kTile - 1 - (warp * kRows + r) : warp * kRows + r;
                return pair_of(reinterpret_cast<const T*>(ring + stage * kStageBytes<kBack, kMaps> + which * kInput) + at * kCols + lane * 2);
            } else {
                const void* p = which == kG ? a.g : which == kIn ? (kBack ? a.dy : a.x) : which == kX ? a.x : a.y;
                const size_t ld = which == kG ? a.ld_g : which == kIn ? (kBack ? a.ld_dy : a.ld_x) : which == kX ? a.ld_x : a.ld_y;
                return load2(static_cast<const T*>(p) + (size_t)(row(r) - (which == kY)) * ld + c, n, a.pairs != 0);
            }
        };
        auto given = [&](const float* p, int r) {                // two columns of the r-th row's sequence in a state
            const int q = __shfl_sync(0xffffffffu, seq, r);
            const float* f = p + (size_t)q * a.D + c;
            return make_float2(n > 0 ? f[0] : 0.f, n > 1 ? f[1] : 0.f);
        };
        if (kTma && !mbar_wait(&s.full[stage], phase)) s.failed[i & 1] = 1;

        // ---- 1
        float2 keep[kRows], feed[kRows];                         // a; forward b, backward 1 - a
        Map m = identity();
        auto collect = [&](auto all) {
            constexpr bool kAll = decltype(all)::value;
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const bool in = kAll || (member >> r & 1) != 0, begins = !kAll && (first >> r & 1) != 0;
                float2 gv = both(0.f), v = both(0.f), z;
                if (in) {
                    gv = fetch(kG, r);
                    v = fetch(kIn, r);
                }
                gate_of(gv, keep[r], z, T());
                if (!in) keep[r] = both(1.f);
                if (begins) {
                    m.A = both(-0.f);
                    m.B = a.before ? given(a.before, r) : both(0.f);
                }
                if (kBack) {
                    feed[r] = z;
                    m.B = mul2(keep[r], add2(m.B, v));
                } else {
                    feed[r] = !in ? both(0.f) : kKind == ABS_RECURRENCE_BLEND ? mul2(v, z) : v;
                    m.B = fma2(keep[r], m.B, feed[r]);
                    if (begins) feed[r] = m.B;                   // the sequence's first state
                }
                m.A = mul2(m.A, keep[r]);
            }
        };
        if (plain) collect(std::true_type());
        else collect(std::false_type());
        s.map[i & 1][warp][lane] = m;
        const bool any_begins = __syncthreads_or(first != 0) != 0;     // a sequence begins in the tile
        // by the tile's parity: who is a tile ahead writes the other one, and nobody is two ahead
        failed = s.failed[i & 1] != 0;
        if (failed) break;
        // forward the tile's image has been read, backward that of the tile before
        if (threadIdx.x == 0 && (!kBack || kMaps || i > 0)) copy_next();
        // ---- 2
        const Map* of = &s.map[i & 1][0][lane];                  // of warp w: of[32 w]
        if constexpr (kMaps) {
            if (warp == 0) {
                Map whole = of[0];
                if (any_begins) {
#pragma unroll
                    for (int w = 1; w < kWarps; ++w) whole = compose<true>(whole, of[32 * w]);
                } else {
#pragma unroll
                    for (int w = 1; w < kWarps; ++w) whole = compose<false>(whole, of[32 * w]);
                }
                const Map last = behind;
                behind = compose<false>(whole, last);            // nothing begins in the tiles behind
                if (no_number(behind.B)) {
                    whole = of[0];
                    for (int w = 1; w < kWarps; ++w) whole = compose<true, true>(whole, of[32 * w]);
                    behind = compose<false, true>(whole, last);
                }
            }
            if (any_begins) break;
        } else {
            const float2 front = start;
            float2 state = front;
            if (any_begins) {
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    if (w == warp) state = start;
                    start = apply<true>(of[32 * w], start);
                }
            } else {
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    if (w == warp) state = start;
                    start = apply<false>(of[32 * w], start);
                }
            }
            if (no_number(state)) {
                state = front;
                for (int w = 0; w < warp; ++w) state = apply<true, true>(of[32 * w], state);
            }
            // ---- 3
            auto finish = [&](auto all) {
                constexpr bool kAll = decltype(all)::value;
                T* out = static_cast<T*>(a.out) + (int64_t)row(0) * (int64_t)a.ld_out + c;
                T* out2 = kBack ? static_cast<T*>(a.out2) + (int64_t)row(0) * (int64_t)a.ld_out2 + c : nullptr;
                const int64_t step = kBack ? -(int64_t)a.ld_out : (int64_t)a.ld_out, step2 = -(int64_t)a.ld_out2;
#pragma unroll
                for (int r = 0; r < kRows; ++r) {
                    const bool in = kAll || (member >> r & 1) != 0, begins = !kAll && (first >> r & 1) != 0, ends = !kAll && (final >> r & 1) != 0;
                    float2 o = both(0.f), o2 = both(0.f);
                    if (kBack) {
                        if (begins) state = a.before ? given(a.before, r) : both(0.f);
                        if (in) {
                            float2 h = both(0.f);
                            if (!ends) h = fetch(kY, r);
                            else if (a.h0) h = given(a.h0, r);
                            const float2 d = add2(state, fetch(kIn, r)), z = feed[r];
                            state = mul2(keep[r], d);
                            o = kKind == ABS_RECURRENCE_BLEND ? mul2(z, d) : d;
                            if (kKind == ABS_RECURRENCE_BLEND) h = fma2(fetch(kX, r), both(-1.f), h);
                            o2 = mul2(mul2(state, z), h);
                        }
                    } else {
                        state = begins ? feed[r] : fma2(keep[r], state, feed[r]);
                        if (in) o = state;
                    }
                    if (kAll) {
                        put_pair(out, o);
                        if (kBack) put_pair(out2, o2);
                    } else if (n > 0 && u0 + r < a.T) {
                        store2(out, n, a.pairs != 0, o);
                        if (kBack) store2(out2, n, a.pairs != 0, o2);
                    }
                    out += step;
                    if (kBack) out2 += step2;
                    if (ends && a.after) {
                        const int q = __shfl_sync(0xffffffffu, seq, r);
                        float* p = a.after + (size_t)q * a.D + c;
                        if (n > 0) p[0] = state.x;
                        if (n > 1) p[1] = state.y;
                    }
                }
            };
            if (plain) finish(std::true_type());
            else finish(std::false_type());
            if (no_number(start)) {
                start = front;
                for (int w = 0; w < kWarps; ++w) start = apply<true, true>(of[32 * w], start);
            }
        }
        if (++stage == kStages) {
            stage = 0;
            phase ^= 1u;
        }
    }
    if constexpr (kMaps) {
        if (failed) behind.A = both(__uint_as_float(kUnformed));
        if (warp == 0) a.maps[((size_t)index * a.strips + strip) * 32 + lane] = behind;
    } else if (seg == 0 && a.after && (a.T == 0 || a.offsets)) { // sequences without rows
        for (int q = warp; q < a.seqs; q += kWarps)
            if (begin_of(a, q + 1) <= begin_of(a, q))
                for (int k = 0; k < n; ++k) a.after[(size_t)q * a.D + c + k] = a.before ? a.before[(size_t)q * a.D + c + k] : 0.f;
    }
    if (threadIdx.x == 0) {
        if (failed) report_timeout();
        for (int i = max(copied - kStages, 0); i < copied; ++i)  // copies in flight land before the CTA's shared memory is released
            mbar_wait(&s.full[i % kStages], (i / kStages) & 1u, failed ? 4096u : kSpinLimit);
    }
}

template <typename T, uint32_t kKind>
__global__ void __launch_bounds__(256) k_recurrence_step(const T* x, size_t ld_x, const T* g, size_t ld_g, const float* h, size_t rows, int D, T* y, size_t ld_y,
                                                         float* out) {
    pdl_wait();
    pdl_trigger();
    for (size_t t = blockIdx.y; t < rows; t += gridDim.y) {
        const int c = blockIdx.x * 256 + threadIdx.x;
        if (c >= D) return;
        float2 a, z;
        gate_of(both(to_f(g[t * ld_g + c])), a, z, T());
        const float v = to_f(x[t * ld_x + c]), s = fmaf(a.x, h[t * D + c], kKind == ABS_RECURRENCE_BLEND ? z.x * v : v);
        out[t * D + c] = s;
        y[t * ld_y + c] = from_f<T>(s);
    }
}

// An input's tiles: kTile rows of 64 columns, as they lie.
bool encode_tiles(CUtensorMap* tm, const void* p, size_t ld, size_t es, const RecArgs& a, int rows) {
    const EncodeTiledFn enc = get_encode();
    if (!enc) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)a.D, (cuuint64_t)a.T}, strides[1] = {ld * es};
    const cuuint32_t box[2] = {kCols, (cuuint32_t)rows}, one[2] = {1, 1};
    return enc(tm, es == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims, strides, box, one,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Segments of a strip: as many as fill the GPU once, or twice where that leaves fewer SMs idle.  One where that fills more than 60 % of
// it, since two and more are read twice (but for what lies in front of a sequence's begin).  In the first pass, which fills the GPU with the segments
// but one, a segment is cut again where that leaves room.
template <typename T, bool kBack>
void cut_segments(RecArgs& a) {
    constexpr int kTile = kTileOf<T, kBack, false>, kMapTile = kTileOf<T, kBack, true>, kResident = kSms * kCtasOf<kBack, false>;
    const int tiles = std::max(1, (a.T + kTile - 1) / kTile);
    int segs = 1;
    if (a.strips * 10 <= kResident * 6) {
        const int once = kResident / a.strips, twice = 2 * kResident / a.strips;
        segs = twice > 2 * once && once < 8 ? twice : once;
    }
    const int per = (tiles + segs - 1) / segs;
    a.segs = (tiles + per - 1) / per;
    a.rows = per * kTile;
    const int map_tiles = per * (kTile / kMapTile);
    a.parts = a.segs > 1 ? std::max(1, std::min(kSms * kCtasOf<kBack, true> / ((a.segs - 1) * a.strips), map_tiles)) : 1;
    a.part_rows = (map_tiles + a.parts - 1) / a.parts * kMapTile;
}

template <typename T, uint32_t kKind, bool kBack, bool kTma, bool kMaps>
cudaError_t run_pass(const RecArgs& a, cudaStream_t s) {
    constexpr int kTile = kTileOf<T, kBack, kMaps>;
    CUtensorMap g{}, x{}, dy{}, y{};
    if (kTma) {
        bool ok = encode_tiles(&g, a.g, a.ld_g, sizeof(T), a, kTile);
        if (!kBack || !kMaps) ok = ok && encode_tiles(&x, a.x, a.ld_x, sizeof(T), a, kTile);
        if (kBack) ok = ok && encode_tiles(&dy, a.dy, a.ld_dy, sizeof(T), a, kTile);
        if (kBack && !kMaps) ok = ok && encode_tiles(&y, a.y, a.ld_y, sizeof(T), a, kTile);
        if (!ok) return cudaErrorInvalidValue;
    }
    const cudaError_t e = allow_smem<k_recurrence<T, kKind, kBack, kTma, kMaps>>();
    if (e != cudaSuccess) return e;
    return launch_kernel(k_recurrence<T, kKind, kBack, kTma, kMaps>, (kMaps ? (a.segs - 1) * a.parts : a.segs) * a.strips, kWarps * 32,
                         smem_bytes<kBack, kMaps>(kTma), s, true, a, g, x, dy, y);
}
template <typename T, uint32_t kKind, bool kBack, bool kTma>
cudaError_t run_passes(const RecArgs& a, cudaStream_t s) {
    const cudaError_t e = a.segs > 1 ? run_pass<T, kKind, kBack, kTma, true>(a, s) : cudaSuccess;
    return e != cudaSuccess ? e : run_pass<T, kKind, kBack, kTma, false>(a, s);
}
template <typename T, uint32_t kKind, bool kBack>
cudaError_t run_tiles(RecArgs a, bool tma, char* workspace, cudaStream_t s) {
    a.strips = (a.D + kCols - 1) / kCols;
    cut_segments<T, kBack>(a);
    a.maps = reinterpret_cast<Map*>(workspace);
    return tma ? run_passes<T, kKind, kBack, true>(a, s) : run_passes<T, kKind, kBack, false>(a, s);
}
template <typename T, uint32_t kKind>
cudaError_t run_kind(const RecArgs& a, bool back, bool tma, char* ws, cudaStream_t s) {
    return back ? run_tiles<T, kKind, true>(a, tma, ws, s) : run_tiles<T, kKind, false>(a, tma, ws, s);
}
template <typename T>
cudaError_t run(const RecArgs& a, uint32_t kind, bool back, bool tma, char* ws, cudaStream_t s) {
    return kind == ABS_RECURRENCE_BLEND ? run_kind<T, ABS_RECURRENCE_BLEND>(a, back, tma, ws, s) : run_kind<T, ABS_RECURRENCE_ADD>(a, back, tma, ws, s);
}

const char* check_sizes(uint64_t tokens, uint64_t width, uint64_t seqs, uint32_t kind, uint32_t dtype, int* code) {
    *code = ABS_EINVAL;
    if (!known_dtype(dtype)) return "dtype must be ABS_F32 or ABS_BF16";
    if (kind > ABS_RECURRENCE_ADD) return "unknown kind of recurrence";
    if (width == 0) return "width must be at least 1";
    if (tokens <= kSizeMax && width <= kSizeMax && seqs <= kSizeMax && ((tokens + kTileMin - 1) / kTileMin) * ((width + kCols - 1) / kCols) <= kSizeMax)
        return nullptr;
    *code = ABS_ELIMIT;
    return "a size exceeds 2^31 - 1024, or there are too many tiles of 32 rows and 64 columns";
}

// `mats`: the inputs, then the outputs.
template <int N>
int launch_scan(RecArgs& a, const MatrixArg (&mats)[N], int inputs, uint32_t kind, uint32_t dtype, bool back, void* workspace, size_t workspace_bytes, cudaStream_t s) {
    bool pairs = true, tma = a.T > 0;
    for (int i = 0; i < N; ++i) {
        pairs = pairs && rows_at(mats[i], 2 * mats[i].es);
        if (i < inputs) tma = tma && rows_at(mats[i], 16);
    }
    a.pairs = pairs;
    const size_t need = abs_recurrence_workspace((uint64_t)a.T, (uint64_t)a.D);
    if (need) {
        if (!workspace || misaligned(workspace, 256)) return thread_error(ABS_EINVAL, "workspace must be non-NULL and 256-byte aligned");
        if (workspace_bytes < need) return thread_error(ABS_ENOMEM, "workspace too small");
    }
    char* ws = static_cast<char*>(workspace);
    const cudaError_t e = dtype == ABS_F32 ? run<float>(a, kind, back, tma, ws, s) : run<bf16>(a, kind, back, tma, ws, s);
    return e == cudaSuccess ? ABS_OK : thread_error(ABS_ECUDA, cudaGetErrorString(e));
}

}  // namespace

cudaError_t take_status_recurrence(int* status, cudaStream_t s) { return take_status(status, s); }

}  // namespace abs_sgd

using namespace abs_sgd;

extern "C" size_t abs_recurrence_workspace(uint64_t tokens, uint64_t width) {
    if (tokens > kSizeMax || width > kSizeMax) return 0;
    if (tokens <= (uint64_t)kTileMin) return 0;
    // maps of the segments' parts: at most twice as many as the CTAs that fill the GPU
    const uint64_t strips = (width + kCols - 1) / kCols, most = std::min<uint64_t>(2 * 4 * kSms, (tokens + kTileMin - 1) / kTileMin * strips);
    return up256((size_t)std::max(most, strips) * 32 * sizeof(Map));
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
    if (last && last == h0) return thread_error(ABS_EINVAL, "last must not be h0");
    if (tokens && (!x || !g || !y)) return thread_error(ABS_EINVAL, "x, g and y must not be NULL");
    if (tokens == 0 && (!last || seqs == 0)) return ABS_OK;
    RecArgs a{};
    a.x = x; a.ld_x = ld_x; a.g = g; a.ld_g = ld_g; a.out = y; a.ld_out = ld_y;
    a.offsets = offsets; a.before = h0; a.after = last; a.T = (int)tokens; a.D = (int)width; a.seqs = (int)seqs;
    return launch_scan(a, m, 2, kind, dtype, false, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
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
    if (dh0 && (dh0 == h0 || dh0 == dlast)) return thread_error(ABS_EINVAL, "dh0 must be neither h0 nor dlast");
    if (tokens == 0 && (!dh0 || seqs == 0)) return ABS_OK;
    RecArgs a{};
    a.x = x; a.ld_x = ld_x; a.g = g; a.ld_g = ld_g; a.dy = dy; a.ld_dy = ld_dy; a.y = y; a.ld_y = ld_y;
    a.out = dx; a.ld_out = ld_dx; a.out2 = dg; a.ld_out2 = ld_dg;
    a.offsets = offsets; a.h0 = h0; a.before = dlast; a.after = dh0; a.T = (int)tokens; a.D = (int)width; a.seqs = (int)seqs;
    return launch_scan(a, m, 4, kind, dtype, true, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
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
