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
#include "llm_host.h"
#include "llm_status.cuh"
#include "row_ops.cuh"
#include "tcgen05.cuh"

namespace abs_sgd {
namespace {

constexpr int kWarps = 8, kCols = 64;    // of a tile; a lane owns two columns
constexpr int kGroupMax = 32;
constexpr int kSms = 148;
constexpr uint64_t kSizeMax = 0x7ffffc00ull;
// Rows of a warp: 32 KB of inputs for a tile (two matrices forward, four backward).
template <typename T, bool kBack>
constexpr int kRowsOf = (kBack ? 8 : 16) * 2 / (int)sizeof(T);
template <typename T, bool kBack>
constexpr int kTileOf = kWarps * kRowsOf<T, kBack>;
template <bool kBack>
constexpr int kStagesOf = kBack ? 2 : 3;
template <bool kBack>
constexpr int kCtasOf = kBack ? 3 : 2;   // of an SM
constexpr int kTileMin = kTileOf<float, true>;
constexpr int kStageBytes = 32768;

struct RecArgs {
    const void *x, *g, *dy, *y;          // y: of the forward pass (backward only)
    size_t ld_x, ld_g, ld_dy, ld_y;
    void *out, *out2;                    // forward: y; backward: dx, dg
    size_t ld_out, ld_out2;
    const int32_t* offsets;
    const float *h0, *before;            // before: h0, backward dlast: the state in front of a sequence in scan order
    float* after;                        // last, backward dh0
    int T, D, seqs;
    int tiles, strips, group;
    int pairs;                           // a lane's two columns are aligned to two elements in every matrix
    uint32_t* ctl;                       // [0]: tickets; then a flag per (tile, strip)
    float4* maps;                        // [tile][strip][lane]: a tile's map (A, B) for two columns, or (-0, state) for the last of a group
};

// sigmoid(g) and 1 - sigmoid(g), each to its own precision.
__device__ __forceinline__ void gate_of(float2 g, float2& a, float2& rest, bf16) {
    float2 v = mul2(g, both(-1.4426950408889634f));
    v.x = v.x > 126.f ? 126.f : v.x;     // keeps a NaN
    v.y = v.y > 126.f ? 126.f : v.y;
    const float2 e = exp2_of(v), d = add2(e, both(1.f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a.x) : "f"(d.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(a.y) : "f"(d.y));
    rest = mul2(e, a);
}
__device__ __forceinline__ void gate_of(float2 g, float2& a, float2& rest, float) {
    const float2 e = make_float2(expf(g.x < -87.f ? 87.f : -g.x), expf(g.y < -87.f ? 87.f : -g.y));
    a = make_float2(1.f / (1.f + e.x), 1.f / (1.f + e.y));
    rest = mul2(e, a);
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
__device__ __forceinline__ void compose2(float4& m, float4 then) {
    compose(m.x, m.y, then.x, then.y);
    compose(m.z, m.w, then.z, then.w);
}
__device__ __forceinline__ float2 apply2(float4 m, float2 s) { return make_float2(apply(m.x, m.y, s.x), apply(m.z, m.w, s.y)); }

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
__device__ __forceinline__ int sequence_of(const RecArgs& a, int t) {
    int lo = 0, hi = a.seqs;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (begin_of(a, mid + 1) <= t) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

struct RecSmem {
    alignas(16) float4 map[2][kWarps][32];       // of a warp's rows, by the tile's parity
    float4 look[kWarps][32];                     // of the tiles in front, a run of them for each warp
    alignas(8) uint64_t full[3];
    int ticket[4];
    uint32_t copies[4];                          // into each stage so far
    int load_failed, look_failed;
};

constexpr size_t kRecSmem = (sizeof(RecSmem) + 127) / 128 * 128;

// A tile: kTileOf rows (in scan order: backward from the last one) of 64 columns.  A CTA takes tiles by ticket, tiles of all strips at the
// same rows before the next rows, so that whoever waits for a tile in front waits for one that a running CTA has.
//   1. a lane reads its rows of two columns, forms the gates, and the map of its warp's rows
//   2. the warps' maps give the tile's map, which is published; the state in front of the tile is that behind the last tile of the group
//      in front (published as such), followed by the maps of the group's tiles so far: always the same tiles in the same order, so
//      that equal inputs give equal bits whoever comes first
//   3. a lane goes over its rows again from their state
// kTma: the tiles that a CTA takes next are copied to shared memory meanwhile.  Otherwise (rows that are not 16-byte aligned) the lanes read memory.
template <typename T, uint32_t kKind, bool kBack, bool kTma>
__global__ void __launch_bounds__(kWarps * 32, kCtasOf<kBack>) k_recurrence(const __grid_constant__ RecArgs a, const __grid_constant__ CUtensorMap tm_g,
                                                                            const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_dy,
                                                                            const __grid_constant__ CUtensorMap tm_y) {
    constexpr int kRows = kRowsOf<T, kBack>, kTile = kTileOf<T, kBack>, kStages = kStagesOf<kBack>, kInputs = kBack ? 4 : 2;
    constexpr int kInput = kTile * kCols * (int)sizeof(T);       // bytes of an input's tile
    static_assert(kInput * kInputs == kStageBytes, "");
    enum { kG, kX, kDy, kY };
    extern __shared__ uint8_t raw[];
    RecSmem& s = *reinterpret_cast<RecSmem*>((reinterpret_cast<uintptr_t>(raw) + 127) & ~(uintptr_t)127);
    uint8_t* const ring = reinterpret_cast<uint8_t*>(&s) + kRecSmem;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int total = a.tiles * a.strips;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&s.full[i], 1);
            s.copies[i] = 0;
        }
        s.load_failed = s.look_failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_wait();
    pdl_trigger();
    // thread 0: the next tile, and its copies
    int coming = 0;                                              // thread 0: a ticket taken, not yet used
    auto take = [&]() { return a.ctl ? (int)atomicAdd(&a.ctl[0], 1u) : coming + (int)gridDim.x; };
    auto start = [&](int stage) {
        s.ticket[stage] = coming;
        if (coming >= total) return;
        if constexpr (kTma) {
            const int u0 = coming / a.strips * kTile, c = coming % a.strips * kCols;
            const int t = kBack ? a.T - u0 - kTile : u0;         // a first row below 0 reads zeros
            uint8_t* to = ring + stage * kStageBytes;
            mbar_expect_tx(&s.full[stage], kStageBytes);
            ++s.copies[stage];
            tma_load_2d(to + kG * kInput, &tm_g, c, t, &s.full[stage]);
            tma_load_2d(to + kX * kInput, &tm_x, c, t, &s.full[stage]);
            if constexpr (kBack) {
                tma_load_2d(to + kDy * kInput, &tm_dy, c, t, &s.full[stage]);
                tma_load_2d(to + kY * kInput, &tm_y, c, t - 1, &s.full[stage]);
            }
        }
        coming = take();
    };
    if (threadIdx.x == 0) {
        coming = a.ctl ? take() : (int)blockIdx.x;
        for (int i = 0; i < kStages; ++i) start(i);
    }
    __syncthreads();

    int stage = 0, n_tile = 0;
    uint32_t phase = 0;
    for (;;) {
        const int mine = s.ticket[stage];
        if (mine >= total) break;
        const int tile = mine / a.strips, strip = mine % a.strips;
        const int c = strip * kCols + lane * 2, n = min(max(a.D - c, 0), 2);
        const int u0 = tile * kTile + warp * kRows;              // first row of the warp, in scan order
        auto row = [&](int r) { return kBack ? a.T - 1 - (u0 + r) : u0 + r; };
        // ---- which rows are in a sequence, and are the first and last one in scan order
        int seq = 0;
        uint32_t member, first, final;
        {
            bool m = false, f = false, l = false;
            if (lane < kRows && u0 + lane < a.T) {
                const int t = row(lane);
                seq = sequence_of(a, t);
                const int from = seq < a.seqs ? begin_of(a, seq) : a.T;
                m = t >= from;
                f = m && t == from;
                l = m && t == begin_of(a, seq + 1) - 1;
            }
            member = __ballot_sync(0xffffffffu, m);
            first = __ballot_sync(0xffffffffu, kBack ? l : f);
            final = __ballot_sync(0xffffffffu, kBack ? f : l);
        }
        // two columns of the r-th row of an input; not for rows of no sequence
        auto fetch = [&](int which, int r) {
            if constexpr (kTma) {
                const int at = kBack ? kTile - 1 - (warp * kRows + r) : warp * kRows + r;
                return pair_of(reinterpret_cast<const T*>(ring + stage * kStageBytes + which * kInput) + at * kCols + lane * 2);
            } else {
                const void* p = which == kG ? a.g : which == kX ? a.x : which == kDy ? a.dy : a.y;
                const size_t ld = which == kG ? a.ld_g : which == kX ? a.ld_x : which == kDy ? a.ld_dy : a.ld_y;
                return load2(static_cast<const T*>(p) + (size_t)(row(r) - (which == kY)) * ld + c, n, a.pairs != 0);
            }
        };
        auto given = [&](const float* p, int r) {                // two columns of the r-th row's sequence in a state
            const int q = __shfl_sync(0xffffffffu, seq, r);
            const float* f = p + (size_t)q * a.D + c;
            return make_float2(n > 0 ? f[0] : 0.f, n > 1 ? f[1] : 0.f);
        };
        if (kTma && !mbar_wait(&s.full[stage], phase)) s.load_failed = 1;

        // ---- 1
        float2 keep[kRows], feed[kRows];                         // a; forward b, backward 1 - a
        float4 m = make_float4(1.f, 0.f, 1.f, 0.f);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const bool in = (member >> r & 1) != 0;
            float2 gv = both(0.f), v = both(0.f), z;             // v: x, backward dy
            if (in) {
                gv = fetch(kG, r);
                v = fetch(kBack ? kDy : kX, r);
            }
            gate_of(gv, keep[r], z, T());
            if (!in) keep[r] = both(1.f);
            if (first >> r & 1) {
                m = make_float4(-0.f, 0.f, -0.f, 0.f);
                if (a.before) {                                  // read once and here: `after` may be `before`
                    const float2 i = given(a.before, r);
                    m.y = i.x;
                    m.w = i.y;
                }
            }
            float2 B = make_float2(m.y, m.w);
            if (kBack) {
                feed[r] = (first >> r & 1) ? B : z;              // a first row's 1 - a is formed again
                B = mul2(keep[r], add2(B, v));
            } else {
                feed[r] = !in ? both(0.f) : kKind == ABS_RECURRENCE_BLEND ? mul2(v, z) : v;
                if (first >> r & 1) feed[r] = fma2(keep[r], B, feed[r]);
                B = (first >> r & 1) ? feed[r] : fma2(keep[r], B, feed[r]);
            }
            m = make_float4(m.x * keep[r].x, B.x, m.z * keep[r].y, B.y);
        }
        s.map[n_tile & 1][warp][lane] = m;
        __syncthreads();
        if (s.load_failed) break;
        // forward the tile's image has been read, backward that of the tile before
        if (threadIdx.x == 0) {
            if (!kBack) start(stage);
            else if (n_tile > 0) start(stage ^ 1);
        }
        // ---- 2
        float2 state = both(0.f);
        if (a.tiles > 1) {
            uint32_t* flags = a.ctl + 1;
            const bool closes = tile % a.group == a.group - 1;
            float4 whole = make_float4(1.f, 0.f, 1.f, 0.f);
            auto publish = [&]() {
                a.maps[((size_t)tile * a.strips + strip) * 32 + lane] = whole;
                __threadfence();
                __syncwarp();
                if (lane == 0) asm volatile("st.release.gpu.global.u32 [%0], %1;" ::"l"(flags + (size_t)tile * a.strips + strip), "r"(1u) : "memory");
            };
            if (warp == 0) {
#pragma unroll
                for (int w = 0; w < kWarps; ++w) compose2(whole, s.map[n_tile & 1][w][lane]);
                if (!closes) publish();
            }
            const int from = max(tile / a.group * a.group - 1, 0), count = tile - from, per = (count + kWarps - 1) / kWarps;
            constexpr int kPer = (kGroupMax + kWarps - 1) / kWarps;
            const int k0 = from + warp * per, k1 = min(k0 + per, tile);
            bool ok = true;
            if (k0 + lane < k1) {
                const uint32_t* f = flags + (size_t)(k0 + lane) * a.strips + strip;
                uint32_t seen = 0;
                for (uint32_t it = 0; it < kSpinLimit && !seen; ++it) asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(f) : "memory");
                ok = seen != 0;
            }
            if (__all_sync(0xffffffffu, ok)) {
                float4 v[kPer], run = make_float4(1.f, 0.f, 1.f, 0.f);
#pragma unroll
                for (int k = 0; k < kPer; ++k)
                    if (k0 + k < k1) v[k] = __ldcg(a.maps + ((size_t)(k0 + k) * a.strips + strip) * 32 + lane);
#pragma unroll
                for (int k = 0; k < kPer; ++k)
                    if (k0 + k < k1) compose2(run, v[k]);
                s.look[warp][lane] = run;
            } else {
                s.look_failed = 1;
            }
            __syncthreads();
            if (s.look_failed) break;
#pragma unroll
            for (int w = 0; w < kWarps; ++w)
                if (w * per < count) state = apply2(s.look[w][lane], state);
            if (closes && warp == 0) {
                const float2 end = apply2(whole, state);
                whole = make_float4(-0.f, end.x, -0.f, end.y);
                publish();
            }
        }
        if (kBack && a.tiles == 1) __syncthreads();              // the next tile's ticket
        for (int w = 0; w < warp; ++w) state = apply2(s.map[n_tile & 1][w][lane], state);
        // ---- 3
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const bool in = (member >> r & 1) != 0;
            float2 o = both(0.f), o2 = both(0.f);
            if (kBack) {
                if (first >> r & 1) {
                    float2 k;
                    state = feed[r];
                    gate_of(fetch(kG, r), k, feed[r], T());
                }
                if (in) {
                    float2 h = both(0.f);
                    if (!(final >> r & 1)) h = fetch(kY, r);
                    if ((final >> r & 1) && a.h0) h = given(a.h0, r);
                    const float2 d = add2(state, fetch(kDy, r)), z = feed[r];
                    state = mul2(keep[r], d);
                    o = kKind == ABS_RECURRENCE_BLEND ? mul2(z, d) : d;
                    if (kKind == ABS_RECURRENCE_BLEND) h = fma2(fetch(kX, r), both(-1.f), h);
                    o2 = mul2(mul2(state, z), h);
                }
            } else {
                state = (first >> r & 1) ? feed[r] : fma2(keep[r], state, feed[r]);
                if (in) o = state;
            }
            if (n > 0 && u0 + r < a.T) {
                const size_t t = (size_t)row(r);
                store2(static_cast<T*>(a.out) + t * a.ld_out + c, n, a.pairs != 0, o);
                if (kBack) store2(static_cast<T*>(a.out2) + t * a.ld_out2 + c, n, a.pairs != 0, o2);
            }
            if ((final >> r & 1) && a.after) {
                const int q = __shfl_sync(0xffffffffu, seq, r);
                float* p = a.after + (size_t)q * a.D + c;
                if (n > 0) p[0] = state.x;
                if (n > 1) p[1] = state.y;
            }
        }
        // ---- sequences without rows
        if (tile == 0 && a.after && (a.T == 0 || a.offsets))
            for (int q = warp; q < a.seqs; q += kWarps)
                if (begin_of(a, q + 1) <= begin_of(a, q))
                    for (int i = 0; i < n; ++i) a.after[(size_t)q * a.D + c + i] = a.before ? a.before[(size_t)q * a.D + c + i] : 0.f;
        ++n_tile;
        if (++stage == kStages) {
            stage = 0;
            phase ^= 1u;
        }
    }
    if (threadIdx.x == 0 && (s.load_failed || s.look_failed)) {
        report_timeout();
        for (int i = 0; i < kStages; ++i)                        // copies in flight land before the CTA's shared memory is released
            if (s.copies[i]) mbar_wait(&s.full[i], (s.copies[i] - 1) & 1u, 4096u);
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

size_t flags_bytes(uint64_t tiles, uint64_t strips) { return up256((1 + tiles * strips) * 4); }

// An input's tiles: kTile rows of 64 columns, as they lie.
bool encode_tiles(CUtensorMap* tm, const void* p, size_t ld, size_t es, const RecArgs& a, int rows) {
    const EncodeTiledFn enc = get_encode();
    if (!enc) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)a.D, (cuuint64_t)a.T}, strides[1] = {ld * es};
    const cuuint32_t box[2] = {kCols, (cuuint32_t)rows}, one[2] = {1, 1};
    return enc(tm, es == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims, strides, box, one,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, uint32_t kKind, bool kBack>
cudaError_t run_tiles(RecArgs a, bool tma, char* workspace, cudaStream_t s) {
    constexpr int kTile = kTileOf<T, kBack>;
    a.tiles = std::max(1, (a.T + kTile - 1) / kTile);
    a.strips = (a.D + kCols - 1) / kCols;
    // the chain of published states takes some 2.5 us a link: a group's tiles of all strips have to keep the memory busy for that long
    a.group = std::min(std::max(331 / a.strips, 1), kGroupMax);
    if (a.tiles > 1) {
        const size_t flags = flags_bytes(a.tiles, a.strips);
        a.ctl = reinterpret_cast<uint32_t*>(workspace);
        a.maps = reinterpret_cast<float4*>(workspace + flags);
        const cudaError_t e = cudaMemsetAsync(workspace, 0, flags, s);
        if (e != cudaSuccess) return e;
    }
    const int grid = std::min(a.tiles * a.strips, kSms * kCtasOf<kBack>);
    CUtensorMap g{}, x{}, dy{}, y{};
    if (!tma) return launch_kernel(k_recurrence<T, kKind, kBack, false>, grid, kWarps * 32, kRecSmem + 128, s, a.tiles == 1, a, g, x, dy, y);
    bool ok = encode_tiles(&g, a.g, a.ld_g, sizeof(T), a, kTile) && encode_tiles(&x, a.x, a.ld_x, sizeof(T), a, kTile);
    if (kBack) ok = ok && encode_tiles(&dy, a.dy, a.ld_dy, sizeof(T), a, kTile) && encode_tiles(&y, a.y, a.ld_y, sizeof(T), a, kTile);
    if (!ok) return cudaErrorInvalidValue;
    const cudaError_t e = allow_smem<k_recurrence<T, kKind, kBack, true>>();
    if (e != cudaSuccess) return e;
    return launch_kernel(k_recurrence<T, kKind, kBack, true>, grid, kWarps * 32, kRecSmem + kStagesOf<kBack> * kStageBytes + 128, s, a.tiles == 1, a, g, x, dy, y);
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
    const uint64_t tiles = (tokens + kTileMin - 1) / kTileMin, strips = (width + kCols - 1) / kCols;
    return tiles > 1 ? flags_bytes(tiles, strips) + tiles * strips * 32 * sizeof(float4) : 0;
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
    if (dh0 && dh0 == h0) return thread_error(ABS_EINVAL, "dh0 must not be h0");
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
