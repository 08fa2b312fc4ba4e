// Layer norm and the residual tail on feature maps (inner > 1): a tile of neighbouring positions with all their features in
// shared memory, so that every array passes once.
//
// A tile is 32 pieces of VP positions (SPREAD: 32 VP positions of one slice, of which lane l has l, l + 32, ...: for slices that
// begin anywhere, element by element); lane l of every warp has piece l, and each warp ITEMS neighbouring features of it.  What a
// thread will work on it copies into shared memory itself (no barrier); the warps exchange sums for each position, which the
// first threads of the block add up, one position each.  A VJP keeps the sums of its features' weights in registers over all of its
// block's tiles and adds them across lanes at the end; weight_grads (prior_norm.cuh) adds up the blocks.
//
// Bound by memory without a mask, as far as the bytes under way reach: a tile waits for its pieces, then for the block's sums twice.
// 20 maps of 60 x 30720 in float32, forward and VJP: 56 + 80 us (5.3 and 5.6 TB/s).  With a mask its products and the rest of
// the arithmetic share the time with the bytes: residual tail of four slices of 100 x 235520 in bf16 203 + 256 us (about 45
// instructions an element; the bytes take 115 + 144, the words alone 54 in each), of 20 maps of 50 x 30720 in float32 84 + 117
// us (75 + 94).  Loops over a warp's features stay rolled where the mask is drawn: unrolled, their code left the instruction
// cache (the bf16 tail 555 us).  Requesting each next piece as its place is used, in place of after the tile, was slower
// (195 + 266 us), and so were one tile an SM with pieces of 16 bytes (246 + 278) and, in the VJP, eight features a thread with 72
// registers (257; the float32 tail 128).
#pragma once
#include "prior_rows.cuh"

namespace gleam {
namespace prior {

// VP positions of one feature as they lie in memory, and the pairs of numbers that they become (one position: half a pair).
template <class T, int VP> struct alignas(VP * sizeof(T)) Piece { T e[VP]; };
template <int VP> constexpr int PAIRS = (VP + 1) / 2;

template <class T, int VP>
__device__ __forceinline__ void unpack(const Piece<T, VP>& p, Two (&v)[PAIRS<VP>]) {
    if constexpr (VP == 1) v[0] = Two(to_float(p.e[0]), 0.f);
    else {
#pragma unroll
        for (int j = 0; j < VP / 2; ++j) {
            if constexpr (std::is_same<T, __nv_bfloat16>::value) {
                const uint32_t w = reinterpret_cast<const uint32_t*>(&p)[j];
                v[j] = Two(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
            } else if constexpr (std::is_same<T, __half>::value) {
                const float2 f = __half22float2(reinterpret_cast<const __half2*>(&p)[j]);
                v[j] = Two(f.x, f.y);
            } else {
                v[j] = Two(p.e[2 * j], p.e[2 * j + 1]);
            }
        }
    }
}
template <class T, int VP>
__device__ __forceinline__ Piece<T, VP> piece_of(const Two (&v)[PAIRS<VP>]) {
    Piece<T, VP> p;
    if constexpr (VP == 1) p.e[0] = from_float<T>(v[0].lo());
    else {
#pragma unroll
        for (int j = 0; j < VP / 2; ++j) {
            if constexpr (std::is_same<T, __nv_bfloat16>::value) reinterpret_cast<__nv_bfloat162*>(&p)[j] = __floats2bfloat162_rn(v[j].lo(), v[j].hi());
            else if constexpr (std::is_same<T, __half>::value) reinterpret_cast<__half2*>(&p)[j] = __floats2half2_rn(v[j].lo(), v[j].hi());
            else { p.e[2 * j] = v[j].lo(); p.e[2 * j + 1] = v[j].hi(); }
        }
    }
    return p;
}
// Where the elements of a piece stand in the mask: by counter where a piece begins one (VP >= 4, inner a multiple of four), else
// by element.
template <int VP, bool SPREAD>
struct MaskPlace {
    static constexpr bool BY_COUNTER = VP >= 4 && !SPREAD;
    uint64_t at;
    __device__ __forceinline__ MaskPlace(const Args& a, uint64_t element) : at(BY_COUNTER ? (element >> 2) + a.offset : element) {}
    __device__ __forceinline__ void next(const Args& a) { at += BY_COUNTER ? a.inner >> 2 : a.inner; }
};
// v = r + s v [s v] for the kept elements of a piece, r [0] for the others.
template <bool RES, int VP>
__device__ __forceinline__ void drop_piece(const Mask& mask, const MaskPlace<VP, false>& place, Two (&v)[PAIRS<VP>], const Two (&r)[PAIRS<VP>]) {
    if constexpr (VP >= 4) mask.apply<RES, true>(place.at, v, r);
    else {
        const uint4 w = mask.words(mask.counter(place.at >> 2));
        const int at = (int)(place.at & 3u);
        const Two kept = RES ? fma2(v[0], Two(mask.a.scale), r[0]) : v[0] * Two(mask.a.scale), gone = RES ? r[0] : Two(0.f);
        v[0] = Two(mask.dropped(w, at) ? gone.lo() : kept.lo(), VP == 2 && mask.dropped(w, at + 1) ? gone.hi() : kept.hi());
    }
}

// The same for a tile that is spread: the positions of a feature in it are 128 neighbours from element `first` on, so its 32 lanes
// draw a counter each and one more where the first one is shared, and find their elements' bits by ballots.  All lanes call.
template <bool RES>
__device__ __forceinline__ void drop_spread(const Mask& mask, uint64_t first, int lane, Two (&v)[2], const Two (&r)[2]) {
    const int shift = (int)(first & 3u);
    const uint64_t counter = mask.counter(first >> 2);
    const uint4 w = mask.words(counter + (uint32_t)lane);
    const uint32_t b0 = __ballot_sync(0xffffffffu, mask.dropped(w, 0)), b1 = __ballot_sync(0xffffffffu, mask.dropped(w, 1));
    const uint32_t b2 = __ballot_sync(0xffffffffu, mask.dropped(w, 2)), b3 = __ballot_sync(0xffffffffu, mask.dropped(w, 3));
    const int which = (lane + shift) & 3, from = (lane + shift) >> 2;
    const uint32_t mine = which == 0 ? b0 : which == 1 ? b1 : which == 2 ? b2 : b3;
    bool beyond = false;
    if (shift) beyond = mask.dropped(mask.words(counter + 32), which);
    auto gone = [&](int m) { return from + 8 * m < 32 ? (mine >> (from + 8 * m)) & 1u : (uint32_t)beyond; };
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const Two kept = RES ? fma2(v[i], Two(mask.a.scale), r[i]) : v[i] * Two(mask.a.scale), none = RES ? r[i] : Two(0.f);
        v[i] = Two(gone(2 * i) ? none.lo() : kept.lo(), gone(2 * i + 1) ? none.hi() : kept.hi());
    }
}

// Warps of a block, and features of a warp and of a map, at most.  20 warps of 32 features in place of 16 of 40: the registers that
// they have less cost maps of 257 to 512 features 17 % (4 x 500 x 16384 in float32, VJP: 123 and 145 us).
constexpr int MAP_TILE_WARPS = 16, MAP_ITEMS = 40, MAP_FEATURES = MAP_ITEMS * MAP_TILE_WARPS;

// A block's view of its tiles.
template <class T, int VP, int ITEMS, int ARRAYS, bool SPREAD>
struct MapTile {
    using P = Piece<T, VP>;
    P* slots;                            // this thread's pieces, a warp's width apart: the warps' shares lie one behind another
    uint32_t address;
    int lane, warp, first, items;        // first feature and number of features of the warp
    int live;                            // positions that this lane has: VP or none (SPREAD: any number)
    long long tiles, o, k;               // number of tiles; slice and position in it of this lane's piece (SPREAD: of its first one)
    __device__ __forceinline__ MapTile(const Args& a, void* shared) {
        lane = threadIdx.x & 31; warp = threadIdx.x >> 5;
        slots = static_cast<P*>(shared) + warp * (ARRAYS * ITEMS * 32) + lane;
        address = (uint32_t)__cvta_generic_to_shared(slots);
        first = warp * ITEMS;
        items = min(ITEMS, (int)a.features - first);
        tiles = SPREAD ? a.outer * row(a) : (a.outer * row(a) + 31) / 32;
        o = k = 0; live = 0;
    }
    // pieces (SPREAD: tiles) of a slice
    __device__ __forceinline__ long long row(const Args& a) const { return SPREAD ? (a.inner + 32 * VP - 1) / (32 * VP) : a.inner / VP; }
    __device__ __forceinline__ P& slot(int array, int j) const { return slots[(array * ITEMS + j) * 32]; }
    __device__ __forceinline__ void go(long long tile, const Args& a) {
        const long long p = SPREAD ? tile : tile * 32 + lane, n = row(a), all = a.outer * n;
        live = p < all ? VP : 0;
        o = !live ? 0 : all <= 0xffffffffll ? (uint32_t)p / (uint32_t)n : p / n;
        k = !live ? 0 : SPREAD ? (p - o * n) * (32 * VP) + lane : (p - o * n) * VP;
        if (SPREAD) live = (int)max(0ll, min((long long)VP, (a.inner - k + 31) / 32));
    }
    __device__ __forceinline__ const T* at(const void* array, long long pitch, const Args& a) const {
        return static_cast<const T*>(array) + (o * pitch + first * a.inner + k);
    }
    __device__ __forceinline__ T* at(void* array, long long pitch, const Args& a) const {
        return static_cast<T*>(array) + (o * pitch + first * a.inner + k);
    }
    // Whether all of the warp's features and positions are there: then nothing is checked.
    __device__ __forceinline__ bool full() const { return items == ITEMS && __all_sync(0xffffffffu, live == VP); }
    // Features that a lane passes over; in a spread tile the lanes of a warp stay together.
    template <bool FULL> __device__ __forceinline__ int count() const { return FULL ? ITEMS : SPREAD || live ? items : 0; }
    template <bool FULL>
    __device__ __forceinline__ void fetch(int array, const void* from, long long pitch, const Args& a) const {
        const T* p = at(from, pitch, a);
        if constexpr (SPREAD && sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < ITEMS; ++j, p += a.inner) {
                if (!FULL && j >= items) break;
#pragma unroll
                for (int m = 0; m < VP; ++m)
                    if (FULL || m < live) copy_small<4>(address + (array * ITEMS + j) * 32 * (uint32_t)sizeof(P) + 4 * m, p + 32 * m);
            }
        } else if constexpr (!SPREAD && sizeof(P) >= 4) {
#pragma unroll
            for (int j = 0; j < ITEMS; ++j, p += a.inner) {
                if (!FULL && !(live && j < items)) continue;
                const uint32_t to = address + (array * ITEMS + j) * 32 * (uint32_t)sizeof(P);
                if constexpr (sizeof(P) == 16) copy16(to, p);
                else copy_small<(int)sizeof(P)>(to, p);
            }
        } else {                                         // two bytes: too few for a copy
            constexpr int STEP = SPREAD ? 32 : 1;
            P v[ITEMS];
#pragma unroll
            for (int j = 0; j < ITEMS; ++j, p += a.inner)
#pragma unroll
                for (int m = 0; m < VP; ++m) v[j].e[m] = FULL || (m < live && j < items) ? p[STEP * m] : from_float<T>(0.f);
#pragma unroll
            for (int j = 0; j < ITEMS; ++j) slot(array, j) = v[j];
        }
    }
    template <bool FULL>
    __device__ __forceinline__ void store(T* p, const P& v) const {
        if constexpr (SPREAD) {
#pragma unroll
            for (int m = 0; m < VP; ++m) if (FULL || m < live) p[32 * m] = v.e[m];
        } else {
            *reinterpret_cast<P*>(p) = v;
        }
    }
    template <int BYTES> static __device__ __forceinline__ void copy_small(uint32_t to, const void* from) {
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(BYTES) : "memory");
    }
    // number of the first element of the warp's first feature (SPREAD: of lane 0)
    __device__ __forceinline__ uint64_t element(const Args& a) const { return (uint64_t)((o * a.features + first) * a.inner + k - (SPREAD ? lane : 0)); }
    // position of number m of this lane, in the arrays of statistics
    __device__ __forceinline__ long long position(int m, const Args& a) const { return o * a.inner + k + (SPREAD ? 32 * m : m); }
};

// Rounding can leave a sum of squares below zero; a NaN stays.
__device__ __forceinline__ float not_negative(float v) { return v < 0.f ? 0.f : v; }

// Two sums for each position of the tile, as (2, warps, 32 VP) floats; `mine` adds a position's up, of which `per_warp` gets
// every warp's pair; what it leaves in the first two rows is read back by all.
template <int VP, class F>
__device__ __forceinline__ void map_exchange(float* sums, int warps, int lane, int warp, const Two (&a)[PAIRS<VP>], const Two (&b)[PAIRS<VP>], Two (&ra)[PAIRS<VP>],
                                             Two (&rb)[PAIRS<VP>], F&& add_up) {
    constexpr int N = 32 * VP;
    auto put = [&](float* row, const Two (&v)[PAIRS<VP>]) {
        if constexpr (VP == 1) row[lane] = v[0].lo();
        else {
#pragma unroll
            for (int j = 0; j < VP / 2; ++j) *reinterpret_cast<unsigned long long*>(row + j * 64 + 2 * lane) = v[j].bits;
        }
    };
    auto get = [&](const float* row, Two (&v)[PAIRS<VP>]) {
        if constexpr (VP == 1) v[0] = Two(row[lane], 0.f);
        else {
#pragma unroll
            for (int j = 0; j < VP / 2; ++j) v[j].bits = *reinterpret_cast<const unsigned long long*>(row + j * 64 + 2 * lane);
        }
    };
    put(sums + warp * N, a);
    put(sums + (warps + warp) * N, b);
    __syncthreads();
    // position i of the exchange: pair j of the lanes, lane, half
    for (int i = threadIdx.x; i < N; i += blockDim.x) add_up(i, sums + i, sums + warps * N + i, sums + 2 * warps * N + i, N);
    __syncthreads();
    get(sums + 2 * warps * N, ra);
    get(sums + (2 * warps + 1) * N, rb);
}
// Floats of the exchange.
constexpr size_t map_exchange_floats(int vp, int warps) { return (size_t)(2 * warps + 2) * 32 * vp; }

template <class T, int VP, int ITEMS, bool TAIL, bool SPREAD>
__global__ void __launch_bounds__(MAP_TILE_WARPS * 32, ITEMS <= 16 ? 2 : 1) map_tile_forward(const __grid_constant__ Args a) {
    grid_dependency_wait();
    extern __shared__ __align__(16) float shared[];
    const int warps = blockDim.x >> 5, n = (int)a.features;
    float* sums = shared;
    float* wt = sums + map_exchange_floats(VP, warps);
    float* bs = wt + warps * ITEMS;
    MapTile<T, VP, ITEMS, TAIL ? 2 : 1, SPREAD> t(a, bs + warps * ITEMS);
    for (int c = threadIdx.x; c < warps * ITEMS; c += blockDim.x) {
        wt[c] = c >= n ? 0.f : a.weight ? weight_at<T>(a.weight, a.weight_f32, c) : 1.f;
        bs[c] = c < n && a.bias ? weight_at<T>(a.bias, a.weight_f32, c) : 0.f;
    }
    const Mask mask(a);
    const float count = (float)n, inv_count = 1.f / count, inv_here = 1.f / (float)t.items;
    const float last_features = (float)(n - (warps - 1) * ITEMS), inv_last = 1.f / last_features;
    bool full = false;
    auto fetch = [&](long long tile) {
        if (tile < t.tiles) {
            t.go(tile, a);
            full = t.full();
            if (full) {
                t.template fetch<true>(0, a.x, a.px, a);
                if (TAIL) t.template fetch<true>(1, a.res, a.pres, a);
            } else {
                t.template fetch<false>(0, a.x, a.px, a);
                if (TAIL) t.template fetch<false>(1, a.res, a.pres, a);
            }
        }
        copies_commit();
    };
    // the warp's features of every position: their sum and the squared deviations from their mean, in one pass.  The latter come
    // from sums relative to the first feature, q - s^2 / k of k numbers; as the first is one of them, the result is at least q / (k
    // + 1), so that the rounding of s^2 / k costs up to k + 1 times itself (k is at most 40) where that feature stands out, and a
    // far mean costs nothing.  Relative error of the variance, worst of 16384 positions: normal values 4e-7 (k = 8) to 7e-7 (40;
    // two passes, as on rows, 3e-7), every share's first feature thirty standard deviations away 1e-6 to 1e-5.
    auto statistics = [&](auto whole_tile, Two (&sum_of)[PAIRS<VP>], Two (&dev)[PAIRS<VP>]) {
        constexpr bool FULL = decltype(whole_tile)::value;
        Two pivot[PAIRS<VP>], s[PAIRS<VP>], q[PAIRS<VP>];
#pragma unroll
        for (int i = 0; i < PAIRS<VP>; ++i) pivot[i] = s[i] = q[i] = sum_of[i] = Two(0.f);
        T* sum = TAIL ? t.at(a.out2, a.pout2, a) : nullptr;
        MaskPlace<VP, SPREAD> place(a, TAIL ? t.element(a) : 0);
        auto value = [&](int j, Two (&v)[PAIRS<VP>]) {
            unpack<T, VP>(t.slot(0, j), v);
            if (!TAIL) return;
            Two r[PAIRS<VP>];
            unpack<T, VP>(t.slot(1, j), r);
            if (a.dropping) {
                if constexpr (SPREAD) drop_spread<true>(mask, place.at, t.lane, v, r);
                else drop_piece<true, VP>(mask, place, v, r);
            } else {
#pragma unroll
                for (int i = 0; i < PAIRS<VP>; ++i) v[i] = v[i] + r[i];
            }
            const Piece<T, VP> stored = piece_of<T, VP>(v);
            unpack<T, VP>(stored, v);
            t.slot(0, j) = stored;
            t.template store<FULL>(sum, stored);
            sum += a.inner; place.next(a);
        };
        const int features = t.template count<FULL>();
        if (FULL || features > 0) {
            value(0, pivot);
#pragma unroll
            for (int i = 0; i < PAIRS<VP>; ++i) { sum_of[i] = pivot[i]; pivot[i] = pivot[i] * Two(-1.f); }
            // two at a time: more of the mask's code than that does not stay in the instruction cache
#pragma unroll 2
            for (int j = 1; j < features; ++j) {
                Two v[PAIRS<VP>];
                value(j, v);
#pragma unroll
                for (int i = 0; i < PAIRS<VP>; ++i) {
                    const Two d = v[i] + pivot[i];
                    sum_of[i] = sum_of[i] + v[i]; s[i] = s[i] + d; q[i] = fma2(d, d, q[i]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < PAIRS<VP>; ++i) dev[i] = fma2(s[i] * Two(-inv_here), s[i], q[i]);
    };
    auto normalise = [&](auto whole_tile, const Two (&mean)[PAIRS<VP>], const Two (&rstd)[PAIRS<VP>]) {
        constexpr bool FULL = decltype(whole_tile)::value;
        T* y = t.at(a.out, a.pout, a);
        Two less[PAIRS<VP>];
#pragma unroll
        for (int i = 0; i < PAIRS<VP>; ++i) less[i] = mean[i] * Two(-1.f);
#pragma unroll 4
        for (int j = 0; j < t.template count<FULL>(); ++j, y += a.inner) {
            Two v[PAIRS<VP>];
            unpack<T, VP>(t.slot(0, j), v);
            const Two w(wt[t.first + j]), b(bs[t.first + j]);
#pragma unroll
            for (int i = 0; i < PAIRS<VP>; ++i) v[i] = fma2((v[i] + less[i]) * rstd[i], w, b);
            t.template store<FULL>(y, piece_of<T, VP>(v));
        }
        if (t.warp == 0 && t.live && (a.mean || a.rstd)) {
#pragma unroll
            for (int i = 0; i < VP; ++i) {
                if (SPREAD && i >= t.live) break;
                if (a.mean) a.mean[t.position(i, a)] = i % 2 ? mean[i / 2].hi() : mean[i / 2].lo();
                if (a.rstd) a.rstd[t.position(i, a)] = i % 2 ? rstd[i / 2].hi() : rstd[i / 2].lo();
            }
        }
    };
    fetch(blockIdx.x);
    __syncthreads();                                     // the weights
    for (long long tile = blockIdx.x; tile < t.tiles; tile += gridDim.x) {
        copies_wait<0>();
        Two mean[PAIRS<VP>], dev[PAIRS<VP>], rstd[PAIRS<VP>];
        if (full) statistics(True{}, mean, dev);
        else statistics(False{}, mean, dev);
        // with m_w a warp's mean, the sum of (d + m_w - m)^2 is that of d^2 and n_w (m_w - m)^2
        map_exchange<VP>(sums, warps, t.lane, t.warp, mean, dev, mean, rstd, [&](int, const float* ps, const float* pd, float* to, int N) {
            float all = 0.f, q = 0.f;
            for (int u = 0; u < warps; ++u) all += ps[u * N];
            const float m = quotient(all, count, inv_count);
            for (int u = 0; u < warps; ++u) {
                const bool last = u == warps - 1;
                const float d = fmaf(ps[u * N], last ? inv_last : 1.f / ITEMS, -m);
                q += fmaf((last ? last_features : (float)ITEMS) * d, d, pd[u * N]);
            }
            to[0] = m;
            to[N] = inverse_root(not_negative(q) * inv_count + a.eps);
        });
        if (full) normalise(True{}, mean, rstd);
        else normalise(False{}, mean, rstd);
        fetch(tile + gridDim.x);
    }
}

template <class T, int VP, int ITEMS, bool TAIL, bool SPREAD>
__global__ void __launch_bounds__(MAP_TILE_WARPS * 32, 1) map_tile_vjp(const __grid_constant__ Args a) {
    grid_dependency_wait();
    extern __shared__ __align__(16) float shared[];
    const int warps = blockDim.x >> 5, n = (int)a.features;
    float* sums = shared;
    float* wt = sums + map_exchange_floats(VP, warps);
    MapTile<T, VP, ITEMS, TAIL ? 3 : 2, SPREAD> t(a, wt + warps * ITEMS * 2);
    for (int c = threadIdx.x; c < warps * ITEMS; c += blockDim.x) wt[c] = c >= n ? 0.f : a.weight ? weight_at<T>(a.weight, a.weight_f32, c) : 1.f;
    const Mask mask(a);
    const bool added = TAIL && a.gsum;
    const float inv_count = 1.f / (float)n;
    Two less[PAIRS<VP>], rstd[PAIRS<VP>];
    bool full = false;
    auto fetch = [&](long long tile) {
        if (tile < t.tiles) {
            t.go(tile, a);
            full = t.full();
            if (full) {
                t.template fetch<true>(0, a.x, a.px, a);
                t.template fetch<true>(1, a.res, a.pres, a);
                if (added) t.template fetch<true>(2, a.gsum, a.pgsum, a);
            } else {
                t.template fetch<false>(0, a.x, a.px, a);
                t.template fetch<false>(1, a.res, a.pres, a);
                if (added) t.template fetch<false>(2, a.gsum, a.pgsum, a);
            }
            if (t.live) {
                auto mean = [&](int m) { return !SPREAD || m < t.live ? -a.mean[t.position(m, a)] : 0.f; };
                auto root = [&](int m) { return !SPREAD || m < t.live ? a.rstd[t.position(m, a)] : 0.f; };
                if constexpr (VP == 1) { less[0] = Two(mean(0), 0.f); rstd[0] = Two(root(0), 0.f); }
                else {
#pragma unroll
                    for (int i = 0; i < VP / 2; ++i) { less[i] = Two(mean(2 * i), mean(2 * i + 1)); rstd[i] = Two(root(2 * i), root(2 * i + 1)); }
                }
            }
        }
        copies_commit();
    };
    float gw[ITEMS], gb[ITEMS];
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) gw[j] = gb[j] = 0.f;
    auto sum_up = [&](auto whole_tile, Two (&s1)[PAIRS<VP>], Two (&s2)[PAIRS<VP>]) {
        constexpr bool FULL = decltype(whole_tile)::value;
#pragma unroll
        for (int i = 0; i < PAIRS<VP>; ++i) s1[i] = s2[i] = Two(0.f);
#pragma unroll
        for (int j = 0; j < ITEMS; ++j) {
            if (!FULL && !(t.live && j < t.items)) continue;
            Two g[PAIRS<VP>], v[PAIRS<VP>], sw(0.f), sb(0.f);
            unpack<T, VP>(t.slot(0, j), g);
            unpack<T, VP>(t.slot(1, j), v);
            if constexpr (SPREAD && !FULL) {             // positions that are not there hold anything
                auto there = [&](Two (&u)[PAIRS<VP>]) {
                    u[0] = Two(u[0].lo(), t.live > 1 ? u[0].hi() : 0.f);
                    u[1] = Two(t.live > 2 ? u[1].lo() : 0.f, t.live > 3 ? u[1].hi() : 0.f);
                };
                there(g);
                there(v);
            }
            const Two w(wt[t.first + j]);
#pragma unroll
            for (int i = 0; i < PAIRS<VP>; ++i) {
                const Two h = (v[i] + less[i]) * rstd[i], d = g[i] * w;
                sw = i ? fma2(g[i], h, sw) : g[i] * h;
                sb = i ? sb + g[i] : g[i];
                s1[i] = s1[i] + d;
                s2[i] = fma2(d, h, s2[i]);
            }
            gw[j] += sw.sum(); gb[j] += sb.sum();
        }
    };
    auto gradient = [&](auto whole_tile, const Two (&c1)[PAIRS<VP>], const Two (&c2)[PAIRS<VP>]) {
        constexpr bool FULL = decltype(whole_tile)::value;
        T* out = t.at(a.out, a.pout, a);
        T* out2 = TAIL ? t.at(a.out2, a.pout2, a) : nullptr;
        MaskPlace<VP, SPREAD> place(a, TAIL ? t.element(a) : 0);
#pragma unroll 2
        for (int j = 0; j < t.template count<FULL>(); ++j, out += a.inner) {
            Two g[PAIRS<VP>], v[PAIRS<VP>];
            unpack<T, VP>(t.slot(0, j), g);
            unpack<T, VP>(t.slot(1, j), v);
            const Two w(wt[t.first + j]);
            // rstd (g w - mean(g w) - h mean(g w h))
#pragma unroll
            for (int i = 0; i < PAIRS<VP>; ++i) v[i] = fma2((v[i] + less[i]) * rstd[i], c2[i], fma2(g[i], w, c1[i])) * rstd[i];
            if (TAIL) {
                if (added) {
                    unpack<T, VP>(t.slot(2, j), g);
#pragma unroll
                    for (int i = 0; i < PAIRS<VP>; ++i) v[i] = v[i] + g[i];
                }
                t.template store<FULL>(out2, piece_of<T, VP>(v));
                if (a.dropping) {
                    if constexpr (SPREAD) drop_spread<false>(mask, place.at, t.lane, v, v);
                    else drop_piece<false, VP>(mask, place, v, v);
                }
                out2 += a.inner; place.next(a);
            }
            t.template store<FULL>(out, piece_of<T, VP>(v));
        }
    };
    fetch(blockIdx.x);
    __syncthreads();                                     // the weights
    for (long long tile = blockIdx.x; tile < t.tiles; tile += gridDim.x) {
        copies_wait<0>();
        Two c1[PAIRS<VP>], c2[PAIRS<VP>];
        if (full) sum_up(True{}, c1, c2);
        else sum_up(False{}, c1, c2);
        map_exchange<VP>(sums, warps, t.lane, t.warp, c1, c2, c1, c2, [&](int, const float* p1, const float* p2, float* to, int N) {
            float all1 = 0.f, all2 = 0.f;
            for (int u = 0; u < warps; ++u) { all1 += p1[u * N]; all2 += p2[u * N]; }
            to[0] = -all1 * inv_count; to[N] = -all2 * inv_count;
        });
        if (full) gradient(True{}, c1, c2);
        else gradient(False{}, c1, c2);
        fetch(tile + gridDim.x);
    }
    if (!a.gw && !a.gb) return;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
        if (j >= t.items) break;
        const float w = lanes_sum<32>(gw[j]), b = lanes_sum<32>(gb[j]);
        const int c = t.first + j;
        if (t.lane != 0) continue;
        if (gridDim.x > 1) {
            a.part[(long long)blockIdx.x * 2 * n + c] = w;
            a.part[((long long)blockIdx.x * 2 + 1) * n + c] = b;
        } else {
            if (a.gw) store_weight_grad<T>(a.gw, a.weight_f32, c, w);
            if (a.gb) store_weight_grad<T>(a.gb, a.weight_f32, c, b);
        }
    }
}

}  // namespace prior
}  // namespace gleam
