// The gated recurrence where a chain's steps lie one behind the other (inner = 1).
//
// Short chains (up to 128 bytes): a block takes 128 of them through shared memory, where each thread runs one; what goes in and out are
// contiguous pieces of 16 bytes.  The VJP has the whole chain at hand, and nothing is saved for it.
//
// Longer chains: a warp takes a run of whole chains, or a part of one, in tiles of 32 lanes with V neighbouring steps each.  A lane composes
// the maps of its own steps, the lanes' maps are composed by shuffles (five turns), and the state behind the tile goes on to the next
// one, whose bytes are already on their way.  Where a chain begins inside a tile its map forgets what came before, so chains share
// tiles.  Tiles begin at multiples of V elements of the whole array, wherever its chains begin.  Tiles inside a chain, nearly
// all of a long one, need no marks of where chains begin: 16 x 262145 float32, forward and VJP, 84 -> 47 us.
#pragma once
#include "scan_stream.cuh"

#include <type_traits>

namespace gleam {
namespace scan {

// ---- short chains

constexpr int SHORT_BYTES = 128, SHORT_ROWS = 128, SHORT_CHUNK = 8;      // steps between the VJP's states
template <class T> constexpr int SHORT_STEPS = SHORT_BYTES / sizeof(T);

// Where byte b of the block's part of an array stands.  Neighbouring chains of 16, 32, 64 or 128 bytes would share their banks: there 16
// bytes more stand between every 128; the others' steps keep them apart.
__host__ __device__ __forceinline__ bool short_skews(int chain) { return 128 % chain == 0; }
__host__ __device__ __forceinline__ int skewed(int b, bool skews) { return skews ? b + (b >> 7) * 16 : b; }
template <class T> __host__ __device__ inline int short_array(long long steps) {
    return (skewed((int)(SHORT_ROWS * steps * sizeof(T)), short_skews((int)(steps * sizeof(T)))) + 31) / 16 * 16;
}
template <class T, int KIND> __host__ inline size_t short_smem(long long steps) {
    return KIND == VJP ? 3 * (size_t)short_array<T>(steps) + sizeof(float) * SHORT_ROWS * (SHORT_STEPS<T> / SHORT_CHUNK) : 2 * (size_t)short_array<T>(steps);
}

// Two neighbouring steps t and t + 1 of a chain.  WHOLE: as one number of 32 bits (16-bit types, an even number of steps).
template <class T, bool WHOLE>
__device__ __forceinline__ Two steps_at(const T* chain, int t) {
    if constexpr (WHOLE) return pair_of(chain + t);
    else return Two(to_float(chain[t]), to_float(chain[t + 1]));
}
template <class T, bool WHOLE>
__device__ __forceinline__ void put_steps(T* chain, int t, Two v) {
    if constexpr (WHOLE) round_pair(chain + t, v);
    else { chain[t] = from_float<T>(v.lo()); chain[t + 1] = from_float<T>(v.hi()); }
}

// DENSE: all arrays without gaps and from 16 bytes on.
template <class T, bool REVERSE, bool DENSE, bool WHOLE, int KIND>
__global__ void __launch_bounds__(SHORT_ROWS) short_kernel(const __grid_constant__ Args a) {
    extern __shared__ __align__(16) unsigned char ring[];
    grid_dependency_wait();
    constexpr bool BACK = KIND == VJP;
    const int steps = (int)a.steps, bytes = short_array<T>(a.steps), chain = steps * (int)sizeof(T);
    const bool skews = short_skews(chain);
    const long long row0 = (long long)blockIdx.x * SHORT_ROWS, row = row0 + threadIdx.x;
    const int rows = (int)(a.rows - row0 < SHORT_ROWS ? a.rows - row0 : SHORT_ROWS), count = rows * steps;
    auto element = [&](unsigned char* from, int i) -> T& { return *reinterpret_cast<T*>(from + skewed(i * (int)sizeof(T), skews)); };
    auto address = [&](const Strides& s, int i) {
        const int r = i / steps;
        const long long u = row0 + r, b = u / a.channels;
        return b * s.batch + (u - b * a.channels) * s.channel + (i - r * steps) * s.step;
    };
    const int whole = DENSE ? count * (int)sizeof(T) / 16 : 0;             // pieces
    auto take = [&](unsigned char* to, const void* from, const Strides& s) {
        const T* p = static_cast<const T*>(from);
        const unsigned char* q = reinterpret_cast<const unsigned char*>(p + row0 * steps);
        for (int i = threadIdx.x; i < whole; i += SHORT_ROWS) copy_async<16>((uint32_t)__cvta_generic_to_shared(to) + skewed(16 * i, skews), q + 16 * i);
        for (int i = whole * (16 / (int)sizeof(T)) + threadIdx.x; i < count; i += SHORT_ROWS) element(to, i) = DENSE ? p[row0 * steps + i] : p[address(s, i)];
    };
    auto give = [&](void* to, const Strides& s, unsigned char* from) {
        T* p = static_cast<T*>(to);
        unsigned char* q = reinterpret_cast<unsigned char*>(p + row0 * steps);
        for (int i = threadIdx.x; i < whole; i += SHORT_ROWS) *reinterpret_cast<uint4*>(q + 16 * i) = *reinterpret_cast<const uint4*>(from + skewed(16 * i, skews));
        for (int i = whole * (16 / (int)sizeof(T)) + threadIdx.x; i < count; i += SHORT_ROWS) {
            if (DENSE) p[row0 * steps + i] = element(from, i);
            else p[address(s, i)] = element(from, i);
        }
    };
    take(ring, a.gate, a.sgate);
    take(ring + bytes, a.x, a.sx);
    if (BACK) take(ring + 2 * bytes, a.dy, a.sdy);
    copies_end();
    copies_wait<0>();
    __syncthreads();
    if (row < a.rows) {
        T* gs = &element(ring, threadIdx.x * steps);                       // the thread's chain; a chain of 2^n bytes lies between two gaps
        T* xs = &element(ring + bytes, threadIdx.x * steps);
        const T* ds = &element(ring + 2 * bytes, threadIdx.x * steps);
        const int valid = a.lengths ? (int)valid_steps(a, row / a.channels) : steps;
        float h = a.state ? a.state[row] : 0.f;
        // position q = 0, 1, ... is step q or T - 1 - q.  Two positions q, q + 1 at a time, whose steps lie side by side from `low` on; an odd
        // number of steps leaves one over at the end, which stands alone in the first half of its pair.
        const int pairs = steps / 2;
        auto low = [&](int pair) { return REVERSE ? steps - 2 - 2 * pair : 2 * pair; };
        const int odd = REVERSE ? 0 : steps - 1;                           // the step that is left over
        auto turned = [](Two v) { return REVERSE ? Two(v.hi(), v.lo()) : v; };
        auto there = [&](int t, int second) { return t + (REVERSE ? 1 - second : second) < valid; };
        if (!BACK) {
            auto run = [&](auto all) {                                     // all: no step is behind the example's length
                constexpr bool ALL = decltype(all)::value;
#pragma unroll 2
                for (int p = 0; p < pairs; ++p) {
                    const int t = low(p);
                    Two f, rest;
                    gates_of<T>(turned(steps_at<T, WHOLE>(gs, t)), f, rest);
                    const Two u = rest * turned(steps_at<T, WHOLE>(xs, t));
                    float v0 = 0.f, v1 = 0.f;
                    if (ALL || there(t, 0)) v0 = h = fmaf(f.lo(), h, u.lo());
                    if (ALL || there(t, 1)) v1 = h = fmaf(f.hi(), h, u.hi());
                    put_steps<T, WHOLE>(xs, t, turned(Two(v0, v1)));
                }
                if (!WHOLE && steps & 1) {
                    float f, rest;
                    gate_of<T>(to_float(gs[odd]), f, rest);
                    if (ALL || odd < valid) h = fmaf(f, h, rest * to_float(xs[odd]));
                    xs[odd] = from_float<T>(ALL || odd < valid ? h : 0.f);
                }
            };
            if (valid == steps) run(std::true_type{});
            else run(std::false_type{});
            if (a.last) a.last[row] = h;
        } else {
            float* starts = reinterpret_cast<float*>(ring + 3 * bytes) + threadIdx.x;     // states at the chunks' starts
            for (int p = 0; p < pairs; ++p) {
                const int t = low(p);
                if (p % (SHORT_CHUNK / 2) == 0) starts[p / (SHORT_CHUNK / 2) * SHORT_ROWS] = h;
                Two f, rest;
                gates_of<T>(turned(steps_at<T, WHOLE>(gs, t)), f, rest);
                const Two u = rest * turned(steps_at<T, WHOLE>(xs, t));
                if (there(t, 0)) h = fmaf(f.lo(), h, u.lo());
                if (there(t, 1)) h = fmaf(f.hi(), h, u.hi());
            }
            float back = a.dlast ? a.dlast[row] : 0.f;
            if (!WHOLE && steps & 1) {                                     // the last position first
                float f, rest, ox = 0.f, og = 0.f;
                gate_of<T>(to_float(gs[odd]), f, rest);
                if (odd < valid) {
                    const float d = back + to_float(ds[odd]), w = h - to_float(xs[odd]);
                    back = d * f;
                    ox = d * rest;
                    og = ox * f * w;
                }
                xs[odd] = from_float<T>(ox);
                gs[odd] = from_float<T>(og);
            }
            for (int p0 = (pairs - 1) / (SHORT_CHUNK / 2) * (SHORT_CHUNK / 2); p0 >= 0 && pairs > 0; p0 -= SHORT_CHUNK / 2) {
                Two f[SHORT_CHUNK / 2], rest[SHORT_CHUNK / 2], w[SHORT_CHUNK / 2];
                h = starts[p0 / (SHORT_CHUNK / 2) * SHORT_ROWS];
#pragma unroll
                for (int k = 0; k < SHORT_CHUNK / 2; ++k) {
                    if (p0 + k >= pairs) break;
                    const int t = low(p0 + k);
                    gates_of<T>(turned(steps_at<T, WHOLE>(gs, t)), f[k], rest[k]);
                    const Two x = turned(steps_at<T, WHOLE>(xs, t)), u = rest[k] * x;
                    const float w0 = h - x.lo();
                    if (there(t, 0)) h = fmaf(f[k].lo(), h, u.lo());
                    w[k] = Two(w0, h - x.hi());
                    if (there(t, 1)) h = fmaf(f[k].hi(), h, u.hi());
                }
#pragma unroll
                for (int k = SHORT_CHUNK / 2 - 1; k >= 0; --k) {
                    if (p0 + k >= pairs) continue;
                    const int t = low(p0 + k);
                    const Two d = turned(steps_at<T, WHOLE>(ds, t));
                    float d0 = 0.f, d1 = 0.f;
                    if (there(t, 1)) { d1 = back + d.hi(); back = d1 * f[k].hi(); }
                    if (there(t, 0)) { d0 = back + d.lo(); back = d0 * f[k].lo(); }
                    const Two ox = Two(d0, d1) * rest[k];
                    Two og = ox * f[k] * w[k];
                    if (valid < steps) og = Two(there(t, 0) ? og.lo() : 0.f, there(t, 1) ? og.hi() : 0.f);       // what is not there may be NaN
                    put_steps<T, WHOLE>(xs, t, turned(valid < steps ? Two(there(t, 0) ? ox.lo() : 0.f, there(t, 1) ? ox.hi() : 0.f) : ox));
                    put_steps<T, WHOLE>(gs, t, turned(og));
                }
            }
            if (a.dstate) a.dstate[row] = back;
        }
    }
    __syncthreads();
    give(BACK ? a.dx : a.y, BACK ? a.sdx : a.sy, ring + bytes);
    if (BACK) give(a.dg, a.sdg, ring);
}

// ---- longer chains

constexpr int ROW_WARPS = 4;
template <class T> constexpr int ROW_V = 8;
template <class T> constexpr int TILE = 32 * ROW_V<T>;

// Chains of a run: enough tiles for a warp to be worth its start, and runs for all SMs.  A multiple of 8, so that runs begin at
// multiples of 16 bytes.  It depends on the sizes alone: the states that the forward call saves are numbered by it.
inline long long run_rows(long long rows, long long steps, int tile) {
    if (steps >= 4 * tile || rows < 8) return 1;
    const long long warps = 148 * 32;
    long long r = (rows + warps - 1) / warps, most = 64ll * tile / steps;
    if (r > most) r = most;
    const long long least = (2ll * tile + steps - 1) / steps;
    if (r < least) r = least;
    return (r + 7) / 8 * 8;
}
// Tiles of a run, wherever it begins.
template <class T> __host__ __device__ inline long long run_tiles(long long run, long long steps) { return (run * steps + ROW_V<T> - 1 + TILE<T> - 1) / TILE<T>; }

// The map s -> a s + b.  a < 0 (a product of gates is not) is s -> b, whatever s is: another chain's NaN is not multiplied away by 0.
struct Map { float a, b; };
constexpr float FORGETS = -1.f;
__device__ __forceinline__ float apply(const Map& m, float s) { return m.a < 0.f ? m.b : fmaf(m.a, s, m.b); }
__device__ __forceinline__ Map then(const Map& first, const Map& second) {
    return Map{second.a < 0.f || first.a < 0.f ? FORGETS : second.a * first.a, apply(second, first.b)};
}

// The maps of all lanes before this one (UP: lower lanes come first), composed; `all`: those of the whole warp.
template <bool UP>
__device__ __forceinline__ Map before_lane(Map m, Map* all) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        Map u;
        u.a = UP ? __shfl_up_sync(0xffffffffu, m.a, o) : __shfl_down_sync(0xffffffffu, m.a, o);
        u.b = UP ? __shfl_up_sync(0xffffffffu, m.b, o) : __shfl_down_sync(0xffffffffu, m.b, o);
        if (UP ? lane >= o : lane + o < 32) m = then(u, m);
    }
    all->a = __shfl_sync(0xffffffffu, m.a, UP ? 31 : 0);
    all->b = __shfl_sync(0xffffffffu, m.b, UP ? 31 : 0);
    Map r;
    r.a = UP ? __shfl_up_sync(0xffffffffu, m.a, 1) : __shfl_down_sync(0xffffffffu, m.a, 1);
    r.b = UP ? __shfl_up_sync(0xffffffffu, m.b, 1) : __shfl_down_sync(0xffffffffu, m.b, 1);
    if (lane == (UP ? 0 : 31)) r = Map{1.f, 0.f};
    return r;
}

// A lane's V elements of an array.
template <class T> union Lane { uint4 piece[ROW_V<T> * sizeof(T) / 16]; T e[ROW_V<T>]; __device__ Lane() {} };

// SINGLE: a run is one chain or a part of one.  Chains are longer than V.
template <class T, bool REVERSE, bool DENSE, bool SINGLE, int KIND>
__global__ void __launch_bounds__(ROW_WARPS * 32) rows_kernel(const __grid_constant__ Args a) {
    grid_dependency_wait();
    constexpr int V = ROW_V<T>, N = TILE<T>;
    constexpr bool MAPS = KIND == MAP_FORWARD || KIND == MAP_VJP, BACK = KIND == VJP || KIND == MAP_VJP, AGAINST = BACK != REVERSE;
    const int lane = threadIdx.x & 31;
    const long long w = (long long)blockIdx.x * ROW_WARPS + (threadIdx.x >> 5);
    const long long row0 = SINGLE ? w / a.parts : w * a.run, part = SINGLE ? w - row0 * a.parts : 0;
    if (row0 >= a.rows) return;
    // Element 0 of tile 0 stands `head` elements before the run; the part's tiles.  Elements of a run are counted in 32 bits.
    const int steps = (int)a.steps, head = SINGLE ? (int)(row0 * a.steps % V) : 0;
    const int length = SINGLE ? steps : (int)((row0 + a.run < a.rows ? a.run : a.rows - row0) * a.steps);
    const int all_tiles = (int)(((long long)length + head + N - 1) / N), each = a.parts > 1 ? (int)(a.part / N) : all_tiles, tile0 = (int)part * each;
    const int tiles = tile0 + each < all_tiles ? each : all_tiles - tile0;
    const long long first_saved = (SINGLE ? row0 : w) * run_tiles<T>(a.run, a.steps) + tile0;
    float state = 0.f, total = 1.f;
    if (!MAPS && a.parts > 1) state = a.maps_b[part * a.rows + row0];

    // the lane's element 0 of a tile, counted from the run's first; AGAINST: tiles from the end of memory to its start
    auto element0 = [&](int k) { return (tile0 + (AGAINST ? tiles - 1 - k : k)) * N + lane * V - head; };
    struct Raw { Lane<T> g, x, d; };
    // where the run begins in an array, and elements of it
    auto start = [&](const Strides& s) { const long long b = row0 / a.channels; return DENSE ? row0 * a.steps : SINGLE ? b * s.batch + (row0 - b * a.channels) * s.channel : 0ll; };
    auto offset = [&](const Strides& s, int e) -> long long {
        if (DENSE) return e;
        if (SINGLE) return e * s.step;
        const int r = e / steps;
        const long long u = row0 + r, b = u / a.channels;
        return b * s.batch + (u - b * a.channels) * s.channel + (e - r * steps) * s.step;
    };
    const T* gate = static_cast<const T*>(a.gate) + start(a.sgate);
    const T* xs = KIND != MAP_VJP ? static_cast<const T*>(a.x) + start(a.sx) : nullptr;
    const T* dys = BACK ? static_cast<const T*>(a.dy) + start(a.sdy) : nullptr;
    T* ys = KIND == FORWARD ? static_cast<T*>(a.y) + start(a.sy) : nullptr;
    T* dxs = KIND == VJP ? static_cast<T*>(a.dx) + start(a.sdx) : nullptr;
    T* dgs = KIND == VJP ? static_cast<T*>(a.dg) + start(a.sdg) : nullptr;
    auto fetch_one = [&](Lane<T>& to, const T* p, const Strides& s, int e) {
        if (DENSE && e >= 0 && e <= length - V) {
#pragma unroll
            for (int j = 0; j < (int)(V * sizeof(T) / 16); ++j) to.piece[j] = reinterpret_cast<const uint4*>(p + e)[j];
            return;
        }
#pragma unroll
        for (int j = 0; j < V; ++j) to.e[j] = e + j >= 0 && e < length - j ? p[offset(s, e + j)] : from_float<T>(0.f);
    };
    auto fetch = [&](int k, Raw& raw) {
        const int e = element0(k);
        fetch_one(raw.g, gate, a.sgate, e);
        if (KIND != MAP_VJP) fetch_one(raw.x, xs, a.sx, e);
        if (BACK) fetch_one(raw.d, dys, a.sdy, e);
    };
    auto store = [&](T* p, const Strides& s, int e, const float (&v)[V]) {
        if (DENSE && e >= 0 && e <= length - V) {
            Lane<T> u;
#pragma unroll
            for (int j = 0; j < V; j += 2) round_pair(u.e + j, Two(v[j], v[j + 1]));
#pragma unroll
            for (int j = 0; j < (int)(V * sizeof(T) / 16); ++j) reinterpret_cast<uint4*>(p + e)[j] = u.piece[j];
            return;
        }
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (e + j >= 0 && e < length - j) p[offset(s, e + j)] = from_float<T>(v[j]);
    };

    // One tile.  inner: all of it is there, and no chain begins or ends in it.
    auto tile = [&](int k, const Raw& raw, auto inner) {
        constexpr bool INNER = decltype(inner)::value;
        const int e = element0(k);
        uint32_t valid = (1u << V) - 1, there = valid, first = 0, last = 0;
        int border = V;
        long long row = row0;
        if (!INNER) {
            // the chain of element 0 and where the next one begins; elements that are there
            int step = e;
            if (!SINGLE && e > 0) { const int r = e / steps; row += r; step -= r * steps; }
            border = steps - step < V ? steps - step : V;
            if (e < 0) there = e <= -V ? 0 : there << -e & there;
            if (e > length - V) there = e >= length ? 0 : there & ((1u << (length - e)) - 1);
            valid = there;
            if (a.lengths && there) {
                const long long n0 = valid_steps(a, row / a.channels) - step;
                uint32_t in = n0 <= 0 ? 0 : n0 >= border ? (1u << border) - 1 : (1u << (int)n0) - 1;
                if (!SINGLE && border < V && row + 1 < a.rows) {
                    const long long n1 = valid_steps(a, (row + 1) / a.channels), most = V - border;
                    in |= ((n1 >= most ? (1u << (int)most) - 1 : (1u << (int)n1) - 1) << border);
                }
                valid &= in;
            }
            // chains begin at step 0 and end at the last one in memory; REVERSE: the other way round
            uint32_t low = step <= 0 && step > -V ? 1u << -step : 0, high = border > 0 && steps - step <= V ? 1u << (border - 1) : 0;
            if (!SINGLE && border < V) low |= 1u << border;
            low &= there; high &= there;
            first = REVERSE ? high : low; last = REVERSE ? low : high;
        }
        auto row_of = [&](int j) { return SINGLE || j < border ? row : row + 1; };

        float f[V], rest[V], x[V], d[V], h[V];                                       // h: forward h_t; VJP h_(t-1)
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            Two f2, rest2;
            gates_of<T>(pair_of(raw.g.e + j), f2, rest2);
            f[j] = f2.lo(); f[j + 1] = f2.hi(); rest[j] = rest2.lo(); rest[j + 1] = rest2.hi();
            if (KIND != MAP_VJP) { const Two v = pair_of(raw.x.e + j); x[j] = v.lo(); x[j + 1] = v.hi(); }
            if (BACK) { const Two v = pair_of(raw.d.e + j); d[j] = v.lo(); d[j + 1] = v.hi(); }
        }
        if (!INNER && valid != (1u << V) - 1) {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (!(valid >> j & 1)) { f[j] = 1.f; rest[j] = 0.f; x[j] = 0.f; d[j] = 0.f; }
        }
        if (KIND != MAP_VJP) {
            // the lane's own steps from a state of zero, then the state before them
            Map own{1.f, 0.f}, all;
            float enters = 0.f;
            const bool begins = !INNER && !MAPS && first;
            if (begins) enters = a.state ? a.state[row_of(__ffs(first) - 1)] : 0.f;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int j = REVERSE ? V - 1 - i : i;
                if (begins && first >> j & 1) own = Map{FORGETS, enters};
                own.b = fmaf(f[j], own.b, rest[j] * x[j]);
                if (own.a >= 0.f || !begins) own.a *= f[j];
            }
            const Map pre = before_lane<!REVERSE>(own, &all);
            if (MAPS) {
                state = apply(all, state); total *= all.a;
            } else {
                float enter = state;
                const long long saved_at = first_saved + (AGAINST ? tiles - 1 - k : k);
                if (KIND == VJP) enter = a.saved[saved_at];
                else if (a.saved && lane == 0) a.saved[saved_at] = state;
                float s = apply(pre, enter);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int j = REVERSE ? V - 1 - i : i;
                    if (begins && first >> j & 1) s = enters;
                    if (KIND == VJP) h[j] = s;
                    s = fmaf(f[j], s, rest[j] * x[j]);
                    if (KIND == FORWARD) {
                        h[j] = s;
                        if (!INNER && last >> j & 1 && a.last) a.last[row_of(j)] = s;
                    }
                }
                if (KIND == FORWARD) state = apply(all, state);
            }
        }
        if (KIND == FORWARD) {
            if (!INNER && valid != there) {
#pragma unroll
                for (int j = 0; j < V; ++j) if (!(valid >> j & 1)) h[j] = 0.f;
            }
            store(ys, a.sy, e, h);
        }
        if (BACK) {
            Map own{1.f, 0.f}, all;
            float enters = 0.f;
            const bool begins = !INNER && !MAPS && last;
            if (begins) enters = a.dlast ? a.dlast[row_of(__ffs(last) - 1)] : 0.f;
#pragma unroll
            for (int i = V - 1; i >= 0; --i) {
                const int j = REVERSE ? V - 1 - i : i;
                if (begins && last >> j & 1) own = Map{FORGETS, enters};
                own.b = f[j] * (own.b + d[j]);
                if (own.a >= 0.f || !begins) own.a *= f[j];
            }
            const Map pre = before_lane<REVERSE>(own, &all);
            if (MAPS) {
                state = apply(all, state); total *= all.a;
            } else {
                float s = apply(pre, state);
                float ox[V], og[V];
#pragma unroll
                for (int i = V - 1; i >= 0; --i) {
                    const int j = REVERSE ? V - 1 - i : i;
                    if (begins && last >> j & 1) s = enters;
                    const float c = s + d[j];
                    ox[j] = c * rest[j];
                    og[j] = ox[j] * f[j] * (h[j] - x[j]);
                    s = f[j] * c;
                    if (!INNER && first >> j & 1 && a.dstate) a.dstate[row_of(j)] = s;
                }
                state = apply(all, state);
                if (!INNER && valid != there) {
#pragma unroll
                    for (int j = 0; j < V; ++j) if (!(valid >> j & 1)) ox[j] = og[j] = 0.f;
                }
                store(dxs, a.sdx, e, ox);
                store(dgs, a.sdg, e, og);
            }
        }
    };

    Raw next;
    if (tiles > 0) fetch(0, next);
    for (int k = 0; k < tiles; ++k) {
        const Raw raw = next;
        if (k + 1 < tiles) fetch(k + 1, next);
        const int begin = element0(k) - lane * V;
        if (SINGLE && !a.lengths && begin > 0 && begin < length - N) tile(k, raw, std::true_type{});
        else tile(k, raw, std::false_type{});
    }
    if (MAPS && lane == 0) {
        a.maps_a[part * a.rows + row0] = total;
        a.maps_b[part * a.rows + row0] = state;
    }
}

}  // namespace scan
}  // namespace gleam
