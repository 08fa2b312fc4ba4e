// The gated recurrence where a chain's steps lie one behind the other (inner = 1).
//
// Short chains (up to 128 bytes): a block takes 128 of them through shared memory, where each thread runs one; what goes in and out are
// contiguous pieces of 16 bytes.  The VJP has the whole chain at hand, and nothing is saved for it.
//
// Longer chains: a warp takes a run of whole chains, or a part of one, in tiles of 32 lanes with V neighbouring steps each.  A lane composes
// the maps of its own steps, the lanes' maps are composed by shuffles (five turns), and the state behind the tile goes on to the next
// one, whose bytes are already on their way.  Where a chain begins inside a tile its map forgets what came before, so chains share
// tiles.  Tiles begin at multiples of V elements of the whole array, wherever its chains begin.
#pragma once
#include "scan_stream.cuh"

namespace gleam {
namespace scan {

// ---- short chains

constexpr int SHORT_BYTES = 128, SHORT_ROWS = 128;
template <class T> constexpr int SHORT_STEPS = SHORT_BYTES / sizeof(T);

// Where byte b of the block's part of an array stands: 16 bytes more every 128, so that neighbouring chains differ in their banks.
__host__ __device__ __forceinline__ int skewed(int b) { return b + (b >> 7) * 16; }
template <class T> __host__ __device__ inline int short_array(long long steps) { return (skewed((int)(SHORT_ROWS * steps * sizeof(T))) + 31) / 16 * 16; }
template <class T, int KIND> __host__ inline size_t short_smem(long long steps) {
    return KIND == VJP ? 3 * (size_t)short_array<T>(steps) + sizeof(float) * SHORT_ROWS * (SHORT_STEPS<T> / CHUNK) : 2 * (size_t)short_array<T>(steps);
}

// DENSE: all arrays without gaps and from 16 bytes on.
template <class T, bool REVERSE, bool DENSE, int KIND>
__global__ void __launch_bounds__(SHORT_ROWS) short_kernel(const __grid_constant__ Args a) {
    extern __shared__ __align__(16) unsigned char ring[];
    grid_dependency_wait();
    constexpr bool BACK = KIND == VJP;
    const int steps = (int)a.steps, bytes = short_array<T>(a.steps);
    const long long row0 = (long long)blockIdx.x * SHORT_ROWS, row = row0 + threadIdx.x;
    const int rows = (int)(a.rows - row0 < SHORT_ROWS ? a.rows - row0 : SHORT_ROWS), count = rows * steps;
    unsigned char* in_g = ring;
    unsigned char* in_x = ring + bytes;
    unsigned char* in_d = ring + 2 * bytes;
    auto element = [&](unsigned char* from, int i) -> T& { return *reinterpret_cast<T*>(from + skewed(i * (int)sizeof(T))); };
    auto address = [&](const Strides& s, int i) {
        const int r = i / steps;
        const long long u = row0 + r, b = u / a.channels;
        return b * s.batch + (u - b * a.channels) * s.channel + (i - r * steps) * s.step;
    };
    const int whole = DENSE ? count * (int)sizeof(T) / 16 : 0;             // pieces
    auto take = [&](unsigned char* to, const void* from, const Strides& s) {
        const T* p = static_cast<const T*>(from);
        const unsigned char* q = reinterpret_cast<const unsigned char*>(p + row0 * steps);
        for (int i = threadIdx.x; i < whole; i += SHORT_ROWS) copy_async<16>((uint32_t)__cvta_generic_to_shared(to) + skewed(16 * i), q + 16 * i);
        for (int i = whole * (16 / (int)sizeof(T)) + threadIdx.x; i < count; i += SHORT_ROWS) element(to, i) = DENSE ? p[row0 * steps + i] : p[address(s, i)];
    };
    auto give = [&](void* to, const Strides& s, unsigned char* from) {
        T* p = static_cast<T*>(to);
        unsigned char* q = reinterpret_cast<unsigned char*>(p + row0 * steps);
        for (int i = threadIdx.x; i < whole; i += SHORT_ROWS) *reinterpret_cast<uint4*>(q + 16 * i) = *reinterpret_cast<const uint4*>(from + skewed(16 * i));
        for (int i = whole * (16 / (int)sizeof(T)) + threadIdx.x; i < count; i += SHORT_ROWS) {
            if (DENSE) p[row0 * steps + i] = element(from, i);
            else p[address(s, i)] = element(from, i);
        }
    };
    take(in_g, a.gate, a.sgate);
    take(in_x, a.x, a.sx);
    if (BACK) take(in_d, a.dy, a.sdy);
    copies_end();
    copies_wait<0>();
    __syncthreads();
    if (row < a.rows) {
        const int valid = a.lengths ? (int)valid_steps(a, row / a.channels) : steps, mine = threadIdx.x * steps;
        float h = a.state ? a.state[row] : 0.f;
        if (!BACK) {
            for (int k = 0; k < steps; k += 2) {
                // two steps at a time: their gates are pairs
                const int t = REVERSE ? steps - 1 - k : k, u = REVERSE ? t - 1 : t + 1;
                const bool two = k + 1 < steps;
                T& x0 = element(in_x, mine + t);
                T& x1 = element(in_x, mine + (two ? u : t));
                const float v0 = to_float(x0), v1 = to_float(x1);
                Two f, rest;
                gates_of(Two(to_float(element(in_g, mine + t)), to_float(element(in_g, mine + (two ? u : t)))), f, rest);
                if (t < valid) h = fmaf(f.lo(), h, rest.lo() * v0);
                x0 = from_float<T>(t < valid ? h : 0.f);
                if (two) {
                    if (u < valid) h = fmaf(f.hi(), h, rest.hi() * v1);
                    x1 = from_float<T>(u < valid ? h : 0.f);
                }
            }
            if (a.last) a.last[row] = h;
        } else {
            float* starts = reinterpret_cast<float*>(ring + 3 * bytes) + threadIdx.x;     // states at the chunks' starts
            for (int k = 0; k < steps; k += 2) {
                const int t = REVERSE ? steps - 1 - k : k, u = REVERSE ? t - 1 : t + 1;
                const bool two = k + 1 < steps;
                if (k % CHUNK == 0) starts[k / CHUNK * SHORT_ROWS] = h;
                Two f, rest;
                gates_of(Two(to_float(element(in_g, mine + t)), to_float(element(in_g, mine + (two ? u : t)))), f, rest);
                if (t < valid) h = fmaf(f.lo(), h, rest.lo() * to_float(element(in_x, mine + t)));
                if (two && u < valid) h = fmaf(f.hi(), h, rest.hi() * to_float(element(in_x, mine + u)));
            }
            float back = a.dlast ? a.dlast[row] : 0.f;
            for (int k0 = (steps - 1) / CHUNK * CHUNK; k0 >= 0; k0 -= CHUNK) {
                float f[CHUNK], rest[CHUNK], w[CHUNK];
                h = starts[k0 / CHUNK * SHORT_ROWS];
#pragma unroll
                for (int k = 0; k < CHUNK; k += 2) {
                    const int q = k0 + k < steps ? k0 + k : k0, r = q + 1 < steps ? q + 1 : q, t = REVERSE ? steps - 1 - q : q, u = REVERSE ? steps - 1 - r : r;
                    Two f2, rest2;
                    gates_of(Two(to_float(element(in_g, mine + t)), to_float(element(in_g, mine + u))), f2, rest2);
                    f[k] = f2.lo(); f[k + 1] = f2.hi(); rest[k] = rest2.lo(); rest[k + 1] = rest2.hi();
                    const float v0 = to_float(element(in_x, mine + t)), v1 = to_float(element(in_x, mine + u));
                    w[k] = h - v0;
                    if (t < valid) h = fmaf(f[k], h, rest[k] * v0);
                    w[k + 1] = h - v1;
                    if (u < valid) h = fmaf(f[k + 1], h, rest[k + 1] * v1);
                }
#pragma unroll
                for (int k = CHUNK - 1; k >= 0; --k) {
                    if (k0 + k >= steps) continue;
                    const int t = REVERSE ? steps - 1 - (k0 + k) : k0 + k;
                    float ox = 0.f, og = 0.f;
                    if (t < valid) {
                        const float d = back + to_float(element(in_d, mine + t));
                        back = d * f[k];
                        ox = d * rest[k];
                        og = ox * f[k] * w[k];
                    }
                    element(in_x, mine + t) = from_float<T>(ox);
                    element(in_g, mine + t) = from_float<T>(og);
                }
            }
            if (a.dstate) a.dstate[row] = back;
        }
    }
    __syncthreads();
    give(BACK ? a.dx : a.y, BACK ? a.sdx : a.sy, in_x);
    if (BACK) give(a.dg, a.sdg, in_g);
}

// ---- longer chains

constexpr int ROW_WARPS = 4;
template <class T> constexpr int ROW_V = 16 / sizeof(T);
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
template <class T> union Lane { uint4 piece; T e[ROW_V<T>]; __device__ Lane() {} };

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
    // element 0 of tile 0 stands `head` elements before the run; the part's tiles
    const int head = SINGLE ? (int)(row0 * a.steps % V) : 0;
    const long long length = (SINGLE ? 1 : row0 + a.run < a.rows ? a.run : a.rows - row0) * a.steps;
    const long long all_tiles = (length + head + N - 1) / N, each = a.parts > 1 ? a.part / N : all_tiles, tile0 = part * each;
    const long long tiles = tile0 + each < all_tiles ? each : all_tiles - tile0;
    const long long first_saved = (SINGLE ? row0 : w) * run_tiles<T>(a.run, a.steps) + tile0;
    float state = 0.f, total = 1.f;
    if (!MAPS && a.parts > 1) state = a.maps_b[part * a.rows + row0];

    // the lane's element 0 of a tile, counted from the run's first; AGAINST: tiles from the end of memory to its start
    auto element0 = [&](long long k) { return (tile0 + (AGAINST ? tiles - 1 - k : k)) * N + lane * V - head; };
    struct Raw { Lane<T> g, x, d; };
    auto offset = [&](const Strides& s, long long e) {
        const long long r = SINGLE ? 0 : e / a.steps, u = row0 + r, b = u / a.channels;
        return b * s.batch + (u - b * a.channels) * s.channel + (e - r * a.steps) * s.step;
    };
    auto fetch_one = [&](Lane<T>& to, const void* from, const Strides& s, long long e) {
        const T* p = static_cast<const T*>(from);
        if (DENSE && e >= 0 && e + V <= length) {
            to.piece = *reinterpret_cast<const uint4*>(p + (row0 * a.steps + e));
            return;
        }
#pragma unroll
        for (int j = 0; j < V; ++j) to.e[j] = e + j >= 0 && e + j < length ? p[offset(s, e + j)] : from_float<T>(0.f);
    };
    auto fetch = [&](long long k, Raw& raw) {
        const long long e = element0(k);
        fetch_one(raw.g, a.gate, a.sgate, e);
        if (KIND != MAP_VJP) fetch_one(raw.x, a.x, a.sx, e);
        if (BACK) fetch_one(raw.d, a.dy, a.sdy, e);
    };
    auto store = [&](void* to, const Strides& s, long long e, const float (&v)[V]) {
        T* p = static_cast<T*>(to);
        if (DENSE && e >= 0 && e + V <= length) {
            Lane<T> u;
#pragma unroll
            for (int j = 0; j < V; j += 2) round_pair(u.e + j, Two(v[j], v[j + 1]));
            *reinterpret_cast<uint4*>(p + (row0 * a.steps + e)) = u.piece;
            return;
        }
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (e + j >= 0 && e + j < length) p[offset(s, e + j)] = from_float<T>(v[j]);
    };

    Raw next;
    if (tiles > 0) fetch(0, next);
    for (long long k = 0; k < tiles; ++k) {
        const Raw raw = next;
        if (k + 1 < tiles) fetch(k + 1, next);
        const long long e = element0(k);
        // the chain of element 0 and where the next one begins; elements that are there
        long long row = row0, step = e;
        if (!SINGLE && e > 0) {
            const long long r = length < (1ll << 32) ? (uint32_t)e / (uint32_t)a.steps : e / a.steps;
            row += r; step -= r * a.steps;
        }
        const int border = a.steps - step < V ? (int)(a.steps - step) : V;           // element where the next chain begins
        uint32_t there = (1u << V) - 1;
        if (e < 0) there = e <= -V ? 0 : there << (int)-e & there;
        if (e + V > length) there = e >= length ? 0 : there & ((1u << (int)(length - e)) - 1);
        uint32_t valid = there;
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
        uint32_t low = step <= 0 && step > -V ? 1u << (int)-step : 0, high = border <= V && border > 0 && a.steps - step <= V ? 1u << (border - 1) : 0;
        if (!SINGLE && border < V) low |= 1u << border;
        low &= there; high &= there;
        const uint32_t first = REVERSE ? high : low, last = REVERSE ? low : high;
        auto row_of = [&](int j) { return SINGLE || j < border ? row : row + 1; };

        float f[V], rest[V], x[V], d[V], h[V];                                       // h: forward h_t; VJP h_(t-1)
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            Two f2, rest2;
            gates_of(pair_of(raw.g.e + j), f2, rest2);
            f[j] = f2.lo(); f[j + 1] = f2.hi(); rest[j] = rest2.lo(); rest[j + 1] = rest2.hi();
            if (KIND != MAP_VJP) { const Two v = pair_of(raw.x.e + j); x[j] = v.lo(); x[j + 1] = v.hi(); }
            if (BACK) { const Two v = pair_of(raw.d.e + j); d[j] = v.lo(); d[j + 1] = v.hi(); }
        }
        if (valid != (1u << V) - 1) {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (!(valid >> j & 1)) { f[j] = 1.f; rest[j] = 0.f; x[j] = 0.f; d[j] = 0.f; }
        }
        if (KIND != MAP_VJP) {
            // the lane's own steps from a state of zero, then the state before them
            Map own{1.f, 0.f}, all;
            float enters = 0.f;
            const bool begins = !MAPS && first;
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
                        if (last >> j & 1 && a.last) a.last[row_of(j)] = s;
                    }
                }
                if (KIND == FORWARD) state = apply(all, state);
            }
        }
        if (KIND == FORWARD) {
            if (valid != there) {
#pragma unroll
                for (int j = 0; j < V; ++j) if (!(valid >> j & 1)) h[j] = 0.f;
            }
            store(a.y, a.sy, e, h);
        }
        if (BACK) {
            Map own{1.f, 0.f}, all;
            float enters = 0.f;
            const bool begins = !MAPS && last;
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
                    if (first >> j & 1 && a.dstate) a.dstate[row_of(j)] = s;
                }
                state = apply(all, state);
                if (valid != there) {
#pragma unroll
                    for (int j = 0; j < V; ++j) if (!(valid >> j & 1)) ox[j] = og[j] = 0.f;
                }
                store(a.dx, a.sdx, e, ox);
                store(a.dg, a.sdg, e, og);
            }
        }
    }
    if (MAPS && lane == 0) {
        a.maps_a[part * a.rows + row0] = total;
        a.maps_b[part * a.rows + row0] = state;
    }
}

}  // namespace scan
}  // namespace gleam
