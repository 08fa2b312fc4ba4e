// The gated recurrence where a chain's steps lie one behind the other (inner = 1).
//
// A warp takes a run of whole chains, or a part of one, in tiles of 32 lanes with V neighbouring steps each.  A lane composes the
// maps of its own steps, the lanes' maps are composed by shuffles (five turns), and the state behind the tile goes on to the next
// one.  Where a chain begins inside a tile its map forgets what came before (FORGETS for a), so chains of any length share tiles.
#pragma once
#include "scan_common.cuh"

namespace gleam {
namespace scan {

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

// Where a lane's V elements lie: element j of the run is step (first_step + j) of chain first_row, or of a later one.
struct Place {
    long long row, step;
    __device__ __forceinline__ void next(long long steps) { if (++step == steps) { step = 0; ++row; } }
};

template <class T> __device__ __forceinline__ long long offset_of(const Args& a, const Strides& s, const Place& p) {
    const long long b = a.rows < (1ll << 32) ? (uint32_t)p.row / (uint32_t)a.channels : p.row / a.channels;
    return b * s.batch + (p.row - b * a.channels) * s.channel + p.step * s.step;
}

// A warp's run: elements [begin, end) of the chains from `row` on, end counted from their first step.
struct Run {
    long long row, begin, end, tiles, saved;       // saved: index of the state at the first tile's start
};
template <class T>
__device__ __forceinline__ bool find_run(const Args& a, Run& r) {
    constexpr int N = TILE<T>;
    const long long w = (long long)blockIdx.x * ROW_WARPS + (threadIdx.x >> 5);
    const long long per_run = (a.run * a.steps + N - 1) / N;       // tiles
    if (a.run > 1) {
        r.row = w * a.run;
        if (r.row >= a.rows) return false;
        const long long rows = r.row + a.run < a.rows ? a.run : a.rows - r.row;
        r.begin = 0; r.end = rows * a.steps;
        r.saved = w * per_run;
    } else {
        const long long p = w % a.parts;
        r.row = w / a.parts;
        if (r.row >= a.rows) return false;
        r.begin = p * a.part;
        r.end = r.begin + a.part < a.steps ? r.begin + a.part : a.steps;
        r.saved = r.row * per_run + r.begin / N;
    }
    r.tiles = (r.end - r.begin + N - 1) / N;
    return true;
}

template <class T> struct Lane { float v[ROW_V<T>]; };

// A lane's elements of one array as numbers.  DENSE: the array has no gaps and its runs start at 16 bytes.
template <class T, bool DENSE>
__device__ __forceinline__ void load_lane(const Args& a, const void* base, const Strides& s, const Place& at, int count, Lane<T>& out) {
    constexpr int V = ROW_V<T>;
    const T* p = static_cast<const T*>(base);
    if (DENSE && count == V) {
        const Pack<T> u = prior::load_pack(p + (at.row * a.steps + at.step));
#pragma unroll
        for (int j = 0; j < V; ++j) out.v[j] = to_float(u.e[j]);
        return;
    }
    Place q = at;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        out.v[j] = j < count ? to_float(p[offset_of<T>(a, s, q)]) : 0.f;
        q.next(a.steps);
    }
}
template <class T, bool DENSE>
__device__ __forceinline__ void store_lane(const Args& a, void* base, const Strides& s, const Place& at, int count, const Lane<T>& in) {
    constexpr int V = ROW_V<T>;
    T* p = static_cast<T*>(base);
    if (DENSE && count == V) {
        Pack<T> u;
#pragma unroll
        for (int j = 0; j < V; ++j) u.e[j] = from_float<T>(in.v[j]);
        prior::store_pack(p + (at.row * a.steps + at.step), u);
        return;
    }
    Place q = at;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        if (j < count) p[offset_of<T>(a, s, q)] = from_float<T>(in.v[j]);
        q.next(a.steps);
    }
}

// What the steps of a lane's elements are: inside their example's length, first or last of their chain in the order of the chain.
struct Marks { uint32_t valid, first, last; };
template <class T, bool REVERSE>
__device__ __forceinline__ Marks marks_of(const Args& a, const Place& at, int count) {
    Marks m{0, 0, 0};
    Place q = at;
#pragma unroll
    for (int j = 0; j < ROW_V<T>; ++j) {
        if (j < count) {
            if (!a.lengths || q.step < valid_steps(a, q.row / a.channels)) m.valid |= 1u << j;
            if (q.step == 0) (REVERSE ? m.last : m.first) |= 1u << j;
            if (q.step == a.steps - 1) (REVERSE ? m.first : m.last) |= 1u << j;
        }
        q.next(a.steps);
    }
    return m;
}
__device__ __forceinline__ long long row_at(const Args& a, const Place& at, int j) { return at.step + j < a.steps ? at.row : at.row + (at.step + j) / a.steps; }

// Elements in the order of the chain: k = 0 first.
template <class T, bool REVERSE> __device__ __forceinline__ constexpr int ordered(int k) { return REVERSE ? ROW_V<T> - 1 - k : k; }

template <class T, bool REVERSE, bool DENSE, int KIND>
__global__ void __launch_bounds__(ROW_WARPS * 32) rows_kernel(const __grid_constant__ Args a) {
    grid_dependency_wait();
    constexpr int V = ROW_V<T>, N = TILE<T>;
    constexpr bool MAPS = KIND == MAP_FORWARD || KIND == MAP_VJP, BACK = KIND == VJP || KIND == MAP_VJP, AGAINST = BACK != REVERSE;
    Run r;
    if (!find_run<T>(a, r)) return;
    const int lane = threadIdx.x & 31;
    const long long part = a.run > 1 ? 0 : r.begin / a.part;
    // AGAINST: tiles from the end of memory to its start
    float state = 0.f, total = 1.f;
    if (!MAPS && a.parts > 1) state = a.maps_b[part * a.rows + r.row];
    for (long long k = 0; k < r.tiles; ++k) {
        const long long tile = AGAINST ? r.tiles - 1 - k : k, e = r.begin + tile * N + lane * V;
        const long long left = r.end - e;
        const int count = left >= V ? V : left > 0 ? (int)left : 0;
        Place at{r.row, e};
        if (e >= a.steps) {
            const long long n = a.rows * a.steps < (1ll << 32) ? (uint32_t)e / (uint32_t)a.steps : e / a.steps;
            at.row += n; at.step -= n * a.steps;
        }
        const Marks m = marks_of<T, REVERSE>(a, at, count);
        const bool dense = DENSE && m.valid == (1u << V) - 1;       // what is not valid is not read
        Lane<T> g, x, d;
        auto load = [&](const void* base, const Strides& s, Lane<T>& to) {
            if (dense || m.valid == 0) { load_lane<T, DENSE>(a, base, s, at, dense ? V : 0, to); return; }
            Place q = at;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                to.v[j] = m.valid >> j & 1 ? to_float(static_cast<const T*>(base)[offset_of<T>(a, s, q)]) : 0.f;
                q.next(a.steps);
            }
        };
        load(a.gate, a.sgate, g);
        if (KIND != MAP_VJP) load(a.x, a.sx, x);
        if (BACK) load(a.dy, a.sdy, d);
        Lane<T> f, rest;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (m.valid >> j & 1) gate_of(g.v[j], f.v[j], rest.v[j]);
            else { f.v[j] = 1.f; rest.v[j] = 0.f; }
        }
        Lane<T> h;                                                   // forward: h_t; VJP: h_(t-1)
        if (KIND != MAP_VJP) {
            // the lane's own steps from a state of zero, then the state before them
            Map own{1.f, 0.f}, all;
#pragma unroll
            for (int k2 = 0; k2 < V; ++k2) {
                const int j = ordered<T, REVERSE>(k2);
                if (!MAPS && m.first >> j & 1) own = Map{FORGETS, a.state ? a.state[row_at(a, at, j)] : 0.f};
                own = then(own, Map{f.v[j], rest.v[j] * x.v[j]});
            }
            const Map pre = before_lane<!REVERSE>(own, &all);
            if (MAPS) {
                state = apply(all, state); total *= all.a;
            } else {
                float enter = state;
                if (KIND == VJP) enter = a.saved[r.saved + tile];
                else if (a.saved && lane == 0) a.saved[r.saved + tile] = state;
                float s = apply(pre, enter);
#pragma unroll
                for (int k2 = 0; k2 < V; ++k2) {
                    const int j = ordered<T, REVERSE>(k2);
                    if (m.first >> j & 1) s = a.state ? a.state[row_at(a, at, j)] : 0.f;
                    if (KIND == VJP) h.v[j] = s;
                    s = fmaf(f.v[j], s, rest.v[j] * x.v[j]);
                    if (KIND == FORWARD) {
                        h.v[j] = m.valid >> j & 1 ? s : 0.f;
                        if (a.last && m.last >> j & 1) a.last[row_at(a, at, j)] = s;
                    }
                }
                if (KIND == FORWARD) state = apply(all, state);
            }
        }
        if (KIND == FORWARD) store_lane<T, DENSE>(a, a.y, a.sy, at, count, h);
        if (BACK) {
            Map own{1.f, 0.f}, all;
#pragma unroll
            for (int k2 = V - 1; k2 >= 0; --k2) {
                const int j = ordered<T, REVERSE>(k2);
                if (!MAPS && m.last >> j & 1) own = Map{FORGETS, a.dlast ? a.dlast[row_at(a, at, j)] : 0.f};
                own = then(own, Map{f.v[j], f.v[j] * d.v[j]});
            }
            const Map pre = before_lane<REVERSE>(own, &all);
            if (MAPS) {
                state = apply(all, state); total *= all.a;
            } else {
                float s = apply(pre, state);
                Lane<T> ox, og;
#pragma unroll
                for (int k2 = V - 1; k2 >= 0; --k2) {
                    const int j = ordered<T, REVERSE>(k2);
                    if (m.last >> j & 1) s = a.dlast ? a.dlast[row_at(a, at, j)] : 0.f;
                    const float c = s + d.v[j], w = c * rest.v[j];
                    ox.v[j] = w;
                    og.v[j] = m.valid >> j & 1 ? w * f.v[j] * (h.v[j] - x.v[j]) : 0.f;
                    s = f.v[j] * c;
                    if (a.dstate && m.first >> j & 1) a.dstate[row_at(a, at, j)] = s;
                }
                state = apply(all, state);
                store_lane<T, DENSE>(a, a.dx, a.sdx, at, count, ox);
                store_lane<T, DENSE>(a, a.dg, a.sdg, at, count, og);
            }
        }
    }
    if (MAPS && lane == 0) {
        a.maps_a[part * a.rows + r.row] = total;
        a.maps_b[part * a.rows + r.row] = state;
    }
}

}  // namespace scan
}  // namespace gleam
