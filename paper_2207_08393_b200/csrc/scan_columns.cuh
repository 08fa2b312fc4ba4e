// The gated recurrence where the chains lie side by side in memory (inner > 1): a thread runs V neighbouring chains.
#pragma once
#include "scan_common.cuh"

namespace gleam {
namespace scan {

constexpr int COLUMN_THREADS = 128;
constexpr int CHUNK = 16;                  // steps whose loads a thread has under way, and between saved states

// steps of a chunk: as few chunks as CHUNK allows, all alike
inline int chunk_steps(long long steps) {
    const long long n = (steps + CHUNK - 1) / CHUNK;
    return n < 1 ? 1 : (int)((steps + n - 1) / n);
}

template <class T, int V> struct alignas(V * sizeof(T)) Piece { T e[V]; };

template <class T, int V>
__device__ __forceinline__ Piece<T, V> load_piece(const T* p) { return *reinterpret_cast<const Piece<T, V>*>(p); }
template <class T, int V>
__device__ __forceinline__ void store_piece(T* p, const Piece<T, V>& v) { *reinterpret_cast<Piece<T, V>*>(p) = v; }
// V states; V > 1 only where their array starts at V * 4 bytes
template <int V>
__device__ __forceinline__ void load_states(const float* p, float (&v)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = 0.f;
    if (!p) return;
    const Piece<float, V> u = load_piece<float, V>(p);
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = u.e[j];
}
template <int V>
__device__ __forceinline__ void store_states(float* p, const float (&v)[V]) {
    Piece<float, V> u;
#pragma unroll
    for (int j = 0; j < V; ++j) u.e[j] = v[j];
    store_piece<float, V>(p, u);
}

// A thread's V chains.
struct Columns {
    long long batch, channel, i, row;
    bool there;
    template <int V> __device__ __forceinline__ void find(const Args& a, long long index) {
        row = index * V;
        there = row < a.rows;
        if (!there) return;
        if (a.rows < (1ll << 32)) {
            const uint32_t n = (uint32_t)a.inner, c = (uint32_t)a.channels, u = (uint32_t)row / n;
            i = (uint32_t)row - u * n; batch = u / c; channel = u - (uint32_t)batch * c;
        } else {
            const long long u = row / a.inner;
            i = row - u * a.inner; batch = u / a.channels; channel = u - batch * a.channels;
        }
    }
    template <class P> __device__ __forceinline__ P* at(P* base, const Strides& s) const { return base + (batch * s.batch + channel * s.channel + i); }
};

// Forward, and the maps of parts for it.  Position q = 0, 1, ... of a chain is step q or T - 1 - q.
template <class T, int V, bool REVERSE, bool MAPS>
__global__ void __launch_bounds__(COLUMN_THREADS) columns_forward(const __grid_constant__ Args a) {
    grid_dependency_wait();
    Columns c{};
    c.find<V>(a, (long long)blockIdx.x * COLUMN_THREADS + threadIdx.x);
    if (!c.there) return;
    const T* x = c.at(static_cast<const T*>(a.x), a.sx);
    const T* gate = c.at(static_cast<const T*>(a.gate), a.sgate);
    T* y = MAPS ? nullptr : c.at(static_cast<T*>(a.y), a.sy);
    const long long valid = valid_steps(a, c.batch), steps = a.steps, part = blockIdx.y;
    const long long begin = part * a.part, end = begin + a.part < steps ? begin + a.part : steps;
    float h[V], prod[V];
    if (MAPS) {
#pragma unroll
        for (int j = 0; j < V; ++j) { h[j] = 0.f; prod[j] = 1.f; }
    } else if (a.parts > 1) {
        load_states(a.maps_b + (part * a.rows + c.row), h);
    } else {
        load_states(a.state ? a.state + c.row : nullptr, h);
    }
    for (long long q0 = begin; q0 < end; q0 += a.chunk) {
        const int count = (int)(q0 + a.chunk < end ? a.chunk : end - q0);
        Piece<T, V> xs[CHUNK], gs[CHUNK];
#pragma unroll
        for (int k = 0; k < CHUNK; ++k) {
            const long long t = REVERSE ? steps - 1 - (q0 + k) : q0 + k;
            if (k < count && t < valid) {
                xs[k] = load_piece<T, V>(x + t * a.sx.step);
                gs[k] = load_piece<T, V>(gate + t * a.sgate.step);
            }
        }
        if (!MAPS && a.saved && q0 > 0) store_states(a.saved + ((q0 / a.chunk - 1) * a.rows + c.row), h);
#pragma unroll
        for (int k = 0; k < CHUNK; ++k) {
            const long long t = REVERSE ? steps - 1 - (q0 + k) : q0 + k;
            if (k >= count) break;
            Piece<T, V> out;
            if (t < valid) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float f, rest;
                    gate_of(to_float(gs[k].e[j]), f, rest);
                    h[j] = fmaf(f, h[j], rest * to_float(xs[k].e[j]));
                    if (MAPS) prod[j] *= f;
                    else out.e[j] = from_float<T>(h[j]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) out.e[j] = from_float<T>(0.f);
            }
            if (!MAPS) store_piece<T, V>(y + t * a.sy.step, out);
        }
    }
    if (MAPS) {
        store_states(a.maps_a + (part * a.rows + c.row), prod);
        store_states(a.maps_b + (part * a.rows + c.row), h);
    } else if (a.last && end == steps) {
        store_states(a.last + c.row, h);
    }
}

// VJP, and the maps of parts for it: part p covers the same positions as in the forward call, taken from its end.
template <class T, int V, bool REVERSE, bool MAPS>
__global__ void __launch_bounds__(COLUMN_THREADS) columns_vjp(const __grid_constant__ Args a) {
    grid_dependency_wait();
    Columns c{};
    c.find<V>(a, (long long)blockIdx.x * COLUMN_THREADS + threadIdx.x);
    if (!c.there) return;
    const T* x = MAPS ? nullptr : c.at(static_cast<const T*>(a.x), a.sx);
    const T* gate = c.at(static_cast<const T*>(a.gate), a.sgate);
    const T* dy = c.at(static_cast<const T*>(a.dy), a.sdy);
    T* dx = MAPS ? nullptr : c.at(static_cast<T*>(a.dx), a.sdx);
    T* dg = MAPS ? nullptr : c.at(static_cast<T*>(a.dg), a.sdg);
    const long long valid = valid_steps(a, c.batch), steps = a.steps, part = blockIdx.y;
    const long long begin = part * a.part, end = begin + a.part < steps ? begin + a.part : steps;
    float back[V], prod[V];
    if (MAPS) {
#pragma unroll
        for (int j = 0; j < V; ++j) { back[j] = 0.f; prod[j] = 1.f; }
    } else if (a.parts > 1) {
        load_states(a.maps_b + (part * a.rows + c.row), back);
    } else {
        load_states(a.dlast ? a.dlast + c.row : nullptr, back);
    }
    for (long long q0 = begin + (end - begin - 1) / a.chunk * a.chunk; q0 >= begin; q0 -= a.chunk) {
        const int count = (int)(q0 + a.chunk < end ? a.chunk : end - q0);
        Piece<T, V> xs[CHUNK], gs[CHUNK], ds[CHUNK];
#pragma unroll
        for (int k = 0; k < CHUNK; ++k) {
            const long long t = REVERSE ? steps - 1 - (q0 + k) : q0 + k;
            if (k < count && t < valid) {
                gs[k] = load_piece<T, V>(gate + t * a.sgate.step);
                ds[k] = load_piece<T, V>(dy + t * a.sdy.step);
                if (!MAPS) xs[k] = load_piece<T, V>(x + t * a.sx.step);
            }
        }
        float before[CHUNK][V];
        if (!MAPS) {
            float h[V];
            load_states(q0 > 0 ? a.saved + ((q0 / a.chunk - 1) * a.rows + c.row) : a.state ? a.state + c.row : nullptr, h);
#pragma unroll
            for (int k = 0; k < CHUNK; ++k) {
                const long long t = REVERSE ? steps - 1 - (q0 + k) : q0 + k;
                if (k < count && t < valid) {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        float f, rest;
                        before[k][j] = h[j];
                        gate_of(to_float(gs[k].e[j]), f, rest);
                        h[j] = fmaf(f, h[j], rest * to_float(xs[k].e[j]));
                    }
                }
            }
        }
#pragma unroll
        for (int k = CHUNK - 1; k >= 0; --k) {
            if (k >= count) continue;
            const long long t = REVERSE ? steps - 1 - (q0 + k) : q0 + k;
            Piece<T, V> ox, og;
            if (t < valid) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float f, rest;
                    gate_of(to_float(gs[k].e[j]), f, rest);
                    const float d = back[j] + to_float(ds[k].e[j]);
                    back[j] = d * f;
                    if (MAPS) { prod[j] *= f; continue; }
                    const float e = d * rest;
                    ox.e[j] = from_float<T>(e);
                    og.e[j] = from_float<T>(e * f * (before[k][j] - to_float(xs[k].e[j])));
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) { ox.e[j] = from_float<T>(0.f); og.e[j] = from_float<T>(0.f); }
            }
            if (!MAPS) {
                store_piece<T, V>(dx + t * a.sdx.step, ox);
                store_piece<T, V>(dg + t * a.sdg.step, og);
            }
        }
    }
    if (MAPS) {
        store_states(a.maps_a + (part * a.rows + c.row), prod);
        store_states(a.maps_b + (part * a.rows + c.row), back);
    } else if (a.dstate && begin == 0) {
        store_states(a.dstate + c.row, back);
    }
}

// The parts' maps joined: maps_b becomes the state that each part starts from.  A thread runs one chain.
template <int AHEAD>
__global__ void __launch_bounds__(COLUMN_THREADS) join_parts(const __grid_constant__ Args a) {
    grid_dependency_wait();
    const long long row = (long long)blockIdx.x * COLUMN_THREADS + threadIdx.x;
    if (row >= a.rows) return;
    float s = a.enter ? a.enter[row] : 0.f;
    const long long step = a.descending ? -a.rows : a.rows;
    long long at = (a.descending ? (a.parts - 1) * a.rows : 0) + row;
    for (int p0 = 0; p0 < a.parts; p0 += AHEAD, at += AHEAD * step) {
        float fa[AHEAD], fb[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (p0 + k < a.parts) { fa[k] = a.maps_a[at + k * step]; fb[k] = a.maps_b[at + k * step]; }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (p0 + k < a.parts) { a.maps_b[at + k * step] = s; s = fmaf(fa[k], s, fb[k]); }
    }
}

// One step with the states updated in place.
template <class T, int V>
__global__ void __launch_bounds__(COLUMN_THREADS) step_kernel(const __grid_constant__ Args a) {
    grid_dependency_wait();
    Columns c{};
    c.find<V>(a, (long long)blockIdx.x * COLUMN_THREADS + threadIdx.x);
    if (!c.there) return;
    const Piece<T, V> x = load_piece<T, V>(c.at(static_cast<const T*>(a.x), a.sx));
    const Piece<T, V> gate = load_piece<T, V>(c.at(static_cast<const T*>(a.gate), a.sgate));
    float h[V];
    load_states(a.last + c.row, h);
    Piece<T, V> out;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        float f, rest;
        gate_of(to_float(gate.e[j]), f, rest);
        h[j] = fmaf(f, h[j], rest * to_float(x.e[j]));
        out.e[j] = from_float<T>(h[j]);
    }
    store_states(a.last + c.row, h);
    store_piece<T, V>(c.at(static_cast<T*>(a.y), a.sy), out);
}

}  // namespace scan
}  // namespace gleam
