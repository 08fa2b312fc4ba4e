// The gated recurrence where rows of neighbouring chains are narrow (a few features or voxels between the steps): a thread runs one
// chain with loads into registers.  And single steps.
#pragma once
#include "scan_stream.cuh"

namespace gleam {
namespace scan {

constexpr int COLUMN_THREADS = 128;

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
template <class T, bool REVERSE, bool MAPS>
__global__ void __launch_bounds__(COLUMN_THREADS) columns_forward(const __grid_constant__ Args a) {
    grid_dependency_wait();
    Columns c{};
    c.find<1>(a, (long long)blockIdx.x * COLUMN_THREADS + threadIdx.x);
    if (!c.there) return;
    const T* x = c.at(static_cast<const T*>(a.x), a.sx);
    const T* gate = c.at(static_cast<const T*>(a.gate), a.sgate);
    T* y = MAPS ? nullptr : c.at(static_cast<T*>(a.y), a.sy);
    const long long valid = valid_steps(a, c.batch), steps = a.steps, part = blockIdx.y;
    const long long begin = part * a.part, end = begin + a.part < steps ? begin + a.part : steps;
    float h = 0.f, prod = 1.f;
    if (!MAPS && a.parts > 1) h = a.maps_b[part * a.rows + c.row];
    else if (!MAPS && a.state) h = a.state[c.row];
    for (long long q0 = begin; q0 < end; q0 += a.chunk) {
        const int count = (int)(q0 + a.chunk < end ? a.chunk : end - q0);
        T xs[CHUNK], gs[CHUNK];
#pragma unroll
        for (int k = 0; k < CHUNK; ++k) {
            const long long t = REVERSE ? steps - 1 - (q0 + k) : q0 + k;
            if (k < count && t < valid) { xs[k] = x[t * a.sx.step]; gs[k] = gate[t * a.sgate.step]; }
        }
        if (!MAPS && a.saved && q0 > 0) a.saved[(q0 / a.chunk - 1) * a.rows + c.row] = h;
#pragma unroll
        for (int k = 0; k < CHUNK; ++k) {
            const long long t = REVERSE ? steps - 1 - (q0 + k) : q0 + k;
            if (k >= count) break;
            float out = 0.f;
            if (t < valid) {
                float f, rest;
                gate_of<T>(to_float(gs[k]), f, rest);
                out = h = fmaf(f, h, rest * to_float(xs[k]));
                prod *= f;
            }
            if (!MAPS) y[t * a.sy.step] = from_float<T>(out);
        }
    }
    if (MAPS) {
        a.maps_a[part * a.rows + c.row] = prod;
        a.maps_b[part * a.rows + c.row] = h;
    } else if (a.last && end == steps) {
        a.last[c.row] = h;
    }
}

// VJP, and the maps of parts for it: part p covers the same positions as in the forward call, taken from its end.
template <class T, bool REVERSE, bool MAPS>
__global__ void __launch_bounds__(COLUMN_THREADS) columns_vjp(const __grid_constant__ Args a) {
    grid_dependency_wait();
    Columns c{};
    c.find<1>(a, (long long)blockIdx.x * COLUMN_THREADS + threadIdx.x);
    if (!c.there) return;
    const T* x = MAPS ? nullptr : c.at(static_cast<const T*>(a.x), a.sx);
    const T* gate = c.at(static_cast<const T*>(a.gate), a.sgate);
    const T* dy = c.at(static_cast<const T*>(a.dy), a.sdy);
    T* dx = MAPS ? nullptr : c.at(static_cast<T*>(a.dx), a.sdx);
    T* dg = MAPS ? nullptr : c.at(static_cast<T*>(a.dg), a.sdg);
    const long long valid = valid_steps(a, c.batch), steps = a.steps, part = blockIdx.y;
    const long long begin = part * a.part, end = begin + a.part < steps ? begin + a.part : steps;
    float back = 0.f, prod = 1.f;
    if (!MAPS && a.parts > 1) back = a.maps_b[part * a.rows + c.row];
    else if (!MAPS && a.dlast) back = a.dlast[c.row];
    for (long long q0 = begin + (end - begin - 1) / a.chunk * a.chunk; q0 >= begin; q0 -= a.chunk) {
        const int count = (int)(q0 + a.chunk < end ? a.chunk : end - q0);
        T xs[CHUNK], gs[CHUNK], ds[CHUNK];
#pragma unroll
        for (int k = 0; k < CHUNK; ++k) {
            const long long t = REVERSE ? steps - 1 - (q0 + k) : q0 + k;
            if (k < count && t < valid) {
                gs[k] = gate[t * a.sgate.step]; ds[k] = dy[t * a.sdy.step];
                if (!MAPS) xs[k] = x[t * a.sx.step];
            }
        }
        float f[CHUNK], rest[CHUNK], w[CHUNK], h = 0.f;                  // w: h_(t-1) - x_t
        if (!MAPS) h = q0 > 0 ? a.saved[(q0 / a.chunk - 1) * a.rows + c.row] : a.state ? a.state[c.row] : 0.f;
#pragma unroll
        for (int k = 0; k < CHUNK; ++k) {
            const long long t = REVERSE ? steps - 1 - (q0 + k) : q0 + k;
            if (k < count && t < valid) {
                gate_of<T>(to_float(gs[k]), f[k], rest[k]);
                if (!MAPS) {
                    const float u = to_float(xs[k]);
                    w[k] = h - u;
                    h = fmaf(f[k], h, rest[k] * u);
                }
            }
        }
#pragma unroll
        for (int k = CHUNK - 1; k >= 0; --k) {
            if (k >= count) continue;
            const long long t = REVERSE ? steps - 1 - (q0 + k) : q0 + k;
            float ox = 0.f, og = 0.f;
            if (t < valid) {
                const float d = back + to_float(ds[k]);
                back = d * f[k];
                prod *= f[k];
                if (!MAPS) { ox = d * rest[k]; og = ox * f[k] * w[k]; }
            }
            if (!MAPS) {
                dx[t * a.sdx.step] = from_float<T>(ox);
                dg[t * a.sdg.step] = from_float<T>(og);
            }
        }
    }
    if (MAPS) {
        a.maps_a[part * a.rows + c.row] = prod;
        a.maps_b[part * a.rows + c.row] = back;
    } else if (a.dstate && begin == 0) {
        a.dstate[c.row] = back;
    }
}

// One step with the states updated in place.
template <class T, int V>
__global__ void __launch_bounds__(COLUMN_THREADS) step_kernel(const __grid_constant__ Args a) {
    grid_dependency_wait();
    Columns c{};
    c.find<V>(a, (long long)blockIdx.x * COLUMN_THREADS + threadIdx.x);
    if (!c.there) return;
    const Piece<T, V> x = *reinterpret_cast<const Piece<T, V>*>(c.at(static_cast<const T*>(a.x), a.sx));
    const Piece<T, V> gate = *reinterpret_cast<const Piece<T, V>*>(c.at(static_cast<const T*>(a.gate), a.sgate));
    Piece<float, V> h = *reinterpret_cast<const Piece<float, V>*>(a.last + c.row);
    Piece<T, V> out;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        float f, rest;
        gate_of<T>(to_float(gate.e[j]), f, rest);
        h.e[j] = fmaf(f, h.e[j], rest * to_float(x.e[j]));
        out.e[j] = from_float<T>(h.e[j]);
    }
    *reinterpret_cast<Piece<float, V>*>(a.last + c.row) = h;
    *reinterpret_cast<Piece<T, V>*>(c.at(static_cast<T*>(a.y), a.sy)) = out;
}

}  // namespace scan
}  // namespace gleam
