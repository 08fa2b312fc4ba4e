// The gated recurrence where the chains lie side by side in memory and a row of them is wide enough for a block: arrays come through
// shared memory by asynchronous copies, several steps ahead of their use.
//
// What bounds it is memory; what it takes is bytes under way (about 40 KB an SM) that cost no registers, and enough warps that the
// chains' arithmetic (some 12 instructions an element forward, 25 for the VJP) hides behind them.  Two forms:
//   private   every row of every array starts at a multiple of a thread's piece (16 or 8 bytes): a thread copies, reads and stores its
//             own V neighbouring chains, and no thread waits for another;
//   strips    rows start anywhere (an odd number of voxels): a block copies the 16-byte pieces that its strip of a row touches and reads
//             from them element by element, lanes side by side; a thread's V chains are a block's width apart.
// 60 x 20 x 30720 float32, forward and VJP: 293 us with loads into registers, <<PRIVATE>>.
#pragma once
#include "scan_common.cuh"

namespace gleam {
namespace scan {

constexpr int STREAM_THREADS = 128;
constexpr int CHUNK = 8;                   // steps between saved states: what a VJP holds at a time
constexpr int BATCH = 4, DEPTH = 4;        // steps of a copy group, and groups of the ring (forward)

// steps of a chunk: as few chunks as CHUNK allows, all alike
inline int chunk_steps(long long steps) {
    const long long n = (steps + CHUNK - 1) / CHUNK;
    return n < 1 ? 1 : (int)((steps + n - 1) / n);
}

template <class T, int V> struct alignas(V * sizeof(T)) Piece { T e[V]; };

template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t to, const void* from) {
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// The chains of a block and a thread, and how rows of them pass through shared memory.
template <class T, int V, bool STRIP>
struct Rows {
    static constexpr int BYTES = V * sizeof(T), WIDTH = STREAM_THREADS * V;
    static constexpr int SLOT = STREAM_THREADS * BYTES + (STRIP ? 16 : 0);       // bytes of a row in shared memory
    long long row, batch;                    // the thread's first chain, its example
    long long at_batch, at_channel, at_i;    // ... (strips: the block's first chain)
    int there;                               // chains of the strip; private: whether there are any

    __device__ __forceinline__ void find(const Args& a) {
        if (STRIP) {
            const long long strips = (a.inner + WIDTH - 1) / WIDTH, u = blockIdx.x / strips, first = (blockIdx.x - u * strips) * WIDTH;
            at_batch = u / a.channels; at_channel = u - at_batch * a.channels; at_i = first;
            there = (int)(a.inner - first < WIDTH ? a.inner - first : WIDTH);
            row = u * a.inner + first + threadIdx.x;
        } else {
            row = ((long long)blockIdx.x * STREAM_THREADS + threadIdx.x) * V;
            there = row < a.rows;
            if (a.rows < (1ll << 32)) {
                const uint32_t n = (uint32_t)a.inner, c = (uint32_t)a.channels, u = (uint32_t)row / n;
                at_i = (uint32_t)row - u * n; at_batch = u / c; at_channel = u - (uint32_t)at_batch * c;
            } else {
                const long long u = row / a.inner;
                at_i = row - u * a.inner; at_batch = u / a.channels; at_channel = u - at_batch * a.channels;
            }
        }
        batch = at_batch;
    }
    template <class P> __device__ __forceinline__ P* at(P* base, const Strides& s) const { return base + (at_batch * s.batch + at_channel * s.channel + at_i); }
    __device__ __forceinline__ bool has(int j) const { return STRIP ? (int)threadIdx.x + j * STREAM_THREADS < there : true; }

    // private: the thread's piece of a row
    __device__ __forceinline__ void copy(uint32_t slot, const T* from) const { copy_async<BYTES>(slot + threadIdx.x * BYTES, from); }
    // strips: piece p of those that the strip touches; what is not inside the row as a whole goes element by element
    __device__ __forceinline__ static int pieces() { return (WIDTH * (int)sizeof(T) + 15) / 16 + 1; }
    __device__ __forceinline__ void copy_piece(const Args& a, unsigned char* slot, const T* from, int p) const {
        const uintptr_t first = (uintptr_t)from, begin = first - at_i * sizeof(T), end = begin + a.inner * sizeof(T), stop = first + there * sizeof(T);
        const uintptr_t x = (first & ~(uintptr_t)15) + 16 * p;
        if (x >= stop) return;
        if (x >= begin && x + 16 <= end) {
            copy_async<16>((uint32_t)__cvta_generic_to_shared(slot) + 16 * p, (const void*)x);
            return;
        }
        for (int e = 0; e < 16; e += sizeof(T))
            if (x + e >= first && x + e < stop) *reinterpret_cast<T*>(slot + 16 * p + e) = *reinterpret_cast<const T*>(x + e);
    }
    __device__ __forceinline__ void read(const unsigned char* slot, const T* from, float (&v)[V]) const {
        if (STRIP) {
            const T* s = reinterpret_cast<const T*>(slot + ((uintptr_t)from & 15)) + threadIdx.x;
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = to_float(s[j * STREAM_THREADS]);
        } else {
            const Piece<T, V> p = *reinterpret_cast<const Piece<T, V>*>(slot + threadIdx.x * BYTES);
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = to_float(p.e[j]);
        }
    }
    __device__ __forceinline__ void write(T* to, const float (&v)[V]) const {
        if (STRIP) {
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (has(j)) to[threadIdx.x + j * STREAM_THREADS] = from_float<T>(v[j]);
        } else {
            Piece<T, V> p;
#pragma unroll
            for (int j = 0; j < V; ++j) p.e[j] = from_float<T>(v[j]);
            *reinterpret_cast<Piece<T, V>*>(to) = p;
        }
    }
    // states of the thread's chains; a null array holds zeros
    __device__ __forceinline__ void read_states(const float* p, float (&v)[V]) const {
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = 0.f;
        if (!p) return;
        if (STRIP) {
#pragma unroll
            for (int j = 0; j < V; ++j) if (has(j)) v[j] = p[row + j * STREAM_THREADS];
        } else {
            const Piece<float, (V > 4 ? 4 : V)>* q = reinterpret_cast<const Piece<float, (V > 4 ? 4 : V)>*>(p + row);
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = q[j / 4].e[j % 4];
        }
    }
    __device__ __forceinline__ void write_states(float* p, const float (&v)[V]) const {
        if (STRIP) {
#pragma unroll
            for (int j = 0; j < V; ++j) if (has(j)) p[row + j * STREAM_THREADS] = v[j];
        } else {
#pragma unroll
            for (int k = 0; k < V; k += 4) {
                Piece<float, (V > 4 ? 4 : V)> u;
#pragma unroll
                for (int j = 0; j < 4 && k + j < V; ++j) u.e[j] = v[k + j];
                reinterpret_cast<Piece<float, (V > 4 ? 4 : V)>*>(p + row)[k / 4] = u;
            }
        }
    }
};

template <class T, int V, bool STRIP> constexpr int stream_smem() { return 2 * BATCH * DEPTH * Rows<T, V, STRIP>::SLOT; }
template <class T, int V, bool STRIP> constexpr int vjp_smem() { return 3 * CHUNK * 2 * Rows<T, V, STRIP>::SLOT; }

// Forward, or the maps of parts for either direction (KIND: FORWARD, MAP_FORWARD, MAP_VJP).
template <class T, int V, bool REVERSE, bool STRIP, int KIND>
__global__ void __launch_bounds__(STREAM_THREADS) stream_kernel(const __grid_constant__ Args a) {
    extern __shared__ __align__(16) unsigned char ring[];
    grid_dependency_wait();
    using R = Rows<T, V, STRIP>;
    constexpr bool MAPS = KIND != FORWARD, BACK = KIND == MAP_VJP;
    R c;
    c.find(a);
    if (!STRIP && !c.there) return;
    const Strides& so = BACK ? a.sdy : a.sx;
    const T* gate = c.at(static_cast<const T*>(a.gate), a.sgate);
    const T* other = c.at(static_cast<const T*>(BACK ? a.dy : a.x), so);
    T* y = MAPS ? nullptr : c.at(static_cast<T*>(a.y), a.sy);
    const long long valid = valid_steps(a, c.batch), part = blockIdx.y, begin = part * a.part, end = begin + a.part < a.steps ? begin + a.part : a.steps;
    // step n of the part, in the order in which it is taken, is t0 + n dt of the array
    constexpr int dt = BACK != REVERSE ? -1 : 1;
    const long long q0 = BACK ? end - 1 : begin, t0 = REVERSE ? a.steps - 1 - q0 : q0;
    const int count = (int)(end - begin);
    float h[V], prod[V];
#pragma unroll
    for (int j = 0; j < V; ++j) { h[j] = 0.f; prod[j] = 1.f; }
    if (!MAPS) c.read_states(a.parts > 1 ? a.maps_b + part * a.rows : a.state, h);

    auto slot = [&](int n, int array) { return ring + (((n / BATCH) % DEPTH * BATCH + n % BATCH) * 2 + array) * R::SLOT; };
    auto fetch = [&](int n0) {
        if (STRIP) {
            const int pieces = R::pieces();
            for (int k = threadIdx.x; k < 2 * BATCH * pieces; k += STREAM_THREADS) {
                const int row = k / pieces, n = n0 + (row >> 1), array = row & 1;
                const long long t = t0 + (long long)n * dt;
                if (n < count && t < valid) c.copy_piece(a, slot(n, array), array ? other + t * so.step : gate + t * a.sgate.step, k - row * pieces);
            }
        } else {
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const long long t = t0 + (long long)(n0 + k) * dt;
                if (n0 + k < count && t < valid) {
                    c.copy((uint32_t)__cvta_generic_to_shared(slot(n0 + k, 0)), gate + t * a.sgate.step);
                    c.copy((uint32_t)__cvta_generic_to_shared(slot(n0 + k, 1)), other + t * so.step);
                }
            }
        }
        copies_end();
    };
    for (int g = 0; g < DEPTH - 1; ++g) fetch(g * BATCH);
    int to_save = a.chunk;
    float* saved = !MAPS && a.saved ? a.saved + begin / a.chunk * a.rows : nullptr;
    for (int n0 = 0; n0 < count; n0 += BATCH) {
        fetch(n0 + (DEPTH - 1) * BATCH);
        copies_wait<DEPTH - 1>();
        if (STRIP) __syncthreads();
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const int n = n0 + k;
            const long long t = t0 + (long long)n * dt;
            if (n >= count) break;
            float out[V];
            if (t < valid) {
                float g[V], u[V];
                c.read(slot(n, 0), gate + t * a.sgate.step, g);
                c.read(slot(n, 1), other + t * so.step, u);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float f, rest;
                    gate_of(g[j], f, rest);
                    h[j] = BACK ? f * (h[j] + u[j]) : fmaf(f, h[j], rest * u[j]);
                    if (MAPS) prod[j] *= f;
                    out[j] = h[j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) out[j] = 0.f;
            }
            if (!MAPS) {
                c.write(y + t * a.sy.step, out);
                if (--to_save == 0) {
                    to_save = a.chunk;
                    if (saved && begin + n + 1 < a.steps) c.write_states(saved, h);
                    if (saved) saved += a.rows;
                }
            }
        }
        if (STRIP) __syncthreads();
    }
    if (MAPS) {
        c.write_states(a.maps_a + part * a.rows, prod);
        c.write_states(a.maps_b + part * a.rows, h);
    } else if (a.last && end == a.steps) {
        c.write_states(a.last, h);
    }
}

// VJP: chunk by chunk from the part's end, the next chunk on its way.  The states before each step come from the saved one.
template <class T, int V, bool REVERSE, bool STRIP>
__global__ void __launch_bounds__(STREAM_THREADS, 3) stream_vjp(const __grid_constant__ Args a) {
    extern __shared__ __align__(16) unsigned char ring[];
    grid_dependency_wait();
    using R = Rows<T, V, STRIP>;
    R c;
    c.find(a);
    if (!STRIP && !c.there) return;
    const T* gate = c.at(static_cast<const T*>(a.gate), a.sgate);
    const T* x = c.at(static_cast<const T*>(a.x), a.sx);
    const T* dy = c.at(static_cast<const T*>(a.dy), a.sdy);
    T* dx = c.at(static_cast<T*>(a.dx), a.sdx);
    T* dg = c.at(static_cast<T*>(a.dg), a.sdg);
    const long long valid = valid_steps(a, c.batch), part = blockIdx.y, begin = part * a.part, end = begin + a.part < a.steps ? begin + a.part : a.steps;
    auto step = [&](long long q) { return REVERSE ? a.steps - 1 - q : q; };
    auto slot = [&](int buffer, int k, int array) { return ring + ((buffer * CHUNK + k) * 3 + array) * R::SLOT; };
    auto fetch = [&](long long q0, int buffer) {
        if (q0 >= begin) {
            const int count = (int)(end - q0 < a.chunk ? end - q0 : a.chunk);
            if (STRIP) {
                const int pieces = R::pieces();
                for (int i = threadIdx.x; i < 3 * count * pieces; i += STREAM_THREADS) {
                    const int row = i / pieces, k = row / 3, array = row - k * 3;
                    const long long t = step(q0 + k);
                    if (t < valid) c.copy_piece(a, slot(buffer, k, array), array == 0 ? gate + t * a.sgate.step : array == 1 ? x + t * a.sx.step : dy + t * a.sdy.step, i - row * pieces);
                }
            } else {
#pragma unroll
                for (int k = 0; k < CHUNK; ++k) {
                    const long long t = step(q0 + k);
                    if (k < count && t < valid) {
                        c.copy((uint32_t)__cvta_generic_to_shared(slot(buffer, k, 0)), gate + t * a.sgate.step);
                        c.copy((uint32_t)__cvta_generic_to_shared(slot(buffer, k, 1)), x + t * a.sx.step);
                        c.copy((uint32_t)__cvta_generic_to_shared(slot(buffer, k, 2)), dy + t * a.sdy.step);
                    }
                }
            }
        }
        copies_end();
    };
    float back[V];
    c.read_states(a.parts > 1 ? a.maps_b + part * a.rows : a.dlast, back);
    const long long from = begin + (end - begin - 1) / a.chunk * a.chunk;
    int buffer = 0;
    fetch(from, 0);
    for (long long q0 = from; q0 >= begin; q0 -= a.chunk, buffer ^= 1) {
        float h[V];
        c.read_states(q0 > 0 ? a.saved + (q0 / a.chunk - 1) * a.rows : a.state, h);
        fetch(q0 - a.chunk, buffer ^ 1);
        copies_wait<1>();
        if (STRIP) __syncthreads();
        const int count = (int)(end - q0 < a.chunk ? end - q0 : a.chunk);
        float f[CHUNK][V], rest[CHUNK][V], w[CHUNK][V];               // w: h_(t-1) - x_t
#pragma unroll
        for (int k = 0; k < CHUNK; ++k) {
            const long long t = step(q0 + k);
            if (k < count && t < valid) {
                float g[V], u[V];
                c.read(slot(buffer, k, 0), gate + t * a.sgate.step, g);
                c.read(slot(buffer, k, 1), x + t * a.sx.step, u);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    gate_of(g[j], f[k][j], rest[k][j]);
                    w[k][j] = h[j] - u[j];
                    h[j] = fmaf(f[k][j], h[j], rest[k][j] * u[j]);
                }
            }
        }
#pragma unroll
        for (int k = CHUNK - 1; k >= 0; --k) {
            if (k >= count) continue;
            const long long t = step(q0 + k);
            float ox[V], og[V];
            if (t < valid) {
                float d[V];
                c.read(slot(buffer, k, 2), dy + t * a.sdy.step, d);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    d[j] += back[j];
                    back[j] = d[j] * f[k][j];
                    ox[j] = d[j] * rest[k][j];
                    og[j] = ox[j] * f[k][j] * w[k][j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) { ox[j] = 0.f; og[j] = 0.f; }
            }
            c.write(dx + t * a.sdx.step, ox);
            c.write(dg + t * a.sdg.step, og);
        }
        if (STRIP) __syncthreads();
    }
    if (a.dstate && begin == 0) c.write_states(a.dstate, back);
}

// The parts' maps joined: maps_b becomes the state that each part starts from.  32 neighbouring chains a block; each of its warps
// composes the maps of a share of the parts, then runs through them from the state that the shares before leave.
constexpr int JOIN_WARPS = 16;
template <int AHEAD>
__global__ void __launch_bounds__(32 * JOIN_WARPS) join_parts(const __grid_constant__ Args a) {
    grid_dependency_wait();
    __shared__ float share_a[JOIN_WARPS][32], share_b[JOIN_WARPS][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long row = (long long)blockIdx.x * 32 + lane;
    const bool there = row < a.rows;
    const int first = (int)((long long)a.parts * warp / JOIN_WARPS), last = (int)((long long)a.parts * (warp + 1) / JOIN_WARPS);
    const long long step = a.descending ? -a.rows : a.rows, base = (a.descending ? (a.parts - 1) * a.rows : 0) + row;
    float pa = 1.f, pb = 0.f;
    for (int p = first; p < last; p += AHEAD) {
        float fa[AHEAD], fb[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const bool in = there && p + k < last;
            fa[k] = in ? a.maps_a[base + (p + k) * step] : 1.f;
            fb[k] = in ? a.maps_b[base + (p + k) * step] : 0.f;
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) { pb = fmaf(fa[k], pb, fb[k]); pa *= fa[k]; }
    }
    share_a[warp][lane] = pa; share_b[warp][lane] = pb;
    __syncthreads();
    float s = there && a.enter ? a.enter[row] : 0.f;
    for (int w = 0; w < warp; ++w) s = fmaf(share_a[w][lane], s, share_b[w][lane]);
    for (int p = first; p < last; p += AHEAD) {
        float fa[AHEAD], fb[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const bool in = there && p + k < last;
            fa[k] = in ? a.maps_a[base + (p + k) * step] : 1.f;
            fb[k] = in ? a.maps_b[base + (p + k) * step] : 0.f;
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (there && p + k < last) { a.maps_b[base + (p + k) * step] = s; s = fmaf(fa[k], s, fb[k]); }
    }
}

}  // namespace scan
}  // namespace gleam
