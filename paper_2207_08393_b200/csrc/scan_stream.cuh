// The gated recurrence where the chains lie side by side in memory and a row of them is wide enough for a block: arrays come through
// shared memory by asynchronous copies, several steps ahead of their use.
//
// What bounds it is memory; what it takes is bytes under way (about 40 KB an SM) that cost no registers, and enough warps that the
// chains' arithmetic (some 18 instructions an element forward, 35 for the VJP) hides behind them.  Two forms:
//   private   every row of every array starts at a multiple of a thread's piece (16 or 8 bytes): a thread copies, reads and stores its
//             own V neighbouring chains, and no thread waits for another;
//   strips    rows start anywhere (an odd number of voxels): a block copies the 16-byte pieces that its strip of a row touches and reads
//             from them element by element, lanes side by side; a thread's V chains are a block's width apart.
// Loads into registers instead (forward + VJP): 60 x 20 x 30720 float32 80 + 219 us for 70 + 117; 4 x 160 x 81920 bf16 335 + 583 for 60 + 103.
// What is left there to the 48 and 80 that memory takes: half of the issue slots, two thirds of that exponentials, reciprocals and
// conversions, in as few warps as there are chains for. The VJP keeps two numbers an element of a chunk in registers: six steps leave room
// for a fifth (pieces of 8 bytes) or third block (16) on the SM; with eight, 60 x 20 x 30720 took 127 and 4 x 160 x 81920 126.
#pragma once
#include "scan_common.cuh"

#include <type_traits>

namespace gleam {
namespace scan {

constexpr int STREAM_THREADS = 64, VJP_THREADS = 128;        // of a block
constexpr int CHUNK = 6;                   // steps between saved states: what a VJP holds at a time
constexpr int BATCH = 4, DEPTH = 3;        // steps of a copy group, and groups of the ring (forward): more groups cost warps, fewer steps instructions

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

__device__ __forceinline__ Two pair_of(const float* p) { return Two(p[0], p[1]); }
__device__ __forceinline__ Two pair_of(const __half* p) { const float2 f = __half22float2(*reinterpret_cast<const __half2*>(p)); return Two(f.x, f.y); }
__device__ __forceinline__ Two pair_of(const __nv_bfloat16* p) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(p);
    return Two(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
__device__ __forceinline__ void round_pair(float* p, Two v) { p[0] = v.lo(); p[1] = v.hi(); }
__device__ __forceinline__ void round_pair(__half* p, Two v) { *reinterpret_cast<__half2*>(p) = __floats2half2_rn(v.lo(), v.hi()); }
__device__ __forceinline__ void round_pair(__nv_bfloat16* p, Two v) { *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(v.lo(), v.hi()); }

// Steps n = 0, 1, ... count - 1 of a part are steps t0 + n dt of the array; those from `first` on, `there` of them, are inside the
// example's length.
struct Span {
    int count, first, there;
    __device__ __forceinline__ bool has(int n) const { return (uint32_t)(n - first) < (uint32_t)there; }
};
__device__ __forceinline__ Span span_of(long long t0, int dt, int count, long long valid) {
    Span s{count, 0, 0};
    if (dt > 0) {
        s.there = (int)(valid - t0 < 0 ? 0 : valid - t0 < count ? valid - t0 : count);
    } else {
        s.first = (int)(t0 - valid + 1 < 0 ? 0 : t0 - valid + 1 < count ? t0 - valid + 1 : count);
        s.there = count - s.first;
    }
    return s;
}

// The chains of a block and a thread, and how rows of them pass through shared memory.
template <class T, int V, bool STRIP, int THREADS>
struct Rows {
    static constexpr int BYTES = V * sizeof(T), WIDTH = THREADS * V;
    static constexpr int SLOT = THREADS * BYTES + (STRIP ? 16 : 0);       // bytes of a row in shared memory
    long long row, batch;                    // the thread's first chain, its example
    long long at_batch, at_channel, at_i;    // ... (strips: the block's first chain)
    int there;                               // chains of the strip; private: whether there are any
    bool inside;                             // strips: they are as many as can be, and 16 bytes more of the row on both sides

    __device__ __forceinline__ void find(const Args& a) {
        if (STRIP) {
            const long long strips = (a.inner + WIDTH - 1) / WIDTH, u = blockIdx.x / strips, first = (blockIdx.x - u * strips) * WIDTH;
            at_batch = u / a.channels; at_channel = u - at_batch * a.channels; at_i = first;
            there = (int)(a.inner - first < WIDTH ? a.inner - first : WIDTH);
            row = u * a.inner + first + threadIdx.x;
            inside = first >= 16 && first + WIDTH + 16 <= a.inner;
        } else {
            row = ((long long)blockIdx.x * THREADS + threadIdx.x) * V;
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
    __device__ __forceinline__ bool has(int j) const { return STRIP ? (int)threadIdx.x + j * THREADS < there : true; }

    // private: the thread's piece of a row
    __device__ __forceinline__ void copy(uint32_t slot, const T* from) const { copy_async<BYTES>(slot + threadIdx.x * BYTES, from); }
    // strips: the 16-byte pieces that the strip touches in one row, by threads number `turn` of `turns`; what is not inside the row as a
    // whole goes element by element
    __device__ __forceinline__ void copy_row(const Args& a, unsigned char* slot, const T* from, int turn, int turns) const {
        const uintptr_t first = (uintptr_t)from, stop = first + there * sizeof(T);
        uintptr_t x = (first & ~(uintptr_t)15) + 16 * turn;
        uint32_t to = (uint32_t)__cvta_generic_to_shared(slot) + 16 * turn;
        if (inside) {
            for (; x < stop; x += 16 * turns, to += 16 * turns) copy_async<16>(to, (const void*)x);
            return;
        }
        const uintptr_t begin = first - at_i * sizeof(T), end = begin + a.inner * sizeof(T);
        for (unsigned char* s = slot + 16 * turn; x < stop; x += 16 * turns, to += 16 * turns, s += 16 * turns) {
            if (x >= begin && x + 16 <= end) copy_async<16>(to, (const void*)x);
            else
                for (int e = 0; e < 16; e += sizeof(T))
                    if (x + e >= first && x + e < stop) *reinterpret_cast<T*>(s + e) = *reinterpret_cast<const T*>(x + e);
        }
    }
    __device__ __forceinline__ void read(const unsigned char* slot, const T* from, Two (&v)[V / 2]) const {
        if (STRIP) {
            const T* s = reinterpret_cast<const T*>(slot + ((uint32_t)(uintptr_t)from & 15u)) + threadIdx.x;
#pragma unroll
            for (int j = 0; j < V; j += 2) v[j / 2] = Two(to_float(s[j * THREADS]), to_float(s[(j + 1) * THREADS]));
        } else {
            const Piece<T, V> p = *reinterpret_cast<const Piece<T, V>*>(slot + threadIdx.x * BYTES);
#pragma unroll
            for (int j = 0; j < V; j += 2) v[j / 2] = pair_of(p.e + j);
        }
    }
    __device__ __forceinline__ void write(T* to, const Two (&v)[V / 2]) const {
        if (STRIP) {
            T* p = to + threadIdx.x;
            if (inside) {
#pragma unroll
                for (int j = 0; j < V; ++j) p[j * THREADS] = from_float<T>(j & 1 ? v[j / 2].hi() : v[j / 2].lo());
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (has(j)) p[j * THREADS] = from_float<T>(j & 1 ? v[j / 2].hi() : v[j / 2].lo());
            }
        } else {
            Piece<T, V> p;
#pragma unroll
            for (int j = 0; j < V; j += 2) round_pair(p.e + j, v[j / 2]);
            *reinterpret_cast<Piece<T, V>*>(to) = p;
        }
    }
    // states of the thread's chains; a null array holds zeros
    __device__ __forceinline__ void read_states(const float* p, Two (&to)[V / 2]) const {
        float v[V];
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = 0.f;
        if (!p) {
        } else         if (STRIP) {
#pragma unroll
            for (int j = 0; j < V; ++j) if (has(j)) v[j] = p[row + j * THREADS];
        } else {
            const Piece<float, (V > 4 ? 4 : V)>* q = reinterpret_cast<const Piece<float, (V > 4 ? 4 : V)>*>(p + row);
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = q[j / 4].e[j % 4];
        }
#pragma unroll
        for (int j = 0; j < V; j += 2) to[j / 2] = Two(v[j], v[j + 1]);
    }
    __device__ __forceinline__ void write_states(float* p, const Two (&of)[V / 2]) const {
        float v[V];
#pragma unroll
        for (int j = 0; j < V; j += 2) { v[j] = of[j / 2].lo(); v[j + 1] = of[j / 2].hi(); }
        if (STRIP) {
#pragma unroll
            for (int j = 0; j < V; ++j) if (has(j)) p[row + j * THREADS] = v[j];
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

template <class T, int V, bool STRIP> constexpr int stream_smem() { return 2 * BATCH * DEPTH * Rows<T, V, STRIP, STREAM_THREADS>::SLOT; }
template <class T, int V, bool STRIP> constexpr int vjp_smem() { return 3 * CHUNK * 2 * Rows<T, V, STRIP, VJP_THREADS>::SLOT; }

// Forward, or the maps of parts for either direction (KIND: FORWARD, MAP_FORWARD, MAP_VJP).
template <class T, int V, bool REVERSE, bool STRIP, int KIND>
__global__ void __launch_bounds__(STREAM_THREADS) stream_kernel(const __grid_constant__ Args a) {
    extern __shared__ __align__(16) unsigned char ring[];
    grid_dependency_wait();
    using R = Rows<T, V, STRIP, STREAM_THREADS>;
    constexpr bool MAPS = KIND != FORWARD, BACK = KIND == MAP_VJP;
    constexpr int P = V / 2, dt = BACK != REVERSE ? -1 : 1;
    R c;
    c.find(a);
    if (!STRIP && !c.there) return;
    const long long part = blockIdx.y, begin = part * a.part, end = begin + a.part < a.steps ? begin + a.part : a.steps;
    const long long q0 = BACK ? end - 1 : begin, t0 = REVERSE ? a.steps - 1 - q0 : q0;
    const Span span = span_of(t0, dt, (int)(end - begin), valid_steps(a, c.batch));
    const Strides& so = BACK ? a.sdy : a.sx;
    const T* gate = c.at(static_cast<const T*>(a.gate), a.sgate) + t0 * a.sgate.step;
    const T* other = c.at(static_cast<const T*>(BACK ? a.dy : a.x), so) + t0 * so.step;
    T* y = MAPS ? nullptr : c.at(static_cast<T*>(a.y), a.sy) + t0 * a.sy.step;
    const long long gate_step = dt * a.sgate.step, other_step = dt * so.step, y_step = dt * a.sy.step;
    Two h[P], prod[P];
#pragma unroll
    for (int j = 0; j < P; ++j) { h[j] = Two(0.f); prod[j] = Two(1.f); }
    if (!MAPS) c.read_states(a.parts > 1 ? a.maps_b + part * a.rows : a.state, h);

    // group g of BATCH steps: slots (g mod DEPTH, step, array)
    const T* next_gate = gate;
    const T* next_other = other;
    auto fetch = [&](int group) {
        unsigned char* slots = ring + group % DEPTH * (2 * BATCH * R::SLOT);
        const int n0 = group * BATCH;
        if (STRIP) {
            constexpr int TURNS = STREAM_THREADS / (2 * BATCH);
            const int row = threadIdx.x / TURNS, n = row >> 1;
            if (span.has(n0 + n)) c.copy_row(a, slots + row * R::SLOT, row & 1 ? next_other + n * other_step : next_gate + n * gate_step, threadIdx.x % TURNS, TURNS);
            next_gate += BATCH * gate_step; next_other += BATCH * other_step;
        } else {
            const uint32_t at = (uint32_t)__cvta_generic_to_shared(slots);
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                if (span.has(n0 + k)) {
                    c.copy(at + 2 * k * R::SLOT, next_gate);
                    c.copy(at + (2 * k + 1) * R::SLOT, next_other);
                }
                next_gate += gate_step; next_other += other_step;
            }
        }
        copies_end();
    };
    for (int g = 0; g < DEPTH - 1; ++g) fetch(g);
    int to_save = a.chunk;
    float* saved = !MAPS && a.saved ? a.saved + begin / a.chunk * a.rows : nullptr;
    for (int n0 = 0, group = 0; n0 < span.count; n0 += BATCH, ++group) {
        fetch(group + DEPTH - 1);
        copies_wait<DEPTH - 1>();
        if (STRIP) __syncthreads();
        const unsigned char* slots = ring + group % DEPTH * (2 * BATCH * R::SLOT);
        auto run = [&](auto whole) {                                       // whole: a full group of steps that are all there
            constexpr bool ALL = decltype(whole)::value;
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const int n = n0 + k;
                if (!ALL && n >= span.count) break;
                Two out[P];
                if (ALL || span.has(n)) {
                    Two g[P], u[P];
                    c.read(slots + 2 * k * R::SLOT, gate, g);
                    c.read(slots + (2 * k + 1) * R::SLOT, other, u);
#pragma unroll
                    for (int j = 0; j < P; ++j) {
                        Two f, rest;
                        gates_of<T>(g[j], f, rest);
                        h[j] = BACK ? f * (h[j] + u[j]) : fma2(f, h[j], rest * u[j]);
                        if (MAPS) prod[j] = prod[j] * f;
                        out[j] = h[j];
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < P; ++j) out[j] = Two(0.f);
                }
                if (!MAPS) {
                    c.write(y, out);
                    y += y_step;
                    if (--to_save == 0) {
                        to_save = a.chunk;
                        if (saved && begin + n + 1 < a.steps) c.write_states(saved, h);
                        if (saved) saved += a.rows;
                    }
                }
                if (STRIP) { gate += gate_step; other += other_step; }      // their low bits say where a row lies in its slot
            }
        };
        if (n0 + BATCH <= span.count && span.has(n0) && span.has(n0 + BATCH - 1)) run(std::true_type{});
        else run(std::false_type{});
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
__global__ void __launch_bounds__(VJP_THREADS, V * sizeof(T) == 16 ? 3 : STRIP ? 6 : 5) stream_vjp(const __grid_constant__ Args a) {
    extern __shared__ __align__(16) unsigned char ring[];
    grid_dependency_wait();
    using R = Rows<T, V, STRIP, VJP_THREADS>;
    constexpr int P = V / 2, dt = REVERSE ? -1 : 1;
    R c;
    c.find(a);
    if (!STRIP && !c.there) return;
    const long long part = blockIdx.y, begin = part * a.part, end = begin + a.part < a.steps ? begin + a.part : a.steps;
    const int last = (int)((end - begin - 1) / a.chunk) * a.chunk;                   // the part's last chunk begins there
    const long long t0 = REVERSE ? a.steps - 1 - begin : begin;
    const Span span = span_of(t0, dt, (int)(end - begin), valid_steps(a, c.batch));
    // all pointers stand at the chunk's first step; copies are one chunk ahead
    const T* gate = c.at(static_cast<const T*>(a.gate), a.sgate) + (t0 + dt * (long long)last) * a.sgate.step;
    const T* x = c.at(static_cast<const T*>(a.x), a.sx) + (t0 + dt * (long long)last) * a.sx.step;
    const T* dy = c.at(static_cast<const T*>(a.dy), a.sdy) + (t0 + dt * (long long)last) * a.sdy.step;
    T* dx = c.at(static_cast<T*>(a.dx), a.sdx) + (t0 + dt * (long long)last) * a.sdx.step;
    T* dg = c.at(static_cast<T*>(a.dg), a.sdg) + (t0 + dt * (long long)last) * a.sdg.step;
    const long long gate_step = dt * a.sgate.step, x_step = dt * a.sx.step, dy_step = dt * a.sdy.step, dx_step = dt * a.sdx.step, dg_step = dt * a.sdg.step;
    auto fetch = [&](int n0, int buffer, const T* g, const T* u, const T* d) {
        if (n0 >= 0) {
            unsigned char* slots = ring + buffer * (3 * CHUNK * R::SLOT);
            const int count = span.count - n0 < a.chunk ? span.count - n0 : a.chunk;
            if (STRIP) {
                constexpr int TURNS = VJP_THREADS / (3 * CHUNK);
                const int row = threadIdx.x / TURNS, k = row / 3, array = row - k * 3;
                if (k < count && span.has(n0 + k))
                    c.copy_row(a, slots + row * R::SLOT, array == 0 ? g + k * gate_step : array == 1 ? u + k * x_step : d + k * dy_step, threadIdx.x % TURNS, TURNS);
            } else {
                const uint32_t at = (uint32_t)__cvta_generic_to_shared(slots);
#pragma unroll
                for (int k = 0; k < CHUNK; ++k) {
                    if (k < count && span.has(n0 + k)) {
                        c.copy(at + 3 * k * R::SLOT, g);
                        c.copy(at + (3 * k + 1) * R::SLOT, u);
                        c.copy(at + (3 * k + 2) * R::SLOT, d);
                    }
                    g += gate_step; u += x_step; d += dy_step;
                }
            }
        }
        copies_end();
    };
    Two back[P];
    c.read_states(a.parts > 1 ? a.maps_b + part * a.rows : a.dlast, back);
    fetch(last, 0, gate, x, dy);
    int buffer = 0;
    for (int n0 = last; n0 >= 0; n0 -= a.chunk, buffer ^= 1) {
        Two h[P];
        const long long chunk = (begin + n0) / a.chunk;
        c.read_states(chunk > 0 ? a.saved + (chunk - 1) * a.rows : a.state, h);
        fetch(n0 - a.chunk, buffer ^ 1, gate - a.chunk * gate_step, x - a.chunk * x_step, dy - a.chunk * dy_step);
        copies_wait<1>();
        if (STRIP) __syncthreads();
        const unsigned char* slots = ring + buffer * (3 * CHUNK * R::SLOT);
        const int count = span.count - n0 < a.chunk ? span.count - n0 : a.chunk;
        Two e[CHUNK][P], w[CHUNK][P];            // exp(-gate), h_(t-1) - x_t: the gates once more cost less than 32 registers to keep them
#pragma unroll
        for (int k = 0; k < CHUNK; ++k) {
            if (k < count && span.has(n0 + k)) {
                Two g[P], u[P];
                c.read(slots + 3 * k * R::SLOT, gate + k * gate_step, g);
                c.read(slots + (3 * k + 1) * R::SLOT, x + k * x_step, u);
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    Two f, rest;
                    e[k][j] = exp_of_minus<T>(g[j]);
                    gates_from(e[k][j], f, rest);
                    w[k][j] = fma2(u[j], Two(-1.f), h[j]);
                    h[j] = fma2(f, h[j], rest * u[j]);
                }
            }
        }
        T* to_x = dx + (count - 1) * dx_step;
        T* to_g = dg + (count - 1) * dg_step;
#pragma unroll
        for (int k = CHUNK - 1; k >= 0; --k) {
            if (k >= count) continue;
            Two ox[P], og[P];
            if (span.has(n0 + k)) {
                Two d[P];
                c.read(slots + (3 * k + 2) * R::SLOT, dy + k * dy_step, d);
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    Two f, rest;
                    gates_from(e[k][j], f, rest);
                    d[j] = d[j] + back[j];
                    back[j] = d[j] * f;
                    ox[j] = d[j] * rest;
                    og[j] = ox[j] * f * w[k][j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < P; ++j) ox[j] = og[j] = Two(0.f);
            }
            c.write(to_x, ox);
            c.write(to_g, og);
            to_x -= dx_step; to_g -= dg_step;
        }
        if (STRIP) __syncthreads();
        gate -= a.chunk * gate_step; x -= a.chunk * x_step; dy -= a.chunk * dy_step; dx -= a.chunk * dx_step; dg -= a.chunk * dg_step;
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
