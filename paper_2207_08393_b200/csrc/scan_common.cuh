// What the kernels of the gated recurrence share: arguments, the gate, strided addresses.
//
//     h_t = f_t h_(t-1) + (1 - f_t) x_t,   f_t = 1 / (1 + exp(-gate_t)),   t = 0, 1, ... or T - 1, T - 2, ... (reverse)
//
// and with D_t the cotangent of h_t and c what the step behind t hands back,
//
//     D_t = dy_t + c,   dx_t = D_t (1 - f_t),   dgate_t = D_t (h_(t-1) - x_t) f_t (1 - f_t),   c <- D_t f_t.
//
// Both are chains of maps s -> a s + b, which compose as (a2, b2) o (a1, b1) = (a2 a1, a2 b1 + b2): a chain can be cut into parts
// whose maps are found side by side, joined, and run again from the right states.  States are 32-bit numbers throughout.  The VJP
// needs h_(t-1): it is computed again from states that the forward call saves at few places, so that neither h as stored (rounded
// to the arrays' type) nor another array of the same size is read.
#pragma once
#include "prior_common.cuh"

namespace gleam {
namespace scan {

using prior::from_float;
using prior::Pack;
using prior::to_float;

struct Strides { long long batch, channel, step; };

struct Args {
    const void* x; const void* gate; const void* dy;      // dy: VJP
    void* y; void* dx; void* dg;
    Strides sx, sgate, sdy, sy, sdx, sdg;
    const float* state;                // initial states (rows) or null: zeros
    float* last;                       // forward: last states, or null
    const float* dlast; float* dstate; // VJP: their cotangents, or null
    float* saved;                      // states at the chunks' (tiles') starts; forward: or null
    float* maps_a; float* maps_b;      // (parts, rows): maps of the parts, then the state (b) that each part starts from
    const int* lengths;                // valid steps of each example, or null
    long long batch, channels, steps, inner, rows;        // rows = batch * channels * inner chains
    int parts; long long part;         // parts of a chain and steps of a part (a multiple of the chunk)
    int chunk;                         // columns: steps between saved states
    long long run;                     // chains of one run where steps are contiguous
    int descending;                    // the chain enters its last part first
    const float* enter;                // join_parts: states at the chain's entry, or null
};

enum { MAP_FORWARD, MAP_VJP, FORWARD, VJP };       // MAP_*: only the parts' maps are formed

// f and 1 - f from e = exp(-gate): f = 1 / (1 + e), 1 - f = e f where e <= 1, the difference where not (there it is exact, and holds for
// e = infinity).  f is exactly 1 or 0 for an infinite gate; both are NaN for one that is NaN.  Two at a time: sums and products of pairs take
// one instruction.
//
// With 32-bit gates e is CUDA's exponential, and f and 1 - f are good to 2^-21 of themselves wherever they are normal numbers.  Gates of
// 16 bits are themselves off by 2^-12 or 2^-9 of their size; e is 2 to the power of -gate log2(e) rounded to 32 bits there, which costs |gate|
// 2^-23 of e and six instructions less (4 x 160 x 81920 bf16, forward and VJP, 166 us; with CUDA's 174).
using prior::fma2;
using prior::Two;
__device__ __forceinline__ float exp2_of(float x) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
__device__ __forceinline__ float inverse_of(float x) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x)); return r; }
template <class T> __device__ __forceinline__ Two exp_of_minus(Two g) {
    if constexpr (sizeof(T) == 4) return Two(expf(-g.lo()), expf(-g.hi()));
    const Two x = g * Two(-1.4426950408889634f);
    return Two(exp2_of(x.lo()), exp2_of(x.hi()));
}
__device__ __forceinline__ void gates_from(Two e, Two& f, Two& rest) {
    const Two d = e + Two(1.f);
    f = Two(inverse_of(d.lo()), inverse_of(d.hi()));
    const Two p = e * f, q = fma2(f, Two(-1.f), Two(1.f));
    rest = Two(e.lo() > 1.f ? q.lo() : p.lo(), e.hi() > 1.f ? q.hi() : p.hi());
}
template <class T> __device__ __forceinline__ void gates_of(Two g, Two& f, Two& rest) { gates_from(exp_of_minus<T>(g), f, rest); }
template <class T> __device__ __forceinline__ void gate_of(float g, float& f, float& rest) {
    const float e = sizeof(T) == 4 ? expf(-g) : exp2_of(g * -1.4426950408889634f);
    f = inverse_of(1.f + e);
    rest = e > 1.f ? 1.f - f : e * f;
}

__device__ __forceinline__ long long valid_steps(const Args& a, long long batch) {
    if (!a.lengths) return a.steps;
    const long long n = a.lengths[batch];
    return n < 0 ? 0 : n > a.steps ? a.steps : n;
}

}  // namespace scan
}  // namespace gleam
