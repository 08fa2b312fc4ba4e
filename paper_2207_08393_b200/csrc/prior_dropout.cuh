// Dropout, with an optional residual add: out = [residual +] (dropped ? 0 : x / (1 - p)).  Its VJP is the same map of the cotangent.
//
// Two or three arrays pass once; what bounds it next to memory are the mask's products: 32 x 32 -> 64 bit products run at a
// quarter of the rate of 32-bit ones, and five an element alone take 54 us for the 94.2 million elements of four knee slices
// with 100 features, where bf16 dropout has to move 58 us' worth of bytes and the residual add 87.  Measured there: 86 us (4.4
// TB/s) and 94 us (6.0 TB/s); in float32, 117 and 162 us (6.4 and 7.0 TB/s).
// One piece of 16 bytes a thread, in a grid that covers the array: 24 to 28 registers, every SM full of warps whose loads are
// under way while others draw words.  Two pieces a thread or a loop with the next piece requested early were slower (bf16: 122 and 93
// to 97 us for the 86, 156 and 109 for the 94): registers, and words that wait for their data, cost warps.
#pragma once
#include "prior_common.cuh"

namespace gleam {
namespace prior {

constexpr int DROP_THREADS = 256;

enum { DROP_FLAT, DROP_FLAT_END, DROP_SLICES, DROP_ELEMENTS };

// FLAT: the arrays are contiguous (one slice), 16-byte aligned and whole pieces; FLAT_END: the last piece is not whole (apart,
// because the code for it costs the others registers: 94 and 117 us for the 86 and 94 above); SLICES: aligned slices of whole
// pieces; ELEMENTS: any pitch and alignment, element by element.  Where nothing is dropped (DROP is false) no words are drawn.
template <class T, bool RES, bool DROP, int FORM>
__global__ void __launch_bounds__(DROP_THREADS) dropout_kernel(const __grid_constant__ Args a) {
    grid_dependency_wait();
    constexpr int V = VEC<T>;
    const Mask mask(a);
    const long long slice = a.features * a.inner, n = a.outer * slice;
    const long long piece = (long long)blockIdx.x * DROP_THREADS + threadIdx.x, i = piece * V;
    if (i >= n) return;
    const T* x = static_cast<const T*>(a.x);
    const T* res = static_cast<const T*>(a.res);
    T* out = static_cast<T*>(a.out);
    long long o = 0, e = i;
    if (FORM == DROP_SLICES || FORM == DROP_ELEMENTS) {
        o = n < (1ll << 32) ? (uint32_t)i / (uint32_t)slice : i / slice;
        e = i - o * slice;
    }
    if (FORM == DROP_FLAT || FORM == DROP_SLICES || (FORM == DROP_FLAT_END && i + V <= n)) {
        Pack<T> xv = load_pack(x + (o * a.px + e)), rv;
        if (RES) rv = load_pack(res + (o * a.pres + e));
        Two v[V / 2], r[V / 2];
        unpack(xv, v);
        if (RES) unpack(rv, r);
        mask.apply<RES, DROP>(mask.counter((uint64_t)(i >> 2)), v, r);
        store_pack(out + (o * a.pout + e), pack<T>(v));
        return;
    }
    if constexpr (FORM == DROP_FLAT_END || FORM == DROP_ELEMENTS) {
        // four elements at a time: they share a counter
#pragma unroll 1
        for (int q = 0; q < V / 4; ++q) {
            uint4 words = make_uint4(0u, 0u, 0u, 0u);
            if (DROP) words = mask.words(mask.counter((uint64_t)(i >> 2) + q));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (i + 4 * q + j >= n) return;
                const bool gone = DROP && mask.dropped(words, j);
                const float v = to_float(x[o * a.px + e]), r = RES ? to_float(res[o * a.pres + e]) : 0.f;
                out[o * a.pout + e] = from_float<T>(RES ? (gone ? r : fmaf(v, a.scale, r)) : gone ? 0.f : v * a.scale);
                if (++e == slice) { e = 0; ++o; }
            }
        }
    }
}

}  // namespace prior
}  // namespace gleam
