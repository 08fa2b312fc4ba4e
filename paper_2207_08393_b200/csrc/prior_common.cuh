// What the operators of the learned prior share: element types, the dropout mask, arguments of the kernels, sums over a block.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "launch_overlap.cuh"

namespace gleam {
namespace prior {

// Arrays are (outer, features, inner) with contiguous slices; pitches are elements from one outer slice to the next.
struct Args {
    const void* x;           // forward: x;  VJP: grad_y (norm, tail), grad_out (dropout)
    const void* res;         // forward: residual or null;  VJP: what was normalised (x, or the stored sum)
    const void* gsum;        // VJP of the tail: grad_sum or null
    void* out;               // forward: y (dropout: out);  VJP: grad_x
    void* out2;              // tail: sum;  its VJP: grad_residual
    const void* weight; const void* bias;      // or null
    float* mean; float* rstd;
    float* part;             // partial sums of the weights' gradients: (parts, 2, features)
    void* gw; void* gb;      // gradients of the weights, or null
    long long outer, inner, features;
    long long px, pres, pgsum, pout, pout2;
    float eps, scale;        // scale = 1 / (1 - p)
    uint32_t last;           // elements whose word is at most this are dropped
    int dropping;            // whether any is
    int weight_f32;          // weights and their gradients are float32, else of the arrays' type
    uint64_t seed, offset;
    const unsigned long long* step;
};

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

template <class T>
__device__ __forceinline__ float weight_at(const void* w, int f32, long long c) {
    return f32 ? static_cast<const float*>(w)[c] : to_float(static_cast<const T*>(w)[c]);
}

// The dropout mask.  Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): ten
// rounds that multiply two words of the counter by constants and exchange the halves of the products, with two key words
// that advance by constants.  Four elements share a counter, so an element costs 5 products and 5 three-way exclusive ors.
struct Mask {
    uint32_t k0, k1, s0, s1, last;
    uint64_t offset;
    __device__ __forceinline__ explicit Mask(const Args& a) {
        k0 = (uint32_t)a.seed; k1 = (uint32_t)(a.seed >> 32);
        const unsigned long long step = a.step ? *a.step : 0ull;
        s0 = (uint32_t)step; s1 = (uint32_t)(step >> 32);
        last = a.last; offset = a.offset;
    }
    __device__ __forceinline__ uint4 words(uint64_t block) const {
        block += offset;
        uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = s0, c3 = s1, q0 = k0, q1 = k1;
#pragma unroll
        for (int r = 0; r < 10; ++r) {
            const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
            c0 = (uint32_t)(p1 >> 32) ^ c1 ^ q0; c1 = (uint32_t)p1;
            c2 = (uint32_t)(p0 >> 32) ^ c3 ^ q1; c3 = (uint32_t)p0;
            q0 += 0x9E3779B9u; q1 += 0xBB67AE85u;
        }
        return make_uint4(c0, c1, c2, c3);
    }
    __device__ __forceinline__ bool dropped(uint32_t word) const { return word <= last; }
    __device__ __forceinline__ bool dropped_at(uint64_t i) const {
        const uint4 w = words(i >> 2);
        const uint32_t lane = (uint32_t)i & 3u;
        return dropped(lane == 0 ? w.x : lane == 1 ? w.y : lane == 2 ? w.z : w.w);
    }
};

// Sums of a pair over the block in a fixed order, in every thread.  One barrier before and one after the exchange.
struct Pair { float a, b; };
template <int WARPS>
__device__ __forceinline__ Pair block_sum(Pair v, float (&buf)[2 * WARPS]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int o = 16; o > 0; o >>= 1) {
        v.a += __shfl_xor_sync(0xffffffffu, v.a, o);
        v.b += __shfl_xor_sync(0xffffffffu, v.b, o);
    }
    __syncthreads();
    if (lane == 0) { buf[2 * warp] = v.a; buf[2 * warp + 1] = v.b; }
    __syncthreads();
    Pair t{0.f, 0.f};
#pragma unroll
    for (int w = 0; w < WARPS; ++w) { t.a += buf[2 * w]; t.b += buf[2 * w + 1]; }
    return t;
}

}  // namespace prior
}  // namespace gleam
