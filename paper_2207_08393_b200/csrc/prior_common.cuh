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
    int aligned;             // rows: all arrays lie alike against multiples of 16 bytes
    int weight_f32;          // weights and their gradients are float32, else of the arrays' type
    uint64_t offset;
    const unsigned long long* step;
    uint32_t keys[20];       // the mask's round keys: constants of the launch, operands of its exclusive ors
};

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Sixteen bytes of an array, as they lie in memory and as numbers.
template <class T> constexpr int VEC = 16 / sizeof(T);
template <class T> struct alignas(16) Pack { T e[VEC<T>]; };
template <class T>
__device__ __forceinline__ Pack<T> load_pack(const T* p) { return *reinterpret_cast<const Pack<T>*>(p); }
template <class T>
__device__ __forceinline__ void store_pack(T* p, const Pack<T>& v) { *reinterpret_cast<Pack<T>*>(p) = v; }

// Two numbers in a register pair: sm_100 multiplies and adds both with one instruction, each rounded as by itself.  What these
// kernels spend their issue slots on is this arithmetic.
struct Two {
    unsigned long long bits;
    Two() = default;
    __device__ __forceinline__ Two(float lo, float hi) { asm("mov.b64 %0, {%1, %2};" : "=l"(bits) : "f"(lo), "f"(hi)); }
    __device__ __forceinline__ explicit Two(float both) : Two(both, both) {}
    __device__ __forceinline__ float lo() const { float l, h; asm("mov.b64 {%0, %1}, %2;" : "=f"(l), "=f"(h) : "l"(bits)); return l; }
    __device__ __forceinline__ float hi() const { float l, h; asm("mov.b64 {%0, %1}, %2;" : "=f"(l), "=f"(h) : "l"(bits)); return h; }
    __device__ __forceinline__ float sum() const { return lo() + hi(); }
};
__device__ __forceinline__ Two operator+(Two a, Two b) { Two r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits)); return r; }
__device__ __forceinline__ Two operator*(Two a, Two b) { Two r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits)); return r; }
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) { Two r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.bits) : "l"(a.bits), "l"(b.bits), "l"(c.bits)); return r; }

__device__ __forceinline__ void unpack(const Pack<float>& p, Two (&v)[2]) {
    v[0] = Two(p.e[0], p.e[1]); v[1] = Two(p.e[2], p.e[3]);
}
__device__ __forceinline__ void unpack(const Pack<__half>& p, Two (&v)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 f = __half22float2(reinterpret_cast<const __half2*>(&p)[j]);
        v[j] = Two(f.x, f.y);
    }
}
__device__ __forceinline__ void unpack(const Pack<__nv_bfloat16>& p, Two (&v)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t w = reinterpret_cast<const uint32_t*>(&p)[j];
        v[j] = Two(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
}
template <class T> __device__ __forceinline__ Pack<T> pack(const Two (&v)[VEC<T> / 2]);
template <> __device__ __forceinline__ Pack<float> pack<float>(const Two (&v)[2]) {
    Pack<float> p;
#pragma unroll
    for (int j = 0; j < 2; ++j) { p.e[2 * j] = v[j].lo(); p.e[2 * j + 1] = v[j].hi(); }
    return p;
}
template <> __device__ __forceinline__ Pack<__half> pack<__half>(const Two (&v)[4]) {
    Pack<__half> p;
#pragma unroll
    for (int j = 0; j < 4; ++j) reinterpret_cast<__half2*>(&p)[j] = __floats2half2_rn(v[j].lo(), v[j].hi());
    return p;
}
template <> __device__ __forceinline__ Pack<__nv_bfloat16> pack<__nv_bfloat16>(const Two (&v)[4]) {
    Pack<__nv_bfloat16> p;
#pragma unroll
    for (int j = 0; j < 4; ++j) reinterpret_cast<__nv_bfloat162*>(&p)[j] = __floats2bfloat162_rn(v[j].lo(), v[j].hi());
    return p;
}

// residual + dropout(x) in the arrays' type: one fused multiply-add, then one rounding to the stored type.
template <class T>
__device__ __forceinline__ T tail_sum(float x, float res, bool dropped, float scale) {
    return from_float<T>(dropped ? res : fmaf(x, scale, res));
}

template <class T>
__device__ __forceinline__ float weight_at(const void* w, int f32, long long c) {
    return f32 ? static_cast<const float*>(w)[c] : to_float(static_cast<const T*>(w)[c]);
}

template <class T>
__device__ __forceinline__ void store_weight_grad(void* to, int f32, long long c, float v) {
    if (f32) static_cast<float*>(to)[c] = v;
    else static_cast<T*>(to)[c] = from_float<T>(v);
}

// The dropout mask.  Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): ten
// rounds that multiply two words of the counter by constants and exchange the halves of the products, with two key words
// that advance by constants from round to round.  Four elements share a counter, so an element costs 5 products of 32 x 32
// bits and 5 three-way exclusive ors; the round keys come ready from the host.
struct Mask {
    const Args& a;
    uint32_t s0, s1;
    __device__ __forceinline__ explicit Mask(const Args& args) : a(args) {
        const unsigned long long step = a.step ? *a.step : 0ull;
        s0 = (uint32_t)step; s1 = (uint32_t)(step >> 32);
    }
    __device__ __forceinline__ uint64_t counter(uint64_t block) const { return block + a.offset; }       // of elements 4 * block on
    __device__ __forceinline__ uint4 words(uint64_t counter) const {
        uint32_t c0 = (uint32_t)counter, c1 = (uint32_t)(counter >> 32), c2 = s0, c3 = s1;
#pragma unroll
        for (int r = 0; r < 10; ++r) {
            const uint64_t p0 = (uint64_t)c0 * 0xD2511F53u, p1 = (uint64_t)c2 * 0xCD9E8D57u;
            c0 = (uint32_t)(p1 >> 32) ^ c1 ^ a.keys[2 * r]; c1 = (uint32_t)p1;
            c2 = (uint32_t)(p0 >> 32) ^ c3 ^ a.keys[2 * r + 1]; c3 = (uint32_t)p0;
        }
        return make_uint4(c0, c1, c2, c3);
    }
    __device__ __forceinline__ bool dropped(const uint4& w, int lane) const {
        return (lane == 0 ? w.x : lane == 1 ? w.y : lane == 2 ? w.z : w.w) <= a.last;
    }
    // v = r + s v [s v] for the elements that are kept, r [0] for the others; the first four have this counter
    template <bool RES, bool DROP, int N>
    __device__ __forceinline__ void apply(uint64_t counter, Two (&v)[N], const Two (&r)[N]) const {
        const Two scale(a.scale);
#pragma unroll
        for (int q = 0; q < N / 2; ++q) {
            uint4 w;
            if (DROP) w = words(counter + q);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                Two& x = v[2 * q + h];
                const Two kept = RES ? fma2(x, scale, r[2 * q + h]) : x * scale, gone = RES ? r[2 * q + h] : Two(0.f);
                x = DROP ? Two(dropped(w, 2 * h) ? gone.lo() : kept.lo(), dropped(w, 2 * h + 1) ? gone.hi() : kept.hi()) : kept;
            }
        }
    }
    __device__ __forceinline__ bool dropped_at(uint64_t i) const { return dropped(words(counter(i >> 2)), (int)(i & 3u)); }
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
