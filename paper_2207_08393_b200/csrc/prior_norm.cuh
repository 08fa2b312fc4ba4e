// Layer norm and the residual tail (dropout, residual add, layer norm): forward, VJP, gradients of the weights, for any number of
// features.  What fits rows in registers (prior_rows.cuh) or maps in tiles (prior_maps.cuh) goes there; these take longer rows (over
// 8192 features, over 8189 in float32 and 8185 in 16 bits where rows begin anywhere) and maps of more features (over 640; a tail's
// VJP in float32 over 560), and read their arrays again for each sum.
//
// Bound by memory: two to three passes where one would do (2000 rows of 20000 in bf16: 113 + 206 us for 25 + 37 us' worth of bytes;
// a map of 2000 x 4096: 35 + 56).  Variances are sums of squared deviations from the mean, so a large mean costs no digits.
// Sums are in 32 bits and in a fixed order.
#pragma once
#include "prior_common.cuh"

namespace gleam {
namespace prior {

constexpr int ROW_THREADS = 256, MAP_WARPS = 32;

// ---- rows (inner == 1), any number of features: a block per row, which it reads again for each sum -------------------------

template <class T, bool TAIL>
__global__ void __launch_bounds__(ROW_THREADS) row_forward(const __grid_constant__ Args a) {
    grid_dependency_wait();
    __shared__ float buf[2 * (ROW_THREADS / 32)];
    const Mask mask(a);
    const float n = (float)a.features;
    for (long long r = blockIdx.x; r < a.outer; r += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + r * a.px;
        T* y = static_cast<T*>(a.out) + r * a.pout;
        const T* v = x;
        float s = 0.f;
        if (TAIL) {
            const T* res = static_cast<const T*>(a.res) + r * a.pres;
            T* sum = static_cast<T*>(a.out2) + r * a.pout2;
            for (long long c = threadIdx.x; c < a.features; c += ROW_THREADS) {
                const bool gone = a.dropping && mask.dropped_at((uint64_t)(r * a.features + c));
                const T t = tail_sum<T>(to_float(x[c]), to_float(res[c]), gone, a.scale);
                sum[c] = t;
                s += to_float(t);
            }
            v = sum;
        } else {
            for (long long c = threadIdx.x; c < a.features; c += ROW_THREADS) s += to_float(v[c]);
        }
        const float mean = block_sum<ROW_THREADS / 32>(Pair{s, 0.f}, buf).a / n;
        float q = 0.f;
        for (long long c = threadIdx.x; c < a.features; c += ROW_THREADS) {
            const float d = to_float(v[c]) - mean;
            q = fmaf(d, d, q);
        }
        const float rstd = 1.f / sqrtf(block_sum<ROW_THREADS / 32>(Pair{q, 0.f}, buf).a / n + a.eps);
        for (long long c = threadIdx.x; c < a.features; c += ROW_THREADS) {
            const float h = (to_float(v[c]) - mean) * rstd;
            const float w = a.weight ? weight_at<T>(a.weight, a.weight_f32, c) : 1.f;
            y[c] = from_float<T>(fmaf(h, w, a.bias ? weight_at<T>(a.bias, a.weight_f32, c) : 0.f));
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
    }
}

template <class T, bool TAIL>
__global__ void __launch_bounds__(ROW_THREADS) row_vjp(const __grid_constant__ Args a) {
    grid_dependency_wait();
    __shared__ float buf[2 * (ROW_THREADS / 32)];
    const Mask mask(a);
    const float n = (float)a.features;
    for (long long r = blockIdx.x; r < a.outer; r += gridDim.x) {
        const T* dy = static_cast<const T*>(a.x) + r * a.px;
        const T* v = static_cast<const T*>(a.res) + r * a.pres;
        const float mean = a.mean[r], rstd = a.rstd[r];
        Pair s{0.f, 0.f};
        for (long long c = threadIdx.x; c < a.features; c += ROW_THREADS) {
            const float g = to_float(dy[c]) * (a.weight ? weight_at<T>(a.weight, a.weight_f32, c) : 1.f);
            s.a += g;
            s.b = fmaf(g, (to_float(v[c]) - mean) * rstd, s.b);
        }
        s = block_sum<ROW_THREADS / 32>(s, buf);
        const float c1 = s.a / n, c2 = s.b / n;
        T* out = static_cast<T*>(a.out) + r * a.pout;
        T* out2 = TAIL ? static_cast<T*>(a.out2) + r * a.pout2 : nullptr;
        const T* gsum = TAIL && a.gsum ? static_cast<const T*>(a.gsum) + r * a.pgsum : nullptr;
        for (long long c = threadIdx.x; c < a.features; c += ROW_THREADS) {
            const float g = to_float(dy[c]) * (a.weight ? weight_at<T>(a.weight, a.weight_f32, c) : 1.f);
            const float h = (to_float(v[c]) - mean) * rstd;
            float d = rstd * (g - c1 - h * c2);
            if (TAIL) {
                if (gsum) d += to_float(gsum[c]);
                out2[c] = from_float<T>(d);
                if (a.dropping) d = mask.dropped_at((uint64_t)(r * a.features + c)) ? 0.f : d * a.scale;
            }
            out[c] = from_float<T>(d);
        }
    }
}

// Partial sums of the weights' gradients: 32 features and a share of the rows per block.
template <class T>
__global__ void __launch_bounds__(256) row_weight_sums(const __grid_constant__ Args a) {
    grid_dependency_wait();
    __shared__ float buf[2][8][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long c = (long long)blockIdx.x * 32 + lane;
    float sw = 0.f, sb = 0.f;
    if (c < a.features) {
        for (long long r = (long long)blockIdx.y * 8 + warp; r < a.outer; r += (long long)gridDim.y * 8) {
            const float dy = to_float(static_cast<const T*>(a.x)[r * a.px + c]);
            const float h = (to_float(static_cast<const T*>(a.res)[r * a.pres + c]) - a.mean[r]) * a.rstd[r];
            sw = fmaf(dy, h, sw);
            sb += dy;
        }
    }
    buf[0][warp][lane] = sw; buf[1][warp][lane] = sb;
    __syncthreads();
    if (warp < 2 && c < a.features) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) t += buf[warp][w][lane];
        a.part[((long long)blockIdx.y * 2 + warp) * a.features + c] = t;
    }
}

// ---- maps (inner > 1) of any number of features: 32 neighbouring positions per block, its warps share the features ----------

// Sums of a pair over the warps of the block, for each lane (position), in every warp.
__device__ __forceinline__ Pair warps_sum(Pair v, float (&buf)[2][MAP_WARPS][32]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    __syncthreads();
    buf[0][warp][lane] = v.a; buf[1][warp][lane] = v.b;
    __syncthreads();
    Pair t{0.f, 0.f};
#pragma unroll
    for (int w = 0; w < MAP_WARPS; ++w) { t.a += buf[0][w][lane]; t.b += buf[1][w][lane]; }
    return t;
}

template <class T, bool TAIL>
__global__ void __launch_bounds__(MAP_WARPS * 32) map_forward(const __grid_constant__ Args a) {
    grid_dependency_wait();
    __shared__ float buf[2][MAP_WARPS][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Mask mask(a);
    const float n = (float)a.features;
    const long long positions = a.outer * a.inner, tiles = (positions + 31) / 32;
    for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const long long pos = tile * 32 + lane;
        const bool live = pos < positions;
        const long long o = live ? pos / a.inner : 0, k = live ? pos - o * a.inner : 0;
        const T* x = static_cast<const T*>(a.x) + o * a.px + k;
        T* y = static_cast<T*>(a.out) + o * a.pout + k;
        const T* v = x;
        float s = 0.f;
        if (TAIL) {
            const T* res = static_cast<const T*>(a.res) + o * a.pres + k;
            T* sum = static_cast<T*>(a.out2) + o * a.pout2 + k;
            for (long long c = warp; live && c < a.features; c += MAP_WARPS) {
                const long long at = c * a.inner;
                const bool gone = a.dropping && mask.dropped_at((uint64_t)(o * a.features * a.inner + at + k));
                const T t = tail_sum<T>(to_float(x[at]), to_float(res[at]), gone, a.scale);
                sum[at] = t;
                s += to_float(t);
            }
            v = sum;
        } else {
            for (long long c = warp; live && c < a.features; c += MAP_WARPS) s += to_float(v[c * a.inner]);
        }
        const float mean = warps_sum(Pair{s, 0.f}, buf).a / n;
        float q = 0.f;
        for (long long c = warp; live && c < a.features; c += MAP_WARPS) {
            const float d = to_float(v[c * a.inner]) - mean;
            q = fmaf(d, d, q);
        }
        const float rstd = 1.f / sqrtf(warps_sum(Pair{q, 0.f}, buf).a / n + a.eps);
        for (long long c = warp; live && c < a.features; c += MAP_WARPS) {
            const float h = (to_float(v[c * a.inner]) - mean) * rstd;
            const float w = a.weight ? weight_at<T>(a.weight, a.weight_f32, c) : 1.f;
            y[c * a.inner] = from_float<T>(fmaf(h, w, a.bias ? weight_at<T>(a.bias, a.weight_f32, c) : 0.f));
        }
        if (live && warp == 0) {
            if (a.mean) a.mean[pos] = mean;
            if (a.rstd) a.rstd[pos] = rstd;
        }
    }
}

template <class T, bool TAIL>
__global__ void __launch_bounds__(MAP_WARPS * 32) map_vjp(const __grid_constant__ Args a) {
    grid_dependency_wait();
    __shared__ float buf[2][MAP_WARPS][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Mask mask(a);
    const float n = (float)a.features;
    const long long positions = a.outer * a.inner, tiles = (positions + 31) / 32;
    for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const long long pos = tile * 32 + lane;
        const bool live = pos < positions;
        const long long o = live ? pos / a.inner : 0, k = live ? pos - o * a.inner : 0;
        const T* dy = static_cast<const T*>(a.x) + o * a.px + k;
        const T* v = static_cast<const T*>(a.res) + o * a.pres + k;
        const float mean = live ? a.mean[pos] : 0.f, rstd = live ? a.rstd[pos] : 0.f;
        Pair s{0.f, 0.f};
        for (long long c = warp; live && c < a.features; c += MAP_WARPS) {
            const float g = to_float(dy[c * a.inner]) * (a.weight ? weight_at<T>(a.weight, a.weight_f32, c) : 1.f);
            s.a += g;
            s.b = fmaf(g, (to_float(v[c * a.inner]) - mean) * rstd, s.b);
        }
        s = warps_sum(s, buf);
        const float c1 = s.a / n, c2 = s.b / n;
        T* out = static_cast<T*>(a.out) + o * a.pout + k;
        T* out2 = TAIL ? static_cast<T*>(a.out2) + o * a.pout2 + k : nullptr;
        const T* gsum = TAIL && a.gsum ? static_cast<const T*>(a.gsum) + o * a.pgsum + k : nullptr;
        for (long long c = warp; live && c < a.features; c += MAP_WARPS) {
            const long long at = c * a.inner;
            const float g = to_float(dy[at]) * (a.weight ? weight_at<T>(a.weight, a.weight_f32, c) : 1.f);
            const float h = (to_float(v[at]) - mean) * rstd;
            float d = rstd * (g - c1 - h * c2);
            if (TAIL) {
                if (gsum) d += to_float(gsum[at]);
                out2[at] = from_float<T>(d);
                if (a.dropping) d = mask.dropped_at((uint64_t)(o * a.features * a.inner + at + k)) ? 0.f : d * a.scale;
            }
            out[at] = from_float<T>(d);
        }
    }
}

// Partial sums of the weights' gradients: one feature and a share of the positions per block.
template <class T>
__global__ void __launch_bounds__(256) map_weight_sums(const __grid_constant__ Args a) {
    grid_dependency_wait();
    __shared__ float buf[16];
    const long long c = blockIdx.x, positions = a.outer * a.inner;
    Pair s{0.f, 0.f};
    for (long long pos = (long long)blockIdx.y * 256 + threadIdx.x; pos < positions; pos += (long long)gridDim.y * 256) {
        const long long o = pos / a.inner, k = pos - o * a.inner;
        const float dy = to_float(static_cast<const T*>(a.x)[o * a.px + c * a.inner + k]);
        const float h = (to_float(static_cast<const T*>(a.res)[o * a.pres + c * a.inner + k]) - a.mean[pos]) * a.rstd[pos];
        s.a = fmaf(dy, h, s.a);
        s.b += dy;
    }
    s = block_sum<8>(s, buf);
    if (threadIdx.x < 2) a.part[((long long)blockIdx.y * 2 + threadIdx.x) * a.features + c] = threadIdx.x ? s.b : s.a;
}

// The weights' gradients from the partial sums: 32 features of one of the two per block, whose 32 warps share the parts.  Bound by
// the latency of a few rounds of loads, ten at a time (6 to 8 us for 296 parts; with eight warps, one load at a time, 15).
constexpr int GRAD_WARPS = 32;
template <class T>
__global__ void __launch_bounds__(GRAD_WARPS * 32) weight_grads(const __grid_constant__ Args a, int parts) {
    grid_dependency_wait();
    __shared__ float buf[GRAD_WARPS][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long c0 = (long long)blockIdx.x * 32, c = c0 + lane;
    float t = 0.f;
    if (c < a.features) {
        const float* part = a.part + blockIdx.y * a.features + c;
#pragma unroll 10
        for (int p = warp; p < parts; p += GRAD_WARPS) t += part[(long long)p * 2 * a.features];
    }
    buf[lane][warp] = t;
    __syncthreads();
    // warp f adds up feature f's 32 sums
    t = buf[warp][lane];
    for (int o = 16; o > 0; o >>= 1) t += __shfl_xor_sync(0xffffffffu, t, o);
    void* to = blockIdx.y ? a.gb : a.gw;
    if (lane == 0 && to && c0 + warp < a.features) store_weight_grad<T>(to, a.weight_f32, c0 + warp, t);
}

}  // namespace prior
}  // namespace gleam
