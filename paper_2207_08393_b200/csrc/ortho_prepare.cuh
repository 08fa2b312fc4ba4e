// The momentum, the norm, and the first X in pieces.
#pragma once
#include "launch_overlap.cuh"
#include "ortho_common.cuh"

namespace gleam {
namespace ortho {

constexpr int PREPARE_THREADS = 256;

// momentum <- mu momentum + gradient, and sums of squares of what is orthogonalised, in a fixed order.
template <class T, bool UPDATE>
__global__ void __launch_bounds__(PREPARE_THREADS) sums_kernel(const __grid_constant__ Args a) {
    grid_dependency_wait();
    const int m = blockIdx.y;
    if (blockIdx.x == 0 && m == 0 && threadIdx.x == 0) *a.status = 0;
    constexpr int AT_ONCE = 8;
    const long long n = a.rows * a.cols, step = (long long)gridDim.x * PREPARE_THREADS;
    float sum = 0.f;
    for (long long i0 = (long long)blockIdx.x * PREPARE_THREADS + threadIdx.x; i0 < n; i0 += AT_ONCE * step) {
        float v[AT_ONCE], w[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const long long i = i0 + k * step;
            v[k] = i < n ? load_at<T>(a.u[m], i) : 0.f;
            if (UPDATE) w[k] = i < n ? a.momentum[m][i] : 0.f;
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            if (UPDATE) {
                w[k] = fmaf(a.mu, w[k], v[k]);
                if (i0 + k * step < n) a.momentum[m][i0 + k * step] = w[k];
                v[k] = a.nesterov ? fmaf(a.mu, w[k], v[k]) : w[k];
            }
            sum = fmaf(v[k], v[k], sum);
        }
    }
    __shared__ float buf[2 * (PREPARE_THREADS / 32)];
    const prior::Pair t = prior::block_sum<PREPARE_THREADS / 32>(prior::Pair{sum, 0.f}, buf);
    if (threadIdx.x == 0) a.part[m * PARTS + blockIdx.x] = t.a;
}

// One block of X_0 = U / (|U| + eps), in pieces.
template <class T, bool UPDATE>
__global__ void __launch_bounds__(PREPARE_THREADS) first_kernel(const __grid_constant__ Args a) {
    grid_dependency_wait();
    extern __shared__ float tile[];                  // a block in 32 bits
    const int m = blockIdx.y, sb = blockIdx.x / a.lblocks, lb = blockIdx.x % a.lblocks;
    float total = 0.f;
    for (int k = threadIdx.x; k < a.parts; k += PREPARE_THREADS) total += a.part[m * PARTS + k];
    __shared__ float buf[2 * (PREPARE_THREADS / 32)];
    total = prior::block_sum<PREPARE_THREADS / 32>(prior::Pair{total, 0.f}, buf).a;
    const float by = SCALE / (sqrtf(total) + a.eps);
    unsigned char* block = a.x + ((long long)(m * a.sblocks + sb) * a.lblocks + lb) * BLOCK_BYTES;
    const long long s0 = (long long)sb * BLOCK, l0 = (long long)lb * BLOCK;
    const int rows = a.S - s0 < BLOCK ? (int)(a.S - s0) : BLOCK, cols = a.L - l0 < BLOCK ? (int)(a.L - l0) : BLOCK;
    // lanes along what is contiguous
    constexpr int AT_ONCE = 16, LINES = PREPARE_THREADS / BLOCK;
    const int along = threadIdx.x & (BLOCK - 1), limit = along < (a.tall ? rows : cols) ? (a.tall ? cols : rows) : 0;
    const long long corner = (a.tall ? l0 * a.cols + s0 : s0 * a.cols + l0) + along;
    const T* u = static_cast<const T*>(a.u[m]) + corner;
    const float* momentum = UPDATE ? a.momentum[m] + corner : nullptr;
    for (int line = threadIdx.x / BLOCK; line < BLOCK; line += AT_ONCE * LINES) {
        float v[AT_ONCE], w[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int n = line + k * LINES;
            v[k] = n < limit && (!UPDATE || a.nesterov) ? to_float(u[n * a.cols]) : 0.f;
            if (UPDATE) w[k] = n < limit ? momentum[n * a.cols] : 0.f;
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int n = line + k * LINES;
            if (UPDATE) v[k] = a.nesterov ? fmaf(a.mu, w[k], v[k]) : w[k];
            tile[a.tall ? sum_at(along, n) : sum_at(n, along)] = v[k] * by;
        }
    }
    __syncthreads();
#pragma unroll 2
    for (int i = threadIdx.x; i < BLOCK * BLOCK / 8; i += PREPARE_THREADS) {
        // eight lanes a core: rows of 16 bytes that lie side by side
        const int r = (i & 7) + (i >> 7) * 8, c = ((i >> 3) & 15) * 8;
        const float4 f = *reinterpret_cast<const float4*>(tile + sum_at(r, c)), g = *reinterpret_cast<const float4*>(tile + sum_at(r, c + 4));
        const float v[8] = {f.x, f.y, f.z, f.w, g.x, g.y, g.z, g.w};
        uint4 hi, lo;
        split8(v, hi, lo);
        *reinterpret_cast<uint4*>(block + core_at(r, c)) = hi;
        *reinterpret_cast<uint4*>(block + PIECE_BYTES + core_at(r, c)) = lo;
    }
}

}  // namespace ortho
}  // namespace gleam
