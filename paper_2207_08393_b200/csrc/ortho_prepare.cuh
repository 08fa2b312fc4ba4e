// The momentum, the norm, and the first X in pieces.
#pragma once
#include "launch_overlap.cuh"
#include "ortho_common.cuh"

namespace gleam {
namespace ortho {

constexpr int PREPARE_THREADS = 256;

// What is orthogonalised: the matrix itself, or gradient and momentum.
template <class T, bool UPDATE>
__device__ __forceinline__ float source(const Args& a, int m, long long i) {
    if (!UPDATE) return load_at<T>(a.u[m], i);
    const float v = a.momentum[m][i];
    return a.nesterov ? fmaf(a.mu, v, load_at<T>(a.u[m], i)) : v;
}

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
    extern __shared__ float tile[];                  // tall: 128 columns of the block with one number between them
    const int m = blockIdx.y, sb = blockIdx.x / a.lblocks, lb = blockIdx.x % a.lblocks;
    float total = 0.f;
    for (int k = threadIdx.x; k < a.parts; k += PREPARE_THREADS) total += a.part[m * PARTS + k];
    __shared__ float buf[2 * (PREPARE_THREADS / 32)];
    total = prior::block_sum<PREPARE_THREADS / 32>(prior::Pair{total, 0.f}, buf).a;
    const float by = SCALE / (sqrtf(total) + a.eps);
    unsigned char* block = a.x + ((long long)(m * a.sblocks + sb) * a.lblocks + lb) * BLOCK_BYTES;
    const long long s0 = (long long)sb * BLOCK, l0 = (long long)lb * BLOCK;
    if (a.tall) {
#pragma unroll 8
        for (int i = threadIdx.x; i < BLOCK * BLOCK; i += PREPARE_THREADS) {
            const int l = i / BLOCK, s = i % BLOCK;
            tile[l * (BLOCK + 1) + s] = s0 + s < a.S && l0 + l < a.L ? source<T, UPDATE>(a, m, (l0 + l) * a.cols + s0 + s) : 0.f;
        }
        __syncthreads();
    }
#pragma unroll 2
    for (int i = threadIdx.x; i < BLOCK * BLOCK / 8; i += PREPARE_THREADS) {
        // eight lanes a core: rows of 16 bytes that lie side by side
        const int r = (i & 7) + (i >> 7) * 8, c = ((i >> 3) & 15) * 8;
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (a.tall) v[j] = tile[(c + j) * (BLOCK + 1) + r];
            else v[j] = s0 + r < a.S && l0 + c + j < a.L ? source<T, UPDATE>(a, m, (s0 + r) * a.cols + l0 + c + j) : 0.f;
            v[j] *= by;
        }
        uint4 hi, lo;
        split8(v, hi, lo);
        *reinterpret_cast<uint4*>(block + core_at(r, c)) = hi;
        *reinterpret_cast<uint4*>(block + PIECE_BYTES + core_at(r, c)) = lo;
    }
}

}  // namespace ortho
}  // namespace gleam
