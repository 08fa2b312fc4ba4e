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
    if (a.fresh && blockIdx.x == 0 && m == 0 && threadIdx.x == 0) *a.status = 0;
    const long long n = a.rows * a.cols, step = (long long)gridDim.x * PREPARE_THREADS;
    const T* u = static_cast<const T*>(a.u[m]);
    float* momentum = UPDATE ? a.momentum[m] : nullptr;
    float sum = 0.f;
    auto one = [&](float g, float& w) {
        w = fmaf(a.mu, w, g);
        return a.nesterov ? fmaf(a.mu, w, g) : w;
    };
    // pieces of 16 bytes where both arrays start at them, then what is left
    constexpr int V = prior::VEC<T>, AT_ONCE = UPDATE ? 2 : 4;
    const bool packed = ((uintptr_t)u | (uintptr_t)momentum) % 16 == 0;
    const long long pieces = packed ? n / V : 0, first = (long long)blockIdx.x * PREPARE_THREADS + threadIdx.x;
    for (long long i0 = first; i0 < pieces; i0 += AT_ONCE * step) {
        prior::Pack<T> g[AT_ONCE];
        float4 w[AT_ONCE][V / 4];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const long long i = i0 + k * step;
            if (i >= pieces) break;
            g[k] = prior::load_pack(u + i * V);
            if (UPDATE) {
#pragma unroll
                for (int j = 0; j < V / 4; ++j) w[k][j] = reinterpret_cast<const float4*>(momentum)[i * (V / 4) + j];
            }
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const long long i = i0 + k * step;
            if (i >= pieces) break;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float v = to_float(g[k].e[j]);
                if (UPDATE) v = one(v, reinterpret_cast<float*>(&w[k][0])[j]);
                sum = fmaf(v, v, sum);
            }
            if (UPDATE) {
#pragma unroll
                for (int j = 0; j < V / 4; ++j) reinterpret_cast<float4*>(momentum)[i * (V / 4) + j] = w[k][j];
            }
        }
    }
    for (long long i = pieces * V + first; i < n; i += step) {
        float v = to_float(u[i]);
        if (UPDATE) {
            float w = momentum[i];
            v = one(v, w);
            momentum[i] = w;
        }
        sum = fmaf(v, v, sum);
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
    const float by = first_scale(total, a.eps);
    if (blockIdx.x == 0 && threadIdx.x == 0) a.size[m] = first_size(total, a.eps);
    unsigned char* block = a.x + ((long long)(m * a.sblocks + sb) * a.lblocks + lb) * BLOCK_BYTES;
    const long long s0 = (long long)sb * BLOCK, l0 = (long long)lb * BLOCK;
    const int rows = a.S - s0 < BLOCK ? (int)(a.S - s0) : BLOCK, cols = a.L - l0 < BLOCK ? (int)(a.L - l0) : BLOCK;
    // lanes along what is contiguous; of wide matrices four neighbours each where lines begin at four numbers' bytes (tall ones' would meet in
    // the banks of the tile: 25 -> 30 us for 9216 x 1024)
    const int width = a.tall ? rows : cols, height = a.tall ? cols : rows;
    const long long corner = a.tall ? l0 * a.cols + s0 : s0 * a.cols + l0;
    const T* u = static_cast<const T*>(a.u[m]) + corner;
    const float* momentum = UPDATE ? a.momentum[m] + corner : nullptr;
    auto value = [&](float g, float w) { return !UPDATE ? g : a.nesterov ? fmaf(a.mu, w, g) : w; };
    if (!a.tall && a.cols % 4 == 0 && (uintptr_t)a.u[m] % (4 * sizeof(T)) == 0 && (!UPDATE || (uintptr_t)a.momentum[m] % 16 == 0)) {
        struct alignas(4 * sizeof(T)) Four { T e[4]; };
        constexpr int AT_ONCE = 8, LINES = PREPARE_THREADS / 32;
        const int along = (threadIdx.x & 31) * 4;
        for (int line = threadIdx.x >> 5; line < BLOCK; line += AT_ONCE * LINES) {
            Four g[AT_ONCE];
            float4 w[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const int n = line + k * LINES;
                if (n >= height || along >= width) continue;               // lines are whole numbers of fours
                g[k] = *reinterpret_cast<const Four*>(u + n * a.cols + along);
                if (UPDATE) w[k] = *reinterpret_cast<const float4*>(momentum + n * a.cols + along);
            }
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const int n = line + k * LINES;
                const bool there = n < height && along < width;
                float v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = there ? by * value(to_float(g[k].e[j]), UPDATE ? reinterpret_cast<const float*>(&w[k])[j] : 0.f) : 0.f;
                *reinterpret_cast<float4*>(tile + sum_at(n, along)) = make_float4(v[0], v[1], v[2], v[3]);
            }
        }
    } else {
        constexpr int AT_ONCE = 16, LINES = PREPARE_THREADS / BLOCK;
        const int along = threadIdx.x & (BLOCK - 1), limit = along < width ? height : 0;
        for (int line = threadIdx.x / BLOCK; line < BLOCK; line += AT_ONCE * LINES) {
            float v[AT_ONCE], w[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const int n = line + k * LINES;
                v[k] = n < limit ? to_float(u[n * a.cols + along]) : 0.f;
                w[k] = UPDATE && n < limit ? momentum[n * a.cols + along] : 0.f;
            }
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) tile[a.tall ? sum_at(along, line + k * LINES) : sum_at(line + k * LINES, along)] = by * value(v[k], w[k]);
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
        *reinterpret_cast<uint4*>(block + LO + core_at(r, c)) = lo;
    }
}

}  // namespace ortho
}  // namespace gleam
