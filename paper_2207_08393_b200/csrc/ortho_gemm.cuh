// The three products of a turn, 128 x 128 of the result a block (or a cluster of blocks that share the sum over K):
//
//     GRAM   A = X X^T            POLY   P = b A + c A A            APPLY   X' = a X + P X  (the last one: the result, or the weights)
//
// A and P are symmetric: the blocks below the diagonal and on it are computed and stored on both sides, and A A is A A^T, so that GRAM and
// POLY read both operands the same way.
#pragma once
#include "launch_overlap.cuh"
#include "ortho_common.cuh"
#include "tensor_core.cuh"

namespace gleam {
namespace ortho {

enum { GRAM, POLY, APPLY, LAST };

constexpr int GEMM_THREADS = 256, STAGES = 3, STEP = 64;                 // STEP: of K, a stage
constexpr int OPERAND_BYTES = 2 * BLOCK * STEP * 2, STAGE_BYTES = 2 * OPERAND_BYTES;
constexpr int GEMM_SMEM = 1024 + STAGES * STAGE_BYTES;                  // the first KB: barriers
constexpr int SUMS = 3;                                                 // hi hi sums side by side in tensor memory, and one of the rest

// Steps of K, and blocks of a result that are computed.
template <int KIND> __host__ __device__ inline int steps_of(const Args& a) { return (int)(((KIND == GRAM ? a.L : a.S) + STEP - 1) / STEP); }
template <int KIND> __host__ inline int tiles_of(const Args& a) { return KIND == GRAM || KIND == POLY ? a.sblocks * (a.sblocks + 1) / 2 : a.sblocks * a.lblocks; }

// The sums as 32-bit numbers in shared memory: rows of 128, their 16-byte pieces in an order that keeps 32 rows apart.
__device__ __forceinline__ int sum_at(int r, int c) { return r * BLOCK + ((((c >> 2) ^ r) & 31) << 2) + (c & 3); }

template <int KIND>
__global__ void __launch_bounds__(GEMM_THREADS, 1) gemm_kernel(const __grid_constant__ Args a) {
    extern __shared__ __align__(1024) unsigned char smem[];
    constexpr bool SIDES = KIND == GRAM || KIND == POLY;               // both operands are rows of one matrix
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, ranks = gridDim.x, rank = ranks > 1 ? (int)tc::cluster_rank() : 0, m = blockIdx.z;
    int bi, bj;
    if (SIDES) {
        bi = 0;
        while ((bi + 1) * (bi + 2) / 2 <= (int)blockIdx.y) ++bi;
        bj = (int)blockIdx.y - bi * (bi + 1) / 2;
    } else {
        bi = (int)blockIdx.y % a.sblocks; bj = (int)blockIdx.y / a.sblocks;
    }
    const uint32_t base = tc::shared_address(smem), bars = base + 16, stages = base + 1024;      // [0]: tensor memory, bars: full, empty, done
    auto full = [&](int s) { return bars + 8 * s; };
    auto empty = [&](int s) { return bars + 8 * (STAGES + s); };
    const uint32_t done = bars + 16 * STAGES;
    if (warp == 0) tc::take_columns(base, 512);
    if (threadIdx.x == 0) {
        for (int s = 0; s < 2 * STAGES + 1; ++s) tc::barrier_init(bars + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t sums = *reinterpret_cast<volatile uint32_t*>(smem);
    grid_dependency_wait();

    const int steps = steps_of<KIND>(a), first = steps * rank / ranks, count = steps * (rank + 1) / ranks - first;
    const long long square = (long long)m * a.sblocks * a.sblocks, wide = (long long)m * a.sblocks * a.lblocks;
    const unsigned char* left = KIND == GRAM ? a.x + wide * BLOCK_BYTES : KIND == POLY ? a.g + square * BLOCK_BYTES : a.p + square * BLOCK_BYTES;
    const unsigned char* right = SIDES ? left : a.x + wide * BLOCK_BYTES;
    const int lblocks = KIND == GRAM ? a.lblocks : a.sblocks;                      // blocks in a row of `left`
    const bool one = SIDES && bi == bj;                                            // the operands are the same
    bool failed = false;

    if (warp == 0) {
        // 16 runs of 1 KB for each piece of an operand: half the columns (left; right of SIDES) or half the rows of a block
        for (int i = 0; i < count; ++i) {
            const int s = i % STAGES, k = first + i, kb = k >> 1, half = k & 1, piece = lane >> 4, run = lane & 15;
            if (i >= STAGES && !tc::barrier_wait(empty(s), (i / STAGES - 1) & 1)) { failed = true; break; }
            const uint32_t to = stages + s * STAGE_BYTES + piece * (OPERAND_BYTES / 2) + run * 1024;
            if (lane == 0) tc::barrier_expect(full(s), one ? OPERAND_BYTES : STAGE_BYTES);
            __syncwarp();
            tc::bulk_copy(to, left + ((long long)bi * lblocks + kb) * BLOCK_BYTES + piece * PIECE_BYTES + run * 2048 + half * 1024, 1024, full(s));
            if (SIDES) {
                if (!one) tc::bulk_copy(to + OPERAND_BYTES, right + ((long long)bj * lblocks + kb) * BLOCK_BYTES + piece * PIECE_BYTES + run * 2048 + half * 1024, 1024, full(s));
            } else {
                tc::bulk_copy(to + OPERAND_BYTES, right + ((long long)kb * a.lblocks + bj) * BLOCK_BYTES + piece * PIECE_BYTES + half * (PIECE_BYTES / 2) + run * 1024, 1024, full(s));
            }
        }
    } else if (warp == 1 && lane == 0) {
        const uint32_t what = tc::instruction(BLOCK, !SIDES);
        for (int i = 0; i < count; ++i) {
            const int s = i % STAGES;
            if (!tc::barrier_wait(full(s), (i / STAGES) & 1)) {
                failed = true;
                for (int k = i; k < count && k < i + STAGES; ++k) tc::barrier_wait(full(k % STAGES), (k / STAGES) & 1);     // copies under way
                break;
            }
            tc::fence_after();
            const uint32_t l = stages + s * STAGE_BYTES, r = one ? l : l + OPERAND_BYTES;
            constexpr int HALF = OPERAND_BYTES / 2;                                 // from hi to lo
#pragma unroll
            for (int q = 0; q < STEP / 16; ++q) {
                // cores of left: 1024 bytes from one to the next along M, 128 along K; of right (!SIDES): 128 along N, 2048 along K
                const uint64_t lh = tc::descriptor(l + q * 256, 128, 1024), ll = tc::descriptor(l + HALF + q * 256, 128, 1024);
                const uint64_t rh = SIDES ? tc::descriptor(r + q * 256, 128, 1024) : tc::descriptor(r + q * 4096, 2048, 128);
                const uint64_t rl = SIDES ? tc::descriptor(r + HALF + q * 256, 128, 1024) : tc::descriptor(r + HALF + q * 4096, 2048, 128);
                tc::product(sums + SUMS * BLOCK, ll, rh, what, i > 0 || q > 0);
                tc::product(sums + SUMS * BLOCK, lh, rl, what, true);
                tc::product(sums + i % SUMS * BLOCK, lh, rh, what, i >= SUMS || q > 0);
            }
            tc::commit(empty(s));
        }
        tc::commit(done);
    }
    __syncwarp();
    if (count > 0 && !tc::barrier_wait(done, 0)) failed = true;
    tc::fence_after();

    // the sums, in units of the stored values
    float* sum = reinterpret_cast<float*>(smem + 1024);
    {
        const int row = (warp & 3) * 32 + lane;
#pragma unroll 1
        for (int c0 = (warp >> 2) * 64; c0 < (warp >> 2) * 64 + 64; c0 += 32) {
            const uint32_t at = sums + ((uint32_t)((warp & 3) * 32) << 16) + c0;
            float v[32], t[32];
            if (count > 0) {
                tc::read_columns(at, v);
#pragma unroll 1
                for (int k = 1; k < SUMS && k < count; ++k) {
                    tc::read_columns(at + k * BLOCK, t);
#pragma unroll
                    for (int j = 0; j < 32; ++j) v[j] += t[j];
                }
                tc::read_columns(at + SUMS * BLOCK, t);
            }
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
                float4 f;
                f.x = count > 0 ? (v[j] + t[j]) * (1.f / SCALE) : 0.f; f.y = count > 0 ? (v[j + 1] + t[j + 1]) * (1.f / SCALE) : 0.f;
                f.z = count > 0 ? (v[j + 2] + t[j + 2]) * (1.f / SCALE) : 0.f; f.w = count > 0 ? (v[j + 3] + t[j + 3]) * (1.f / SCALE) : 0.f;
                *reinterpret_cast<float4*>(sum + sum_at(row, c0 + j)) = f;
            }
        }
    }
    tc::fence_before();
    __syncthreads();
    if (warp == 0) tc::free_columns(sums, 512);
    if (failed) atomicOr(a.status, 1);
    if (ranks > 1) tc::cluster_sync();

    // eight columns of a row, summed over the cluster
    auto take = [&](int r, int c, float (&v)[8]) {
        float4 f[2];
        const uint32_t at[2] = {base + 1024 + 4 * sum_at(r, c), base + 1024 + 4 * sum_at(r, c + 4)};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f[h] = ranks > 1 ? tc::read_remote(at[h], 0) : *reinterpret_cast<const float4*>(smem + (at[h] - base));
            for (int k = 1; k < ranks; ++k) {
                const float4 g = tc::read_remote(at[h], k);
                f[h].x += g.x; f[h].y += g.y; f[h].z += g.z; f[h].w += g.w;
            }
        }
        v[0] = f[0].x; v[1] = f[0].y; v[2] = f[0].z; v[3] = f[0].w; v[4] = f[1].x; v[5] = f[1].y; v[6] = f[1].z; v[7] = f[1].w;
    };
    auto blend = [&](const unsigned char* block, int r, int c, float by, float (&v)[8], float times) {
        float u[8];
        join8(*reinterpret_cast<const uint4*>(block + core_at(r, c)), *reinterpret_cast<const uint4*>(block + PIECE_BYTES + core_at(r, c)), u);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fmaf(by, u[j], times * v[j]);
    };
    auto put = [&](unsigned char* block, int r, int c, const float (&v)[8]) {
        uint4 hi, lo;
        split8(v, hi, lo);
        *reinterpret_cast<uint4*>(block + core_at(r, c)) = hi;
        *reinterpret_cast<uint4*>(block + PIECE_BYTES + core_at(r, c)) = lo;
    };
    const int items = BLOCK * BLOCK / 8 / ranks;
    if (KIND != LAST) {
        const unsigned char* old = KIND == POLY ? a.g + (square + (long long)bi * a.sblocks + bj) * BLOCK_BYTES : a.x + (wide + (long long)bi * a.lblocks + bj) * BLOCK_BYTES;
        unsigned char* to = KIND == APPLY ? a.y + (wide + (long long)bi * a.lblocks + bj) * BLOCK_BYTES
                                          : (KIND == GRAM ? a.g : a.p) + (square + (long long)bi * a.sblocks + bj) * BLOCK_BYTES;
        for (int i = rank * items + threadIdx.x; i < (rank + 1) * items; i += GEMM_THREADS) {
            const int r = (i & 7) + (i >> 7) * 8, c = ((i >> 3) & 15) * 8;
            float v[8];
            take(r, c, v);
            if (KIND == POLY) blend(old, r, c, a.b, v, a.c);
            if (KIND == APPLY) blend(old, r, c, a.a, v, 1.f);
            put(to, r, c, v);
        }
        if (SIDES && !one) {
            // the block on the other side of the diagonal
            const unsigned char* mirror = a.g + (square + (long long)bj * a.sblocks + bi) * BLOCK_BYTES;
            unsigned char* over = (KIND == GRAM ? a.g : a.p) + (square + (long long)bj * a.sblocks + bi) * BLOCK_BYTES;
            for (int i = rank * items + threadIdx.x; i < (rank + 1) * items; i += GEMM_THREADS) {
                const int r = (i & 7) + (i >> 7) * 8, c = ((i >> 3) & 15) * 8;
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t at = base + 1024 + 4 * (sum_at(c + j, r) & ~3);
                    float s = 0.f;
                    for (int k = 0; k < ranks; ++k) {
                        const float4 f = ranks > 1 ? tc::read_remote(at, k) : *reinterpret_cast<const float4*>(smem + (at - base));
                        const float g = (r & 3) == 0 ? f.x : (r & 3) == 1 ? f.y : (r & 3) == 2 ? f.z : f.w;
                        s = k == 0 ? g : s + g;
                    }
                    v[j] = s;
                }
                if (KIND == POLY) blend(mirror, r, c, a.b, v, a.c);
                put(over, r, c, v);
            }
        }
    } else {
        const unsigned char* old = a.x + (wide + (long long)bi * a.lblocks + bj) * BLOCK_BYTES;
        const long long s0 = (long long)bi * BLOCK, l0 = (long long)bj * BLOCK;
        auto finish = [&](long long at, float v) {
            v *= 1.f / SCALE;
            if (a.update) v = fmaf(a.keep, load_as(a.out[m], a.dtype, at), -a.move * v);
            store_as(a.out[m], a.dtype, at, v);
        };
        for (int i = threadIdx.x; i < BLOCK * BLOCK / 8; i += GEMM_THREADS) {
            const int r = a.tall ? (i & 7) + (i >> 7) * 8 : i >> 4, c = a.tall ? ((i >> 3) & 15) * 8 : (i & 15) * 8;
            float v[8];
            take(r, c, v);
            blend(old, r, c, a.a, v, 1.f);
            if (a.tall) {
                *reinterpret_cast<float4*>(sum + sum_at(r, c)) = make_float4(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<float4*>(sum + sum_at(r, c + 4)) = make_float4(v[4], v[5], v[6], v[7]);
            } else if (s0 + r < a.S) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (l0 + c + j < a.L) finish((s0 + r) * a.cols + l0 + c + j, v[j]);
            }
        }
        if (a.tall) {
            __syncthreads();
            for (int i = threadIdx.x; i < BLOCK * BLOCK; i += GEMM_THREADS) {
                const int s = i & (BLOCK - 1), l = i / BLOCK;
                if (s0 + s < a.S && l0 + l < a.L) finish((l0 + l) * a.cols + s0 + s, sum[sum_at(s, l)]);
            }
        }
    }
    if (ranks > 1) tc::cluster_sync();             // nobody leaves while others read its sums
}

}  // namespace ortho
}  // namespace gleam
