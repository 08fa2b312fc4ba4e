// The three products of a turn, 128 x 128 of the result a block (or a cluster of blocks that share the sum over K):
//
//     GRAM   A = X X^T            POLY   P = b A + c A A            APPLY   X' = a X + P X  (the last one: the result, or the weights)
//
// A and P are symmetric: the blocks below the diagonal and on it are computed and stored on both sides, and A A is A A^T, so that GRAM and
// POLY read both operands the same way.
//
// One warp copies, one thread issues products, all eight warps finish: sums from tensor memory to shared memory, there added over the
// cluster and blended with the old values, which were fetched while the products ran.
#pragma once
#include "launch_overlap.cuh"
#include "ortho_common.cuh"
#include "tensor_core.cuh"

namespace gleam {
namespace ortho {

enum { GRAM, POLY, APPLY, LAST };

constexpr int GEMM_THREADS = 256, STAGES = 3;
// What a product holds.  GRAM and POLY: 64 of K a stage, one block an SM, two sums in turn (each of hi hi and of the rest).  APPLY: few terms, of
// either sign; 32 of K a stage and one sum leave room for a second block on the SM, whose products run while this one finishes (9216 x 1024: 57 -> 46 us).
// LONG: the tensor core cuts a sum off where it adds, by 2^-24 of it on average, which tells in sums whose terms have one sign.  Where a block has
// more than LONG_FROM steps its sums are added up in registers, rounded, after every SPAN at most, and start again at zero; APPLY, whose
// second block would have no registers for that, takes the form of the others then.  130 x 1048576, five turns: off by 6.7e-6 of the result, 6e-4
// without; 4096 x 4096: 7.5e-6, 3.2e-5 without, 3900 us of kernels for 3700.
constexpr int SPAN = 32;                           // steps of 64
template <int KIND> constexpr int LONG_FROM = KIND == GRAM || KIND == POLY ? 56 : 32;
template <int KIND, bool LONG> struct Form {
    static constexpr bool SIDES = KIND == GRAM || KIND == POLY;                // both operands are rows of one matrix
    static constexpr bool ALONE = SIDES || LONG;                               // on the SM
    static constexpr int STEP = ALONE ? 64 : 32, SUMS = ALONE ? 2 : 1, COLUMNS = SUMS * 2 * BLOCK, BLOCKS = ALONE ? 1 : 2;
    static constexpr int OPERAND = 2 * BLOCK * STEP * 2, STAGE = 2 * OPERAND;                   // bytes of an operand's pieces, of both operands
    static constexpr int SMEM = 1024 + STAGES * STAGE;                         // the first KB: barriers
};

// Steps of K, and blocks of a result that are computed.
template <int KIND, bool LONG> __host__ __device__ inline int steps_of(const Args& a) {
    return (int)(((KIND == GRAM ? a.L : a.S) + Form<KIND, LONG>::STEP - 1) / Form<KIND, LONG>::STEP);
}
template <int KIND> __host__ inline int tiles_of(const Args& a) { return KIND == GRAM || KIND == POLY ? a.sblocks * (a.sblocks + 1) / 2 : a.sblocks * a.lblocks; }

// T: the type of results (LAST)
template <int KIND, int RANKS, bool LONG, class T>
__global__ void __launch_bounds__(GEMM_THREADS, Form<KIND, LONG>::BLOCKS) gemm_kernel(const __grid_constant__ Args a, const __grid_constant__ CUtensorMap map) {
    extern __shared__ __align__(1024) unsigned char smem[];
    constexpr int ranks = RANKS, GROUP_ITEMS = BLOCK, GROUPS = BLOCK / 8;         // eights of a row in eight rows; eights of rows
    constexpr int ITEMS = ((GROUPS + RANKS - 1) / RANKS * GROUP_ITEMS + GEMM_THREADS - 1) / GEMM_THREADS;     // eights that a thread finishes at most
    using F = Form<KIND, LONG>;
    constexpr bool SIDES = F::SIDES;
    constexpr int STEP = F::STEP, SUMS = F::SUMS, PARTS_OF_BLOCK = BLOCK / STEP;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = ranks > 1 ? (int)tc::cluster_rank() : 0, m = blockIdx.z;
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
    if (warp == 0) tc::take_columns(base, F::COLUMNS);
    if (warp == 1 && lane == 0) asm volatile("prefetch.tensormap [%0];" ::"l"(&map) : "memory");
    if (threadIdx.x == 0) {
        for (int s = 0; s < 2 * STAGES + 1; ++s) tc::barrier_init(bars + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t sums = *reinterpret_cast<volatile uint32_t*>(smem);
    grid_dependency_wait();

    const int steps = steps_of<KIND, LONG>(a), first = steps * rank / ranks, count = steps * (rank + 1) / ranks - first;
    const long long square = (long long)m * a.sblocks * a.sblocks, wide = (long long)m * a.sblocks * a.lblocks;
    const unsigned char* left = KIND == GRAM ? a.x + wide * BLOCK_BYTES : KIND == POLY ? a.g + square * BLOCK_BYTES : a.p + square * BLOCK_BYTES;
    const unsigned char* right = SIDES ? left : a.x + wide * BLOCK_BYTES;
    const int lblocks = KIND == GRAM ? a.lblocks : a.sblocks;                      // blocks in a row of `left`
    const bool one = SIDES && bi == bj;                                            // the operands are the same
    bool failed = false;

    // what is blended in is fetched while the products run (POLY), or half of it at a time
    constexpr int AHEAD = SIDES ? ITEMS : ITEMS / 2;
    const int g0 = GROUPS * rank / RANKS, g1 = GROUPS * (rank + 1) / RANKS;            // this block's share of the rows, in eights
    const unsigned char* old = KIND == POLY ? a.g + (square + (long long)bi * a.sblocks + bj) * BLOCK_BYTES : a.x + (wide + (long long)bi * a.lblocks + bj) * BLOCK_BYTES;
    uint4 old_hi[AHEAD], old_lo[AHEAD];
    auto row_of = [&](int k) { const int i = g0 * GROUP_ITEMS + k * GEMM_THREADS + threadIdx.x; return (i & 7) + (i >> 7) * 8; };
    auto has = [&](int k) { return RANKS == 1 || k * GEMM_THREADS + (int)threadIdx.x < (g1 - g0) * GROUP_ITEMS; };
    const int col = ((threadIdx.x >> 3) & 15) * 8;
    auto fetch = [&](int k0) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (!has(k0 + k)) break;
            old_hi[k] = *reinterpret_cast<const uint4*>(old + core_at(row_of(k0 + k), col));
            old_lo[k] = *reinterpret_cast<const uint4*>(old + LO + core_at(row_of(k0 + k), col));
        }
    };
    // X = 2^e X^ and its successor (LAST: the result itself): b A and c A A, a X and P X are blended with these
    float old_by = 1.f, sum_by = 1.f;
    auto prepare = [&]() {
        if (KIND == GRAM) return;
        fetch(0);
        Exponent now(a.size[m]);
        for (int k = 0; k < a.turn && now.most <= 0.5f; ++k) now.turn(a);
        Exponent next = now;
        next.turn(a);
        const int to = KIND == LAST ? 0 : next.e;
        old_by = KIND == POLY ? a.b : a.a * power_of_two(now.e - to);
        sum_by = KIND == POLY ? a.c * power_of_two(2 * now.e) : power_of_two(3 * now.e - to);
    };
    // a thread's row and half of the columns of the sums
    auto read_sums = [&](int half, float (&v)[32]) {
        const uint32_t at = sums + ((uint32_t)((warp & 3) * 32) << 16) + (warp >> 2) * 64 + half * 32;
        float t[32];
        tc::read_columns(at, v);
        tc::read_columns(at + BLOCK, t);
        if (SUMS > 1 && count > 1) {
            float u[32];
            tc::read_columns(at + 2 * BLOCK, u);
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] += u[j];
            tc::read_columns(at + 3 * BLOCK, u);
#pragma unroll
            for (int j = 0; j < 32; ++j) t[j] += u[j];
        }
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] += t[j];
    };

    float before[LONG ? 64 : 1] = {};                                              // the sums of the spans before
    const int spans = LONG ? (count + SPAN - 1) / SPAN : 1;
    for (int span = 0;; ++span) {
        const int i0 = LONG ? (int)((long long)count * span / spans) : 0, i1 = LONG ? (int)((long long)count * (span + 1) / spans) : count;
        if (warp == 0 && lane == 0) {
            // rows of cores from the first block to left's and right's
            const long long lrow = (left - a.blocks) / ROW_BYTES + (long long)bi * lblocks * 16, rrow = (right - a.blocks) / ROW_BYTES + (long long)bj * lblocks * 16;
            for (int i = i0; i < i1; ++i) {
                const int s = i % STAGES, k = first + i, kb = k / PARTS_OF_BLOCK, share = k % PARTS_OF_BLOCK;
                if (i >= STAGES && !tc::barrier_wait(empty(s), (i / STAGES - 1) & 1)) { failed = true; break; }
                const uint32_t to = stages + s * F::STAGE;
                tc::barrier_expect(full(s), one ? F::OPERAND : F::STAGE);
#pragma unroll
                for (int h = 0; h < STEP / 32; ++h) {
#pragma unroll
                    for (int piece = 0; piece < 2; ++piece) {                   // 32 columns of 128 rows: 8 KB
                        const uint32_t at = to + h * 16384 + piece * 8192;
                        const int part = piece * 4 + share * (STEP / 32) + h;
                        tc::tiled_copy(at, &map, part, (int)(lrow + kb * 16), full(s));
                        if (SIDES && !one) tc::tiled_copy(at + F::OPERAND, &map, part, (int)(rrow + kb * 16), full(s));
                    }
                }
                if (!SIDES) tc::bulk_copy(to + F::OPERAND, right + ((long long)kb * a.lblocks + bj) * BLOCK_BYTES + share * F::OPERAND, F::OPERAND, full(s));
            }
        } else if (warp == 1 && lane == 0) {
            const uint32_t what = tc::instruction(BLOCK, !SIDES);
            for (int i = i0; i < i1; ++i) {
                const int s = i % STAGES;
                if (!tc::barrier_wait(full(s), (i / STAGES) & 1)) {
                    failed = true;
                    for (int k = i; k < i1 && k < i + STAGES; ++k) tc::barrier_wait(full(k % STAGES), (k / STAGES) & 1);     // copies under way
                    break;
                }
                tc::fence_after();
                const uint32_t l = stages + s * F::STAGE, r = one ? l : l + F::OPERAND, to = sums + (i - i0) % SUMS * 2 * BLOCK;
#pragma unroll
                for (int q = 0; q < STEP / 16; ++q) {
                    // cores of left: 512 bytes from one to the next along M, 128 along K; of right (!SIDES): 128 along N, 4096 along K
                    const uint32_t at = (q >> 1) * 16384 + (q & 1) * 256;
                    const uint64_t lh = tc::descriptor(l + at, 128, 512), ll = tc::descriptor(l + 8192 + at, 128, 512);
                    const uint64_t rh = SIDES ? tc::descriptor(r + at, 128, 512) : tc::descriptor(r + q * 8192, 4096, 128);
                    const uint64_t rl = SIDES ? tc::descriptor(r + 8192 + at, 128, 512) : tc::descriptor(r + LO + q * 8192, 4096, 128);
                    tc::product(to + BLOCK, ll, rh, what, i - i0 >= SUMS || q > 0);
                    tc::product(to + BLOCK, lh, rl, what, true);
                    tc::product(to, lh, rh, what, i - i0 >= SUMS || q > 0);
                }
                tc::commit(empty(s));
            }
            tc::commit(done);
        }
        __syncwarp();
        if (!LONG) prepare();
        if (!tc::barrier_wait(done, span & 1)) failed = true;
        failed = __syncthreads_or(failed);
        tc::fence_after();
        if (!LONG || span + 1 == spans || failed) break;
#pragma unroll
        for (int half = 0; half < (LONG ? 2 : 0); ++half) {
            float v[32];
            read_sums(half, v);
#pragma unroll
            for (int j = 0; j < 32; ++j) before[(LONG ? half * 32 : 0) + (LONG ? j : 0)] += v[j];
        }
        tc::fence_before();
        __syncthreads();                                                           // the next products start the sums again
    }

    // the sums, in units of the stored values; NaN where a wait gave up, and so the results
    float* sum = reinterpret_cast<float*>(smem + 1024);
    const float unit = unit_of(failed);
#pragma unroll (LONG ? 2 : 1)
    for (int half = 0; half < 2; ++half) {
        const int row = (warp & 3) * 32 + lane, c0 = (warp >> 2) * 64 + half * 32;
        float v[32];
        read_sums(half, v);
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = (LONG ? v[j] + before[LONG ? half * 32 + j : 0] : v[j]) * unit;
#pragma unroll
        for (int j = 0; j < 32; j += 4) *reinterpret_cast<float4*>(sum + sum_at(row, c0 + j)) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
    }
    if (LONG) prepare();
    tc::fence_before();
    __syncthreads();
    if (warp == 0) tc::free_columns(sums, F::COLUMNS);
    if (failed && threadIdx.x == 0) atomicOr(a.status, 1);

    // a cluster's blocks add a share of the rows each, lanes along a row as remote reads want it; these rows of a block's own sums are
    // nobody else's
    if (RANKS > 1) {
        tc::cluster_sync();
        constexpr int AT_ONCE = RANKS > 4 ? 2 : RANKS > 2 ? 3 : 4;              // rows in eights whose reads are under way together
        for (int g = g0; g < g1; g += AT_ONCE) {
            float4 f[AT_ONCE][RANKS];
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j)
#pragma unroll
                for (int k = 0; k < RANKS; ++k)
                    if (g + j < g1) f[j][k] = tc::read_remote(base + 1024 + 16 * ((g + j) * 256 + threadIdx.x), k);
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                if (g + j >= g1) break;
#pragma unroll
                for (int k = 1; k < RANKS; ++k) { f[j][0].x += f[j][k].x; f[j][0].y += f[j][k].y; f[j][0].z += f[j][k].z; f[j][0].w += f[j][k].w; }
                reinterpret_cast<float4*>(sum)[(g + j) * 256 + threadIdx.x] = f[j][0];
            }
        }
        tc::cluster_arrive();                      // waited for at the end: nobody leaves while others read its sums
        __syncthreads();
    }
    auto take8 = [&](int r, int c, float (&v)[8]) {
        const float4 f = *reinterpret_cast<const float4*>(sum + sum_at(r, c)), g = *reinterpret_cast<const float4*>(sum + sum_at(r, c + 4));
        v[0] = f.x; v[1] = f.y; v[2] = f.z; v[3] = f.w; v[4] = g.x; v[5] = g.y; v[6] = g.z; v[7] = g.w;
    };
    auto blend = [&](const uint4& hi, const uint4& lo, float (&v)[8]) {
        float u[8];
        join8(hi, lo, u);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fmaf(old_by, u[j], sum_by * v[j]);
    };
    // zeros beyond the matrix
    auto put = [&](unsigned char* block, int r, int c, float (&v)[8], long long rows, long long cols) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (r >= rows || c + j >= cols) v[j] = 0.f;
        uint4 hi, lo;
        split8(v, hi, lo);
        *reinterpret_cast<uint4*>(block + core_at(r, c)) = hi;
        *reinterpret_cast<uint4*>(block + LO + core_at(r, c)) = lo;
    };
    const long long rows = a.S - (long long)bi * BLOCK, cols = (SIDES ? a.S : a.L) - (long long)bj * BLOCK;
    if (KIND != LAST) {
        unsigned char* to = KIND == APPLY ? a.y + (wide + (long long)bi * a.lblocks + bj) * BLOCK_BYTES
                                          : (KIND == GRAM ? a.g : a.p) + (square + (long long)bi * a.sblocks + bj) * BLOCK_BYTES;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            float v[8];
            if (!has(k)) break;
            if (KIND == APPLY && k == AHEAD) fetch(k);
            take8(row_of(k), col, v);
            if (KIND != GRAM) blend(old_hi[k % AHEAD], old_lo[k % AHEAD], v);
            put(to, row_of(k), col, v, rows, cols);
        }
        if (SIDES && !one) {
            // the block on the other side of the diagonal: this block's rows are columns there
            const long long at = (square + (long long)bj * a.sblocks + bi) * BLOCK_BYTES;
            const int eights = RANKS == 1 ? GROUPS : g1 - g0;               // of columns
            auto mirror_row = [&](int k) { const int i = (k * GEMM_THREADS + threadIdx.x) >> 3; return (threadIdx.x & 7) + i / eights * 8; };
            auto mirror_col = [&](int k) { const int i = (k * GEMM_THREADS + threadIdx.x) >> 3; return (g0 + i % eights) * 8; };
            if (KIND == POLY) {
#pragma unroll
                for (int k = 0; k < ITEMS; ++k) {
                    if (!has(k)) break;
                    old_hi[k % AHEAD] = *reinterpret_cast<const uint4*>(a.g + at + core_at(mirror_row(k), mirror_col(k)));
                    old_lo[k % AHEAD] = *reinterpret_cast<const uint4*>(a.g + at + LO + core_at(mirror_row(k), mirror_col(k)));
                }
            }
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                if (!has(k)) break;
                const int r = mirror_row(k), c = mirror_col(k);
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = sum[sum_at(c + j, r)];
                if (KIND == POLY) blend(old_hi[k], old_lo[k], v);
                put((KIND == GRAM ? a.g : a.p) + at, r, c, v, cols, rows);
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            float v[8];
            if (k == AHEAD) fetch(k);
            take8(row_of(k), col, v);
            blend(old_hi[k % AHEAD], old_lo[k % AHEAD], v);
            *reinterpret_cast<float4*>(sum + sum_at(row_of(k), col)) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4*>(sum + sum_at(row_of(k), col + 4)) = make_float4(v[4], v[5], v[6], v[7]);
        }
        __syncthreads();
        // lanes along what is contiguous
        constexpr int AT_ONCE = 16, LINES = GEMM_THREADS / BLOCK;
        const long long s0 = (long long)bi * BLOCK, l0 = (long long)bj * BLOCK;
        const int along = threadIdx.x & (BLOCK - 1), r1 = rows < BLOCK ? (int)rows : BLOCK, c1 = cols < BLOCK ? (int)cols : BLOCK;
        const int limit = along < (a.tall ? r1 : c1) ? (a.tall ? c1 : r1) : 0;
        T* out = static_cast<T*>(a.out[m]) + (a.tall ? l0 * a.cols + s0 : s0 * a.cols + l0) + along;
        const long long step = LINES * a.cols;
        int line = threadIdx.x / BLOCK;
        out += line * a.cols;
        for (; line < BLOCK; line += AT_ONCE * LINES, out += AT_ONCE * step) {
            float w[AT_ONCE], v[AT_ONCE];
            T* p = out;
            if (a.update) {
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k, p += step) w[k] = line + k * LINES < limit ? to_float(*p) : 0.f;
            }
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) v[k] = sum[a.tall ? sum_at(along, line + k * LINES) : sum_at(line + k * LINES, along)] * (1.f / SCALE);
            if (a.update) {
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k) v[k] = fmaf(a.keep, w[k], -a.move * v[k]);
            }
            p = out;
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k, p += step)
                if (line + k * LINES < limit) *p = from_float<T>(v[k]);
        }
    }
    if (ranks > 1) tc::cluster_wait();
}

}  // namespace ortho
}  // namespace gleam
