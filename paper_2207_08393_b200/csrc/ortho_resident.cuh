// The whole update of a matrix whose shorter side is at most 128 in one launch: a cluster of up to sixteen blocks keeps X in shared memory
// through all turns.
//
// A block holds up to seven tiles of 128 columns of X (all R rows of them, R = S rounded up to 16) as pieces.  In a turn it
//   - sums X X^T over its tiles on the tensor cores; the blocks add their sums through distributed shared memory, each a share of the
//     rows, and write the pieces of A to all;
//   - computes P = b A + c A A, which costs less than sharing it;
//   - replaces its tiles by a X + P X.
// Two barriers of the cluster a turn, nothing but the matrix itself through global memory, once each way.  32 x 100 x 900 float32 in clusters of
// four with two tiles a block: 76 us, a turn 22,000 cycles, of which products a third (64 cycles an instruction for N = 128, hardly fewer
// for less, so tiles are laid out for N = 128); the sums of A and its pieces on their way
// through the cluster, at 10 to 14 bytes a cycle, another; the rest brings sums from tensor memory back as pieces.  Issuing the next
// turn's X X^T tile by tile while the other tile is stored gained nothing.
#pragma once
#include "ortho_gemm.cuh"

namespace gleam {
namespace ortho {

constexpr int RESIDENT_THREADS = 512, RESIDENT_RANKS = 16, RESIDENT_PORTABLE = 8, RESIDENT_HEAD = 1024;
constexpr int RESIDENT_LEAST = 120 * 1024;       // shared memory that keeps a second block, which would wait for tensor memory, off the SM
constexpr int RESIDENT_MOST = 227 * 1024;

// Shared memory: head, tiles, A (then P), sums in 32 bits.  A product reads 128 rows of an operand whatever R is: into what stands behind
// it, up to (128 - R) * 256 bytes, for rows of the result that nobody takes.
__host__ __device__ inline int resident_rows(long long S) { return (int)((S + 15) / 16 * 16); }
__host__ inline int resident_bytes(int R, int tiles) {
    const int beyond = (BLOCK - R) * 256 - R * 512, n = RESIDENT_HEAD + (2 + tiles) * R * 512 + (beyond > 0 ? beyond : 0);
    return n < RESIDENT_LEAST ? RESIDENT_LEAST : n;
}

template <class T, bool UPDATE>
__global__ void __launch_bounds__(RESIDENT_THREADS, 1) resident_kernel(const __grid_constant__ Args a, int tiles, int turns) {
    extern __shared__ __align__(1024) unsigned char smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, ranks = gridDim.x, rank = ranks > 1 ? (int)tc::cluster_rank() : 0, m = blockIdx.y;
    const int R = resident_rows(a.S), square = R * 512;                    // bytes of R rows of 128 as pieces, or in 32 bits
    const uint32_t base = tc::shared_address(smem), done = base + 16, second = base + 24;
    unsigned char* X = smem + RESIDENT_HEAD;
    unsigned char* A_ = X + tiles * square;
    float* sum = reinterpret_cast<float*>(A_ + square);
    float* part = reinterpret_cast<float*>(smem + 64);                     // a rank's sum of squares; the block's sums behind it
    float* blends = reinterpret_cast<float*>(smem + 192);                  // of two turns, the norm's bound behind them
    const uint32_t x_at = base + RESIDENT_HEAD, a_at = x_at + tiles * square, sum_from = a_at + square;
    if (warp == 0) tc::take_columns(base, 512);
    if (threadIdx.x == 0) {
        tc::barrier_init(done, 1);
        tc::barrier_init(second, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t cols0 = *reinterpret_cast<volatile uint32_t*>(smem);    // tensor memory: two results, of two sums each
    grid_dependency_wait();

    const long long first = (long long)rank * tiles;                       // this block's tiles
    const int mine = (int)((a.L + BLOCK - 1) / BLOCK - first < tiles ? (a.L + BLOCK - 1) / BLOCK - first : tiles);
    bool failed = false;
    uint32_t phase = 0, second_phase = 0;
    if (a.fresh && threadIdx.x == 0 && m == 0 && rank == 0) *a.status = 0;

    // byte of element (r, c) of a piece of R rows
    auto at = [&](int r, int c) { return (r >> 3) * 2048 + (c >> 3) * CORE + (r & 7) * 16; };
    const int lo = R * 256;                                                // from hi to lo
    auto wait = [&](uint32_t bar, uint32_t& turns_of) {
        if (!failed && !tc::barrier_wait(bar, turns_of)) failed = true;
        turns_of ^= 1;
        tc::fence_after();
    };
    // shared memory written by threads is there for the products; tensor memory that was read may be written
    auto settle = [&]() {
        tc::fence_shared();
        tc::fence_before();
        __syncthreads();
        tc::fence_after();
    };

    // the source in 32 bits where its tile will stand, and the sum of squares
    float squares = 0.f;
    // Elements of a tile: lanes along what is contiguous in the matrix, four lines at a time.
    constexpr int AT_ONCE = 16, LINES = RESIDENT_THREADS / BLOCK;
    const int along = threadIdx.x & (BLOCK - 1), line0 = threadIdx.x / BLOCK, lines = a.tall ? BLOCK : R;
    auto spot = [&](int line) { return a.tall ? sum_at(along, line) : sum_at(line, along); };
    for (int t = 0; t < mine; ++t) {
        float* to = reinterpret_cast<float*>(X + t * square);
        const long long l0 = (first + t) * BLOCK;
        const int width = a.L - l0 < BLOCK ? (int)(a.L - l0) : BLOCK, limit = along < (a.tall ? (int)a.S : width) ? (a.tall ? width : (int)a.S) : 0;
        const long long corner = (a.tall ? l0 * a.cols : l0) + along;
        const T* from = static_cast<const T*>(a.u[m]) + corner;
        float* momentum = UPDATE ? a.momentum[m] + corner : nullptr;
        const long long step = LINES * a.cols;
        from += line0 * a.cols;
        if (UPDATE) momentum += line0 * a.cols;
        for (int line = line0; line < lines; line += AT_ONCE * LINES, from += AT_ONCE * step, momentum += UPDATE ? AT_ONCE * step : 0) {
            float v[AT_ONCE], w[AT_ONCE];
            const T* p = from;
            float* q = momentum;
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k, p += step, q += UPDATE ? step : 0) {
                v[k] = line + k * LINES < limit ? to_float(*p) : 0.f;
                if (UPDATE) w[k] = line + k * LINES < limit ? *q : 0.f;
            }
            if (UPDATE) {
                q = momentum;
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k, q += step) {
                    w[k] = fmaf(a.mu, w[k], v[k]);
                    if (line + k * LINES < limit) *q = w[k];
                    v[k] = a.nesterov ? fmaf(a.mu, w[k], v[k]) : w[k];
                }
            }
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const int n = line + k * LINES;
                squares = fmaf(v[k], v[k], squares);
                if (n < lines && (!a.tall || along < R)) to[spot(n)] = v[k];
            }
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) squares += __shfl_xor_sync(0xffffffffu, squares, o);
    if (lane == 0) part[4 + warp] = squares;
    __syncthreads();
    if (threadIdx.x == 0) {
        float s = 0.f;
        for (int k = 0; k < RESIDENT_THREADS / 32; ++k) s += part[4 + k];
        part[0] = s;
    }
    if (ranks > 1) tc::cluster_sync(); else __syncthreads();
    float total = 0.f;
    for (int k = 0; k < ranks; ++k) total += ranks > 1 ? tc::read_remote(base + 64, k).x : part[0];
    const float by = first_scale(total, a.eps);

    // ... and as pieces
    const int eights = R * BLOCK / 8;
    for (int t = 0; t < mine; ++t) {
        constexpr int MOST = BLOCK * BLOCK / 8 / RESIDENT_THREADS;
        float v[MOST][8];
        unsigned char* tile = X + t * square;
        const float* from = reinterpret_cast<const float*>(tile);
#pragma unroll
        for (int k = 0; k < MOST; ++k) {
            const int i = threadIdx.x + k * RESIDENT_THREADS, r = (i & 7) + (i >> 7) * 8, c = ((i >> 3) & 15) * 8;
            if (i < eights) {
                const float4 f = *reinterpret_cast<const float4*>(from + sum_at(r, c)), g = *reinterpret_cast<const float4*>(from + sum_at(r, c + 4));
                v[k][0] = f.x * by; v[k][1] = f.y * by; v[k][2] = f.z * by; v[k][3] = f.w * by;
                v[k][4] = g.x * by; v[k][5] = g.y * by; v[k][6] = g.z * by; v[k][7] = g.w * by;
            }
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < MOST; ++k) {
            const int i = threadIdx.x + k * RESIDENT_THREADS, r = (i & 7) + (i >> 7) * 8, c = ((i >> 3) & 15) * 8;
            if (i < eights) {
                uint4 h, l;
                split8(v[k], h, l);
                *reinterpret_cast<uint4*>(tile + at(r, c)) = h;
                *reinterpret_cast<uint4*>(tile + lo + at(r, c)) = l;
            }
        }
    }

    // a warp's part of a result: 32 rows, 32 columns
    const int row = (warp & 3) * 32 + lane, col0 = (warp >> 2) * 32;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    auto read_sums = [&](uint32_t columns, float (&v)[32]) {
        float u[32];
        tc::read_columns(cols0 + lanes + columns + col0, v);
        tc::read_columns(cols0 + lanes + columns + BLOCK + col0, u);
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] = (v[j] + u[j]) * unit_of(failed);     // NaN where a wait gave up, and so the results
    };
    // eight of them joined with what stands at (row, c) of these pieces: v <- by old + times v
    auto blend = [&](const unsigned char* from, int c, float by_, float times, const float* v, float (&w)[8]) {
        join8(*reinterpret_cast<const uint4*>(from + at(row, c)), *reinterpret_cast<const uint4*>(from + lo + at(row, c)), w);
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = fmaf(by_, w[j], times * v[j]);
    };
    auto put = [&](unsigned char* to, int c, const float (&w)[8]) {
        uint4 h, l;
        split8(w, h, l);
        *reinterpret_cast<uint4*>(to + at(row, c)) = h;
        *reinterpret_cast<uint4*>(to + lo + at(row, c)) = l;
    };

    if (threadIdx.x == 0) blends[8] = first_size(total, a.eps);
    for (int turn = 0; turn < turns; ++turn) {
        // what A A is blended with, X and P X: in shared memory, which costs less than registers (32 x 100 x 900: 82 -> 80 us)
        const float* by = blends + (turn & 1) * 4;
        if (threadIdx.x == 0) {
            const Exponent now(blends[8]);
            Exponent next = now;
            next.turn(a);
            blends[8] = next.most;
            const int to = turn + 1 < turns ? next.e : 0;                  // the last one is the result itself
            blends[(turn & 1) * 4] = a.c * power_of_two(2 * now.e);
            blends[(turn & 1) * 4 + 1] = a.a * power_of_two(now.e - to);
            blends[(turn & 1) * 4 + 2] = power_of_two(3 * now.e - to);
        }
        settle();
        if (threadIdx.x == 0 && !failed) {
            const uint32_t what = tc::instruction(R, false);
            for (int t = 0; t < mine; ++t)
                for (int k = 0; k < BLOCK / 16; ++k) {
                    const uint32_t p = x_at + t * square + k * 256;
                    const uint64_t h = tc::descriptor(p, 128, 2048), l = tc::descriptor(p + lo, 128, 2048);
                    tc::product(cols0 + BLOCK, l, h, what, t > 0 || k > 0);
                    tc::product(cols0 + BLOCK, h, l, what, true);
                    tc::product(cols0, h, h, what, t > 0 || k > 0);
                }
            tc::commit(done);
        }
        wait(done, phase);
        if (col0 < R) {
            float v[32];
            read_sums(0, v);
            if (row < R) {
#pragma unroll
                for (int j = 0; j < 32; j += 4)
                    if (col0 + j < R) *reinterpret_cast<float4*>(sum + sum_at(row, col0 + j)) = make_float4(v[j], v[j + 1], v[j + 2], v[j + 3]);
            }
        }
        // A = the sum over the cluster: each block adds a share of the rows (eights of them), lanes along a row as remote reads want it, ...
        const int g0 = R / 8 * rank / ranks, g1 = R / 8 * (rank + 1) / ranks;
        if (ranks > 1) {
            tc::cluster_sync();
            for (int i = g0 * 256 + threadIdx.x; i < g1 * 256; i += RESIDENT_THREADS) {
                if ((((i & 31) ^ (i >> 5)) & 31) * 4 >= R) continue;             // 16 bytes of a row beyond R
                float4 total{0.f, 0.f, 0.f, 0.f};
                for (int k0 = 0; k0 < ranks; k0 += 8) {                           // eight reads under way together
                    float4 f[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (k0 + k < ranks) f[k] = tc::read_remote(sum_from + 16 * i, k0 + k);
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (k0 + k < ranks) { total.x += f[k].x; total.y += f[k].y; total.z += f[k].z; total.w += f[k].w; }
                }
                reinterpret_cast<float4*>(sum)[i] = total;                        // these rows of this block's sums are nobody else's
            }
        }
        __syncthreads();
        // ... and writes its pieces to all
        const int across = R / 8;
        for (int i = threadIdx.x; i < (g1 - g0) * across * 8; i += RESIDENT_THREADS) {
            const int r = (i & 7) + (g0 + (i >> 3) / across) * 8, c = (i >> 3) % across * 8;
            const float4 f = *reinterpret_cast<const float4*>(sum + sum_at(r, c)), g = *reinterpret_cast<const float4*>(sum + sum_at(r, c + 4));
            const float v[8] = {f.x, f.y, f.z, f.w, g.x, g.y, g.z, g.w};
            uint4 h, l;
            split8(v, h, l);
            if (ranks > 1) {
                for (int k = 0; k < ranks; ++k) {
                    tc::write_remote(a_at + at(r, c), k, h);
                    tc::write_remote(a_at + lo + at(r, c), k, l);
                }
            } else {
                *reinterpret_cast<uint4*>(A_ + at(r, c)) = h;
                *reinterpret_cast<uint4*>(A_ + lo + at(r, c)) = l;
            }
        }
        if (ranks > 1) tc::cluster_sync();
        settle();
        if (threadIdx.x == 0 && !failed) {
            const uint32_t what = tc::instruction(R, false);
            for (int k = 0; k < R / 16; ++k) {
                const uint32_t p = a_at + k * 256;
                const uint64_t h = tc::descriptor(p, 128, 2048), l = tc::descriptor(p + lo, 128, 2048);
                tc::product(cols0 + 3 * BLOCK, l, h, what, k > 0);
                tc::product(cols0 + 3 * BLOCK, h, l, what, true);
                tc::product(cols0 + 2 * BLOCK, h, h, what, k > 0);
            }
            tc::commit(done);
        }
        wait(done, phase);
        if (col0 < R) {
            float v[32];
            read_sums(2 * BLOCK, v);
            if (row < R) {
#pragma unroll
                for (int j = 0; j < 32; j += 8)
                    if (col0 + j < R) {
                        float w[8];
                        blend(A_, col0 + j, a.b, by[0], v + j, w);
                        put(A_, col0 + j, w);
                    }
            }
        }
        // two tiles at a time, as tensor memory allows
        for (int t0 = 0; t0 < mine; t0 += 2) {
            settle();
            if (threadIdx.x == 0 && !failed) {
                const uint32_t what = tc::instruction(BLOCK, true);
                for (int t = t0; t < mine && t < t0 + 2; ++t) {
                    for (int k = 0; k < R / 16; ++k) {
                        // cores of P: 2048 bytes from one to the next along M, 128 along K; of X: 128 along N, 2048 along K
                        const uint32_t p = a_at + k * 256, q = x_at + t * square + k * 4096, to = cols0 + (t - t0) * 2 * BLOCK;
                        const uint64_t ph = tc::descriptor(p, 128, 2048), pl = tc::descriptor(p + lo, 128, 2048);
                        const uint64_t xh = tc::descriptor(q, 2048, 128), xl = tc::descriptor(q + lo, 2048, 128);
                        tc::product(to + BLOCK, pl, xh, what, k > 0);
                        tc::product(to + BLOCK, ph, xl, what, true);
                        tc::product(to, ph, xh, what, k > 0);
                    }
                    tc::commit(t == t0 ? done : second);
                }
            }
            for (int t = t0; t < mine && t < t0 + 2; ++t) {
                if (t == t0) wait(done, phase); else wait(second, second_phase);         // the second product runs while the first is stored
                float v[32];
                read_sums((t - t0) * 2 * BLOCK, v);
                if (turn + 1 < turns) {
                    if (row < R) {
#pragma unroll
                        for (int j = 0; j < 32; j += 8) {
                            float w[8];
                            blend(X + t * square, col0 + j, by[1], by[2], v + j, w);
                            put(X + t * square, col0 + j, w);
                        }
                    }
                    continue;
                }
                // the result, through shared memory so that lanes lie along what is contiguous
                __syncthreads();
                if (row < R) {
#pragma unroll
                    for (int j = 0; j < 32; j += 8) {
                        float w[8];
                        blend(X + t * square, col0 + j, by[1], by[2], v + j, w);
                        *reinterpret_cast<float4*>(sum + sum_at(row, col0 + j)) = make_float4(w[0], w[1], w[2], w[3]);
                        *reinterpret_cast<float4*>(sum + sum_at(row, col0 + j + 4)) = make_float4(w[4], w[5], w[6], w[7]);
                    }
                }
                __syncthreads();
                const long long l0 = (first + t) * BLOCK;
                const int width = a.L - l0 < BLOCK ? (int)(a.L - l0) : BLOCK, limit = along < (a.tall ? (int)a.S : width) ? (a.tall ? width : (int)a.S) : 0;
                T* out = static_cast<T*>(a.out[m]) + (a.tall ? l0 * a.cols : l0) + along;
                const long long step = LINES * a.cols;
                out += line0 * a.cols;
                for (int line = line0; line < lines; line += AT_ONCE * LINES, out += AT_ONCE * step) {
                    float w[AT_ONCE], x[AT_ONCE];
                    T* p = out;
                    if (UPDATE) {
#pragma unroll
                        for (int k = 0; k < AT_ONCE; ++k, p += step) w[k] = line + k * LINES < limit ? to_float(*p) : 0.f;
                    }
#pragma unroll
                    for (int k = 0; k < AT_ONCE; ++k) {
                        x[k] = line + k * LINES < limit ? sum[spot(line + k * LINES)] * (1.f / SCALE) : 0.f;
                        if (UPDATE) x[k] = fmaf(a.keep, w[k], -a.move * x[k]);
                    }
                    p = out;
#pragma unroll
                    for (int k = 0; k < AT_ONCE; ++k, p += step)
                        if (line + k * LINES < limit) *p = from_float<T>(x[k]);
                }
            }
        }
    }
    tc::fence_before();
    __syncthreads();
    if (warp == 0) tc::free_columns(cols0, 512);
    if (failed) atomicOr(a.status, 1);
    if (ranks > 1) tc::cluster_sync();             // nobody leaves while others may read or write its shared memory
}

}  // namespace ortho
}  // namespace gleam
