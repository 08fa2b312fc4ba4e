// What the kernels of the orthogonalised update share.
//
// With X of S x L (S the shorter side, L the longer one, tall matrices taken transposed), X_0 = U / (|U| + eps), every turn is
//
//     A = X X^T,   P = b A + c A A,   X <- a X + P X,
//
// which takes each singular value v to a v + b v^3 + c v^5 and leaves the singular vectors: after a few turns of suitable (a, b, c)
// all values but the smallest are near 1 (K. Jordan et al., "Muon: an optimizer for hidden layers in neural networks", 2024).
//
// The products run on the tensor cores in float16 with 32-bit sums, and come near the precision of 32-bit numbers: X, A and P are stored as
// two pieces, hi = x rounded to float16 and lo = x - hi rounded to float16 (22 bits, where a 32-bit number has 24), and a product is
// hi hi + hi lo + lo hi; what is left out is 2^-24 of it.  All stored values are scaled by 2^10 (up to 64 in front of the scale), so that lo keeps
// its bits down to values of 2^-13 and is off by 2^-35 below; X also by a power of two where its norm is small against eps (Exponent).  The
// term a X is added in 32 bits.  Five turns of 100 x 900 of falling singular values are off by 2.0e-6, 2.8e-6 in 32-bit products; of 9216 x 1024 by
// 8.7e-6 and 6.1e-6.  float16 or bfloat16 products without the second piece would be off by 1e-3 or 1e-2.
//
// Matrices are stored in blocks of 128 x 128 with zeros beyond their sides, 64 KB: 16 rows of cores, in each those of hi, then those of lo, 16
// cores of 8 rows by 8 columns, a row of a core 16 bytes: the shape that the matrix instructions read, along either side.  An operand's
// tile is a few copies of 8 or 16 KB: rows lie in one run with both their pieces, 32 of the columns in runs of 512 bytes, which a tiled
// copy takes at once.  (With a copy for each run the copies, not the products, took the time: 4 x 512 x 4608, A: 89 us instead of 38.)
// Products run at the tensor core's rate (64 cycles for 128 x 128 x 16, 4096 products a cycle); instructions with N = 64 take as long, for
// the 128 rows of their other operand.  All products that add to one sum have one shape and one place in tensor memory: only such
// ones are sure to follow each other in the order of their issue.  hi (hi, lo) as one instruction of twice the width and lo hi added to half of
// its sums took 2 % less, and an update of it could be lost.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "prior_common.cuh"

namespace gleam {
namespace ortho {

using prior::from_float;
using prior::to_float;

constexpr int BLOCK = 128, CORE = 128, LO = 16 * CORE, ROW_BYTES = 2 * LO, BLOCK_BYTES = 16 * ROW_BYTES;    // from hi to lo; a row of cores
constexpr float SCALE = 1024.f;
constexpr int GROUP = 64;                          // matrices of a launch
constexpr int PARTS = 592;                         // partial sums of squares of a matrix at most

struct Args {
    const void* u[GROUP];                          // matrices or gradients
    float* momentum[GROUP];                        // update: momenta, else null
    void* out[GROUP];                              // results, or weights
    long long rows, cols, S, L;
    int tall, dtype;                               // GLEAM_F32, ...
    int sblocks, lblocks, parts;
    int update, nesterov;
    int fresh;                                     // the first launch of a call: the status is set to 0
    float a, b, c, eps, mu, keep, move;            // weight <- keep weight - move result
    unsigned char* x; unsigned char* y;            // X and its successor: (count, sblocks, lblocks) blocks
    unsigned char* g; unsigned char* p;            // A and P: (count, sblocks, sblocks) blocks
    float* part; int* status;
    float* size;                                   // norms of X_0
    int turn;                                      // the turn of a launch
    unsigned char* blocks;                         // all blocks of the workspace: what the tiled copies' map covers
};

// Byte of element (r, c) of a block's hi.
__host__ __device__ __forceinline__ int core_at(int r, int c) { return (r >> 3) * ROW_BYTES + (c >> 3) * CORE + (r & 7) * 16 + (c & 7) * 2; }

// A block's sums as 32-bit numbers in shared memory: rows of 128, their 16-byte pieces in an order that keeps 32 rows apart.
__device__ __forceinline__ int sum_at(int r, int c) { return r * BLOCK + ((((c >> 2) ^ r) & 31) << 2) + (c & 3); }

template <class T> __device__ __forceinline__ float load_at(const void* p, long long i) { return to_float(static_cast<const T*>(p)[i]); }
template <class T> __device__ __forceinline__ void store_at(void* p, long long i, float v) { static_cast<T*>(p)[i] = from_float<T>(v); }

// 2^n; zero below the smallest normal number.
__device__ __forceinline__ float power_of_two(int n) { return n < -126 ? 0.f : __int_as_float((n < 127 ? n + 127 : 254) << 23); }

// The norm of what is orthogonalised may be small against eps, and X then starts far below 1.  So that its pieces keep their bits, X = 2^e X^
// is stored as X^, with e = 0 as soon as X may have a norm above 1/2 (from the first turn on where eps is small) and otherwise such that a
// bound of X^'s norm lies in [1/2, 1).  The bound: |X_0|, then |X| (|a| + |b| |X|^2 + |c| |X|^4).  A turn in terms of X^ is
//
//     A^ = X^ X^^T,   P^ = b A^ + c 2^2e A^ A^,   X^ <- 2^(e - e') (a X^ + 2^2e P^ X^),
//
// powers of two throughout: where all e are 0 nothing changes, and nowhere is anything rounded for it.
struct Exponent {
    static constexpr int LEAST = -120;
    float most;                                    // the bound; e = 0 from where it is not below 1/2 (or no number) on
    int e;
    __device__ __forceinline__ explicit Exponent(float size) : most(size), e(0) { set(); }
    __device__ __forceinline__ void set() {
        if (!(most <= 0.5f)) { e = 0; return; }
        e = (__float_as_int(most) >> 23) - 126;
        if (e < LEAST) e = LEAST;
    }
    __device__ __forceinline__ void turn(const Args& a) {
        if (!(most <= 0.5f)) return;
        const float square = most * most;
        most = fmaxf(most * (fabsf(a.a) + square * (fabsf(a.b) + square * fabsf(a.c))), 7.5e-37f);       // 2^LEAST
        set();
    }
};

// The norm of X_0, from the sum of squares.  Squares below 2^-149 are lost: a norm below 2^-64 counts as that (what is stored is then smaller than it
// could be, but right).
__device__ __forceinline__ float first_size(float total, float eps) {
    const float norm = sqrtf(total);
    return fmaxf(norm, 5.42101086e-20f) / (norm + eps);
}
// What turns U into the stored X_0.  Finite, so that zeros stay zeros under the smallest eps; NaN where the sum is.
__device__ __forceinline__ float first_scale(float total, float eps) {
    const float by = ldexpf(SCALE / (sqrtf(total) + eps), -Exponent(first_size(total, eps)).e);
    return by > 3.402823466e38f ? 3.402823466e38f : by;
}

// What brings a product's sums to the stored values' units: a launch that gave up waiting leaves NaN, in weights too, which no caller overlooks.
__device__ __forceinline__ float unit_of(bool failed) { return failed ? __int_as_float(0x7fffffff) : 1.f / SCALE; }

// Eight neighbours of a row as two pieces, and back.
__device__ __forceinline__ void split8(const float (&v)[8], uint4& hi, uint4& lo) {
    uint32_t h[4], l[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const __half2 a = __floats2half2_rn(v[2 * j], v[2 * j + 1]);
        const float2 f = __half22float2(a);
        const __half2 r = __floats2half2_rn(v[2 * j] - f.x, v[2 * j + 1] - f.y);
        h[j] = reinterpret_cast<const uint32_t&>(a);
        l[j] = reinterpret_cast<const uint32_t&>(r);
    }
    hi = make_uint4(h[0], h[1], h[2], h[3]);
    lo = make_uint4(l[0], l[1], l[2], l[3]);
}
__device__ __forceinline__ void join8(const uint4& hi, const uint4& lo, float (&v)[8]) {
    const uint32_t h[4] = {hi.x, hi.y, hi.z, hi.w}, l[4] = {lo.x, lo.y, lo.z, lo.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float2 a = __half22float2(reinterpret_cast<const __half2&>(h[j])), b = __half22float2(reinterpret_cast<const __half2&>(l[j]));
        v[2 * j] = a.x + b.x; v[2 * j + 1] = a.y + b.y;
    }
}

}  // namespace ortho
}  // namespace gleam
