// Launches of the prior's operators, one set for each element type (kernels_prior.cu).
#pragma once
#include <cuda_runtime.h>
#include "prior_common.cuh"

namespace gleam {
namespace prior {

struct Ops {
    cudaError_t (*forward)(const Args& a, bool tail, cudaStream_t s);
    cudaError_t (*vjp)(const Args& a, bool tail, cudaStream_t s);
    cudaError_t (*dropout)(const Args& a, cudaStream_t s);
};
extern const Ops ops_f32, ops_f16, ops_bf16;

// Maps in tiles (kernels_prior_maps.cu).  Nothing is launched (taken = false, blocks = 0) where the features of a tile do not fit.
template <class T> struct Maps {
    static cudaError_t forward(const Args& a, bool tail, bool* taken, cudaStream_t s);
    static cudaError_t vjp(const Args& a, bool tail, int* blocks, cudaStream_t s);
};

// Rows of partial sums of the weights' gradients that a VJP writes at most (its blocks come eight at a time in one form).
constexpr int SMS = 148;
constexpr int PARTS_MOST = 2 * SMS, MAP_PARTS_MOST = 8 * SMS;
inline int parts_most(const Args& a) {
    const long long positions = a.outer * a.inner, most = a.inner == 1 ? PARTS_MOST : MAP_PARTS_MOST;
    return (int)(positions + 7 < most ? positions + 7 : most);
}

}  // namespace prior
}  // namespace gleam
