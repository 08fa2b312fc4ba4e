// Launches of the gated recurrence, one set for each element type (kernels_scan.cu), and the sizes that both sides go by.
#pragma once
#include <cuda_runtime.h>
#include "scan_common.cuh"

namespace gleam {
namespace scan {

struct Ops {
    // fills the parts, chunks and runs of a call from its sizes alone; states to save and 32-bit numbers of workspace
    void (*plan)(Args& a, long long* saved, long long* scratch);
    cudaError_t (*forward)(const Args& a, bool reverse, cudaStream_t s);
    cudaError_t (*vjp)(const Args& a, bool reverse, cudaStream_t s);
    cudaError_t (*step)(const Args& a, cudaStream_t s);
};
extern const Ops ops_f32, ops_f16, ops_bf16;

}  // namespace scan
}  // namespace gleam
