// Instantiation unit of the prior's operators for one element type: GLEAM_PRIOR_TYPE is 0 (float32), 1 (float16) or 2 (bfloat16).
#include "dc_entry.h"
#include "prior_entry.h"
#include "prior_norm.cuh"

namespace gleam {
namespace prior {

#if GLEAM_PRIOR_TYPE == 0
using T = float;
#define GLEAM_PRIOR_OPS ops_f32
#elif GLEAM_PRIOR_TYPE == 1
using T = __half;
#define GLEAM_PRIOR_OPS ops_f16
#else
using T = __nv_bfloat16;
#define GLEAM_PRIOR_OPS ops_bf16
#endif

#define PRIOR_LAUNCH(...) do { cudaError_t e_ = prof_mark(GLEAM_K_PRIOR, s); if (e_ == cudaSuccess) e_ = launch_overlapped(true, __VA_ARGS__); \
                               if (e_ != cudaSuccess) return e_; } while (0)

static unsigned bounded(long long n, long long most) { return (unsigned)(n < 1 ? 1 : n < most ? n : most); }
constexpr long long GRID = 1ll << 20;                    // blocks of a launch at most; the kernels stride over what is beyond

static cudaError_t forward(const Args& a, bool tail, cudaStream_t s) {
    if (a.inner == 1) {
        const dim3 grid(bounded(a.outer, GRID));
        if (tail) PRIOR_LAUNCH(row_forward<T, true>, grid, dim3(ROW_THREADS), 0, s, a);
        else PRIOR_LAUNCH(row_forward<T, false>, grid, dim3(ROW_THREADS), 0, s, a);
    } else {
        const dim3 grid(bounded((a.outer * a.inner + 31) / 32, GRID));
        if (tail) PRIOR_LAUNCH(map_forward<T, true>, grid, dim3(MAP_WARPS * 32), 0, s, a);
        else PRIOR_LAUNCH(map_forward<T, false>, grid, dim3(MAP_WARPS * 32), 0, s, a);
    }
    return prof_mark(-1, s);
}

static cudaError_t vjp(const Args& a, bool tail, cudaStream_t s) {
    // the weights' gradients first: grad_x may take grad_y's place
    if (a.gw || a.gb) {
        const int parts = weight_parts(a);
        const unsigned pieces = (unsigned)((a.features + 31) / 32);
        if (a.inner == 1) PRIOR_LAUNCH(row_weight_sums<T>, dim3(pieces, parts), dim3(256), 0, s, a);
        else PRIOR_LAUNCH(map_weight_sums<T>, dim3((unsigned)a.features, parts), dim3(256), 0, s, a);
        PRIOR_LAUNCH(weight_grads<T>, dim3(pieces, 2), dim3(256), 0, s, a, parts);
    }
    if (a.inner == 1) {
        const dim3 grid(bounded(a.outer, GRID));
        if (tail) PRIOR_LAUNCH(row_vjp<T, true>, grid, dim3(ROW_THREADS), 0, s, a);
        else PRIOR_LAUNCH(row_vjp<T, false>, grid, dim3(ROW_THREADS), 0, s, a);
    } else {
        const dim3 grid(bounded((a.outer * a.inner + 31) / 32, GRID));
        if (tail) PRIOR_LAUNCH(map_vjp<T, true>, grid, dim3(MAP_WARPS * 32), 0, s, a);
        else PRIOR_LAUNCH(map_vjp<T, false>, grid, dim3(MAP_WARPS * 32), 0, s, a);
    }
    return prof_mark(-1, s);
}

static cudaError_t dropout(const Args& a, cudaStream_t s) {
    const long long n = a.outer * a.features * a.inner;
    PRIOR_LAUNCH(dropout_kernel<T>, dim3(bounded((n + 255) / 256, GRID)), dim3(256), 0, s, a);
    return prof_mark(-1, s);
}

extern const Ops GLEAM_PRIOR_OPS;
const Ops GLEAM_PRIOR_OPS = {forward, vjp, dropout};

}  // namespace prior
}  // namespace gleam
