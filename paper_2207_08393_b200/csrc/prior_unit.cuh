// What the instantiation units of the prior's operators share: the element type, launches, alignment of arrays.  GLEAM_PRIOR_TYPE is
// 0 (float32), 1 (float16) or 2 (bfloat16).
#pragma once
#include "dc_entry.h"
#include "launch_state.cuh"
#include "prior_entry.h"

#include <initializer_list>
#include <type_traits>
#include <utility>

namespace gleam {
namespace prior {

#if GLEAM_PRIOR_TYPE == 0
using T = float;
#elif GLEAM_PRIOR_TYPE == 1
using T = __half;
#else
using T = __nv_bfloat16;
#endif

template <> cudaError_t Maps<T>::forward(const Args& a, bool tail, bool* taken, cudaStream_t s);
template <> cudaError_t Maps<T>::vjp(const Args& a, bool tail, int* blocks, cudaStream_t s);

#define PRIOR_LAUNCH(...) do { cudaError_t e_ = prof_mark(GLEAM_K_PRIOR, s); if (e_ == cudaSuccess) e_ = launch_overlapped(true, __VA_ARGS__); \
                               if (e_ != cudaSuccess) return e_; } while (0)

static inline unsigned bounded(long long n, long long most) { return (unsigned)(n < 1 ? 1 : n < most ? n : most); }
constexpr long long GRID = 1ll << 20;                    // blocks of a launch at most; the kernels stride over what is beyond

using yes = std::true_type;
using no = std::false_type;
template <int N> using number = std::integral_constant<int, N>;

// Whether all the arrays (null: absent) start at 16 bytes and, where they step, step by multiples of them more than `beyond`.
static inline bool packed(const Args& a, long long beyond, std::initializer_list<std::pair<const void*, long long>> arrays) {
    for (const auto& v : arrays)
        if (v.first && ((uintptr_t)v.first % 16 != 0 || (a.outer > 1 && (v.second - beyond) % VEC<T> != 0))) return false;
    return true;
}

template <auto KERNEL> static PerDevice kernel_state;

}  // namespace prior
}  // namespace gleam
