// The gated recurrence for one element type: GLEAM_SCAN_TYPE is 0 (float32), 1 (float16) or 2 (bfloat16).
#include "dc_entry.h"
#include "launch_state.cuh"
#include "scan_columns.cuh"
#include "scan_entry.h"
#include "scan_rows.cuh"

#include <initializer_list>
#include <type_traits>

namespace gleam {
namespace scan {

#if GLEAM_SCAN_TYPE == 0
using T = float;
#define OPS ops_f32
#elif GLEAM_SCAN_TYPE == 1
using T = __half;
#define OPS ops_f16
#else
using T = __nv_bfloat16;
#define OPS ops_bf16
#endif

#define SCAN_LAUNCH(...) do { cudaError_t e_ = prof_mark(GLEAM_K_SCAN, s); if (e_ == cudaSuccess) e_ = launch_overlapped(true, __VA_ARGS__); \
                              if (e_ != cudaSuccess) return e_; } while (0)

constexpr int SMS = 148, WIDE = 8 / sizeof(T);           // chains of a thread's piece of 8 bytes
constexpr int PARTS_MOST = 512;                         // more of them would take the launch that joins them longer than they save
constexpr int NARROW = 128;                              // rows of fewer chains, where they start anywhere, are no strips

static long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// Parts of the chains: where there are too few chains to fill the SMs.  Two more passes over part of the arrays (the maps, and joining
// them) have to pay for themselves, so a part has two chunks or tiles at least.
static void plan(Args& a, long long* saved, long long* scratch) {
    a.rows = a.batch * a.channels * a.inner;
    a.parts = 1; a.run = 1; a.chunk = 1; a.part = a.steps;
    *saved = *scratch = 0;
    if (a.rows == 0 || a.steps == 0) return;
    long long units, threads;
    if (a.inner > 1) {
        a.chunk = chunk_steps(a.steps);
        units = ceil_div(a.steps, a.chunk);
        threads = a.rows / WIDE + 1;
        *saved = (units - 1) * a.rows;
    } else {
        if (a.steps <= SHORT_STEPS<T>) return;
        a.run = run_rows(a.rows, a.steps, TILE<T>);
        a.chunk = TILE<T>;
        units = run_tiles<T>(a.run, a.steps);
        threads = 16 * a.rows;                       // half a warp: series take twice the warps of columns, a tile's shuffles are slow
        *saved = ceil_div(a.rows, a.run) * units;
    }
    const long long wanted = SMS * (a.inner > 1 ? 640 : 512);
    if (a.run == 1 && units >= 4 && threads < wanted / 2) {
        long long parts = wanted / threads;
        if (parts > units / 2) parts = units / 2;
        if (parts > PARTS_MOST) parts = PARTS_MOST;
        const long long each = ceil_div(units, parts);
        a.part = each * a.chunk;
        a.parts = (int)ceil_div(units, each);
    }
    if (a.parts == 1) a.part = a.steps;
    else *scratch = 2 * ceil_div(a.parts * a.rows, 64) * 64;
}

// Whether V neighbouring chains can be taken at once.
struct Array { const void* p; const Strides* s; };
static bool wide(const Args& a, int v, std::initializer_list<Array> arrays, std::initializer_list<const void*> states) {
    if (a.inner % v) return false;
    for (const Array& u : arrays) {
        if (!u.p) continue;
        if ((uintptr_t)u.p % (v * sizeof(T))) return false;
        if ((a.batch > 1 && u.s->batch % v) || (a.channels > 1 && u.s->channel % v) || (a.steps > 1 && u.s->step % v)) return false;
    }
    for (const void* p : states)
        if ((uintptr_t)p % ((v < 4 ? v : 4) * sizeof(float))) return false;
    return true;
}

// Whether the steps lie without gaps from chain to chain, from 16 bytes on.
static bool dense(const Args& a, std::initializer_list<Array> arrays) {
    for (const Array& u : arrays) {
        if (!u.p) continue;
        if ((uintptr_t)u.p % 16 || (a.steps > 1 && u.s->step != 1) || (a.channels > 1 && u.s->channel != a.steps) ||
            (a.batch > 1 && u.s->batch != a.channels * a.steps)) return false;
    }
    return true;
}

template <class F> static cudaError_t by_bool(bool v, F f) { return v ? f(std::true_type{}) : f(std::false_type{}); }

template <auto KERNEL> static PerDevice kernel_state;

static cudaError_t join(const Args& a, bool back, bool descending, cudaStream_t s) {
    Args j = a;
    j.descending = descending; j.enter = back ? a.dlast : a.state;
    SCAN_LAUNCH(join_parts<8>, dim3((unsigned)ceil_div(a.rows, 32)), dim3(32 * JOIN_WARPS), 0, s, j);
    return cudaSuccess;
}

template <int V, bool REVERSE, bool STRIP, int KIND>
static cudaError_t stream(const Args& a, cudaStream_t s) {
    constexpr int THREADS = KIND == VJP ? VJP_THREADS : STREAM_THREADS;
    const long long blocks = STRIP ? a.batch * a.channels * ceil_div(a.inner, THREADS * V) : ceil_div(a.rows / V, THREADS);
    const dim3 grid((unsigned)blocks, (unsigned)a.parts), block(THREADS);
    if constexpr (KIND == VJP) {
        constexpr auto KERNEL = stream_vjp<T, V, REVERSE, STRIP>;
        const cudaError_t e = ensure_smem(KERNEL, vjp_smem<T, V, STRIP>(), kernel_state<KERNEL>);
        if (e != cudaSuccess) return e;
        SCAN_LAUNCH(KERNEL, grid, block, (size_t)vjp_smem<T, V, STRIP>(), s, a);
    } else {
        constexpr auto KERNEL = stream_kernel<T, V, REVERSE, STRIP, KIND>;
        const cudaError_t e = ensure_smem(KERNEL, stream_smem<T, V, STRIP>(), kernel_state<KERNEL>);
        if (e != cudaSuccess) return e;
        SCAN_LAUNCH(KERNEL, grid, block, (size_t)stream_smem<T, V, STRIP>(), s, a);
    }
    return cudaSuccess;
}

template <int V, bool REVERSE, bool STRIP, bool BACK>
static cudaError_t streams(const Args& a, cudaStream_t s) {
    cudaError_t e;
    if (a.parts > 1) {
        if ((e = stream<V, REVERSE, STRIP, BACK ? MAP_VJP : MAP_FORWARD>(a, s)) != cudaSuccess) return e;
        if ((e = join(a, BACK, BACK, s)) != cudaSuccess) return e;
    }
    return stream<V, REVERSE, STRIP, BACK ? VJP : FORWARD>(a, s);
}

template <bool REVERSE, bool BACK>
static cudaError_t columns(const Args& a, cudaStream_t s) {
    const dim3 grid((unsigned)ceil_div(a.rows, COLUMN_THREADS), (unsigned)a.parts), block(COLUMN_THREADS);
    cudaError_t e;
    if (a.parts > 1) {
        if constexpr (BACK) SCAN_LAUNCH(columns_vjp<T, REVERSE, true>, grid, block, 0, s, a);
        else SCAN_LAUNCH(columns_forward<T, REVERSE, true>, grid, block, 0, s, a);
        if ((e = join(a, BACK, BACK, s)) != cudaSuccess) return e;
    }
    if constexpr (BACK) SCAN_LAUNCH(columns_vjp<T, REVERSE, false>, grid, block, 0, s, a);
    else SCAN_LAUNCH(columns_forward<T, REVERSE, false>, grid, block, 0, s, a);
    return cudaSuccess;
}

template <bool REVERSE, bool DENSE, bool SINGLE, bool BACK>
static cudaError_t rows_of(const Args& a, cudaStream_t s) {
    const long long warps = SINGLE ? a.rows * a.parts : ceil_div(a.rows, a.run);
    const dim3 grid((unsigned)ceil_div(warps, ROW_WARPS)), block(32 * ROW_WARPS);
    if (SINGLE && a.parts > 1) {
        SCAN_LAUNCH(rows_kernel<T, REVERSE, DENSE, true, BACK ? MAP_VJP : MAP_FORWARD>, grid, block, 0, s, a);
        const cudaError_t e = join(a, BACK, BACK != REVERSE, s);                 // parts are numbered from the first step
        if (e != cudaSuccess) return e;
    }
    SCAN_LAUNCH(rows_kernel<T, REVERSE, DENSE, SINGLE, BACK ? VJP : FORWARD>, grid, block, 0, s, a);
    return cudaSuccess;
}

template <bool REVERSE, bool DENSE, bool BACK>
static cudaError_t rows(const Args& a, cudaStream_t s) {
    if (a.steps <= SHORT_STEPS<T>)
        return by_bool(sizeof(T) == 2 && a.steps % 2 == 0, [&](auto w) -> cudaError_t {
            constexpr bool WHOLE = sizeof(T) == 2 && decltype(w)::value;
            constexpr auto KERNEL = short_kernel<T, REVERSE, DENSE, WHOLE, BACK ? VJP : FORWARD>;
            const cudaError_t e = ensure_smem(KERNEL, short_smem<T, BACK ? VJP : FORWARD>(SHORT_STEPS<T>), kernel_state<KERNEL>);
            if (e != cudaSuccess) return e;
            SCAN_LAUNCH(KERNEL, dim3((unsigned)ceil_div(a.rows, SHORT_ROWS)), dim3(SHORT_ROWS), (short_smem<T, BACK ? VJP : FORWARD>(a.steps)), s, a);
            return cudaSuccess;
        });
    return a.run == 1 ? rows_of<REVERSE, DENSE, true, BACK>(a, s) : rows_of<REVERSE, DENSE, false, BACK>(a, s);
}

template <bool BACK>
static cudaError_t chains(const Args& a, bool reverse, std::initializer_list<Array> arrays, std::initializer_list<const void*> states, cudaStream_t s) {
    return by_bool(reverse, [&](auto r) {
        constexpr bool R = decltype(r)::value;
        if (a.inner == 1) return by_bool(dense(a, arrays), [&](auto d) { return rows<R, decltype(d)::value, BACK>(a, s); });
        // pieces of 16 bytes where there are chains enough: fewer instructions (8 x 512 x 45000 float16: forward 275 -> 212 us, VJP 377 -> 344;
        // where there are not, 8000 x 2048 bf16, forward 35 -> 37)
        if (a.rows * a.parts / (2 * WIDE) >= SMS * 192 && wide(a, 2 * WIDE, arrays, states)) return streams<2 * WIDE, R, false, BACK>(a, s);
        if (wide(a, WIDE, arrays, states)) return streams<WIDE, R, false, BACK>(a, s);
        if (a.inner >= NARROW) return streams<WIDE, R, true, BACK>(a, s);
        return columns<R, BACK>(a, s);
    });
}

static cudaError_t forward(const Args& a, bool reverse, cudaStream_t s) {
    return chains<false>(a, reverse, {{a.x, &a.sx}, {a.gate, &a.sgate}, {a.y, &a.sy}}, {a.state, a.last, a.saved}, s);
}

static cudaError_t vjp(const Args& a, bool reverse, cudaStream_t s) {
    return chains<true>(a, reverse, {{a.x, &a.sx}, {a.gate, &a.sgate}, {a.dy, &a.sdy}, {a.dx, &a.sdx}, {a.dg, &a.sdg}},
                        {a.state, a.saved, a.dlast, a.dstate}, s);
}

static cudaError_t step(const Args& a, cudaStream_t s) {
    const bool w = wide(a, WIDE, {{a.x, &a.sx}, {a.gate, &a.sgate}, {a.y, &a.sy}}, {a.last});
    const long long threads = w ? a.rows / WIDE : a.rows;
    const dim3 grid((unsigned)ceil_div(threads, COLUMN_THREADS)), block(COLUMN_THREADS);
    if (w) SCAN_LAUNCH(step_kernel<T, WIDE>, grid, block, 0, s, a);
    else SCAN_LAUNCH(step_kernel<T, 1>, grid, block, 0, s, a);
    return cudaSuccess;
}

const Ops OPS = {plan, forward, vjp, step};

}  // namespace scan
}  // namespace gleam
