// Rows, dropout and the choice of the kernels, for one element type (prior_unit.cuh).
#include "prior_unit.cuh"
#include "prior_dropout.cuh"
#include "prior_norm.cuh"
#include "prior_rows.cuh"

namespace gleam {
namespace prior {

// How rows are dealt to teams of threads (prior_rows.cuh); fits = false where a row is too long for one.
struct RowPlan {
    bool fits, edges;
    int team, warps, teams, threads;             // lanes of a team (0: warps of it), warps a team, teams and threads a block
};
static RowPlan row_plan(const Args& a) {
    RowPlan p{};
    constexpr int V = VEC<T>, ITEMS = ROW_ITEMS<T, 32>, SHARED_ITEMS = ROW_ITEMS<T, 0>;
    p.edges = !a.aligned || a.features % V != 0;
    const long long pieces = p.edges ? (a.features + 2 * (V - 1)) / V : a.features / V;
    if (pieces > SHARED_ITEMS * ROW_BLOCK_MOST) return p;
    p.fits = true;
    p.warps = 1;
    if (pieces > 32 * ITEMS) {
        p.warps = (int)((pieces + 32 * SHARED_ITEMS - 1) / (32 * SHARED_ITEMS));
        p.teams = p.warps > ROW_BLOCK / 32 ? 1 : ROW_BLOCK / 32 / p.warps;
        p.threads = p.teams * p.warps * 32;
        return p;
    }
    p.team = 2;
    while (pieces > p.team * ITEMS) p.team *= 2;
    p.teams = ROW_BLOCK / p.team;
    p.threads = ROW_BLOCK;
    return p;
}
// Blocks of the launch, of which `most` are on the GPU at once.
static int row_grid(const Args& a, const RowPlan& p, bool vjp, int most) {
    constexpr int V = VEC<T>;
    if (p.edges) {                               // V blocks at a time: the rows of a block begin alike
        const long long need = ((a.outer + V - 1) / V + p.teams - 1) / p.teams;
        return (int)(V * (need < most / V ? need : most / V));
    }
    const long long need = (a.outer + p.teams - 1) / p.teams;
    // a few rows per team in one block: it writes the weights' gradients itself
    if (vjp && (a.gw || a.gb) && need <= 4) return 1;
    return (int)(need < most ? need : most);
}

template <bool VJP, bool TAIL, bool EDGES, int TEAM>
static cudaError_t launch_rows(const Args& a, const RowPlan& p, int* blocks, cudaStream_t s) {
    constexpr int FEATURES = row_features(TEAM);
    constexpr size_t PER_THREAD = sizeof(T) * FEATURES * ((VJP ? 2 : 1) + TAIL) * row_stages(VJP, TAIL, sizeof(T), TEAM), SM_BYTES = 227 * 1024;
    constexpr auto KERNEL = [] { if constexpr (VJP) return row_team_vjp<T, TEAM, EDGES, TAIL>; else return row_team_forward<T, TEAM, EDGES, TAIL>; }();
    const size_t weights = (VJP ? 1 : 2) * sizeof(float) * FEATURES * (p.team ? p.team : p.warps * 32);
    // a block of several teams adds up their weights' gradients
    const size_t sums = VJP && p.teams > 1 ? 2 * sizeof(float) * FEATURES * p.threads : 0;
    size_t shared = EXCHANGE_BYTES + PER_THREAD * p.threads + weights;
    if (shared < sums) shared = sums;
    const cudaError_t e = ensure_smem(KERNEL, SM_BYTES, kernel_state<KERNEL>);
    if (e != cudaSuccess) return e;
    // blocks that are resident at once: what registers and shared memory hold
    int resident = row_blocks(VJP, TEAM) * row_block(VJP, TEAM) / p.threads;
    const int fit = (int)(SM_BYTES / (shared + 1024));
    if (resident > fit) resident = fit;
    if (VJP && resident > PARTS_MOST / SMS) resident = PARTS_MOST / SMS;
    *blocks = row_grid(a, p, VJP, SMS * (resident > 0 ? resident : 1));
    PRIOR_LAUNCH(KERNEL, dim3((unsigned)*blocks), dim3(p.threads), shared, s, a, p.warps, p.teams);
    return cudaSuccess;
}
template <bool VJP, bool TAIL, bool EDGES>
static cudaError_t launch_rows(const Args& a, const RowPlan& p, int* blocks, cudaStream_t s) {
    switch (p.team) {
        case 2: return launch_rows<VJP, TAIL, EDGES, 2>(a, p, blocks, s);
        case 4: return launch_rows<VJP, TAIL, EDGES, 4>(a, p, blocks, s);
        case 8: return launch_rows<VJP, TAIL, EDGES, 8>(a, p, blocks, s);
        case 16: return launch_rows<VJP, TAIL, EDGES, 16>(a, p, blocks, s);
        case 32: return launch_rows<VJP, TAIL, EDGES, 32>(a, p, blocks, s);
        default: return launch_rows<VJP, TAIL, EDGES, 0>(a, p, blocks, s);
    }
}
template <bool VJP>
static cudaError_t launch_rows(const Args& a, const RowPlan& p, bool tail, int* blocks, cudaStream_t s) {
    return tail ? (p.edges ? launch_rows<VJP, true, true>(a, p, blocks, s) : launch_rows<VJP, true, false>(a, p, blocks, s))
                : (p.edges ? launch_rows<VJP, false, true>(a, p, blocks, s) : launch_rows<VJP, false, false>(a, p, blocks, s));
}

static cudaError_t forward(const Args& given, bool tail, cudaStream_t s) {
    Args a = given;
    cudaError_t e;
    if (a.inner == 1) {
        a.aligned = packed(a, a.features, {{a.x, a.px}, {a.res, a.pres}, {a.out, a.pout}, {a.out2, a.pout2}});
        const RowPlan p = row_plan(a);
        int blocks = 0;
        if (p.fits) return (e = launch_rows<false>(a, p, tail, &blocks, s)) != cudaSuccess ? e : prof_mark(-1, s);
        const dim3 grid(bounded(a.outer, GRID));
        if (tail) PRIOR_LAUNCH(row_forward<T, true>, grid, dim3(ROW_THREADS), 0, s, a);
        else PRIOR_LAUNCH(row_forward<T, false>, grid, dim3(ROW_THREADS), 0, s, a);
    } else {
        bool taken = false;
        if ((e = Maps<T>::forward(a, tail, &taken, s)) != cudaSuccess) return e;
        if (taken) return prof_mark(-1, s);
        const dim3 grid(bounded((a.outer * a.inner + 31) / 32, GRID));
        if (tail) PRIOR_LAUNCH(map_forward<T, true>, grid, dim3(MAP_WARPS * 32), 0, s, a);
        else PRIOR_LAUNCH(map_forward<T, false>, grid, dim3(MAP_WARPS * 32), 0, s, a);
    }
    return prof_mark(-1, s);
}

static cudaError_t weight_grads_from(const Args& a, int parts, cudaStream_t s) {
    PRIOR_LAUNCH(weight_grads<T>, dim3((unsigned)((a.features + 31) / 32), 2), dim3(GRAD_WARPS * 32), 0, s, a, parts);
    return cudaSuccess;
}

static cudaError_t vjp(const Args& given, bool tail, cudaStream_t s) {
    Args a = given;
    cudaError_t e;
    if (a.inner == 1) {
        a.aligned = packed(a, a.features, {{a.x, a.px}, {a.res, a.pres}, {a.gsum, a.pgsum}, {a.out, a.pout}, {a.out2, a.pout2}});
        const RowPlan p = row_plan(a);
        if (p.fits) {
            int blocks = 0;
            if ((e = launch_rows<true>(a, p, tail, &blocks, s)) != cudaSuccess) return e;
            if ((a.gw || a.gb) && blocks > 1 && (e = weight_grads_from(a, blocks, s)) != cudaSuccess) return e;
            return prof_mark(-1, s);
        }
    } else {
        int blocks = 0;
        if ((e = Maps<T>::vjp(a, tail, &blocks, s)) != cudaSuccess) return e;
        if (blocks) {
            if ((a.gw || a.gb) && blocks > 1 && (e = weight_grads_from(a, blocks, s)) != cudaSuccess) return e;
            return prof_mark(-1, s);
        }
    }
    // the weights' gradients first: grad_x may take grad_y's place
    if (a.gw || a.gb) {
        const unsigned pieces = (unsigned)((a.features + 31) / 32);
        // enough blocks to fill the GPU over the pieces of features, each with some hundred positions at least
        const long long wide = a.inner == 1 ? pieces : a.features, share = (a.outer * a.inner + 255) / 256, fill = (8 * SMS + wide - 1) / wide;
        const int parts = (int)bounded(fill < share ? fill : share, PARTS_MOST);
        if (a.inner == 1) PRIOR_LAUNCH(row_weight_sums<T>, dim3(pieces, parts), dim3(256), 0, s, a);
        else PRIOR_LAUNCH(map_weight_sums<T>, dim3((unsigned)a.features, parts), dim3(256), 0, s, a);
        if ((e = weight_grads_from(a, parts, s)) != cudaSuccess) return e;
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

static cudaError_t dropout(const Args& given, cudaStream_t s) {
    Args a = given;
    long long slice = a.features * a.inner;
    const long long n = a.outer * slice;
    if (a.px == slice && a.pout == slice && (!a.res || a.pres == slice)) { a.outer = 1; a.features = 1; a.inner = slice = n; }
    const bool aligned = packed(a, 0, {{a.x, a.px}, {a.res, a.pres}, {a.out, a.pout}}), whole = slice % VEC<T> == 0;
    const long long blocks = ((n + VEC<T> - 1) / VEC<T> + DROP_THREADS - 1) / DROP_THREADS;
    if (blocks > 0x7fffffffll) return cudaErrorInvalidConfiguration;
    const int form = !aligned ? DROP_ELEMENTS : a.outer == 1 ? (whole ? DROP_FLAT : DROP_FLAT_END) : whole ? DROP_SLICES : DROP_ELEMENTS;
    auto pick = [&](auto res, auto drop) {
        constexpr bool R = decltype(res)::value, D = decltype(drop)::value;
        return form == DROP_FLAT ? dropout_kernel<T, R, D, DROP_FLAT> : form == DROP_FLAT_END ? dropout_kernel<T, R, D, DROP_FLAT_END>
             : form == DROP_SLICES ? dropout_kernel<T, R, D, DROP_SLICES> : dropout_kernel<T, R, D, DROP_ELEMENTS>;
    };
    auto kernel = a.res ? (a.dropping ? pick(yes{}, yes{}) : pick(yes{}, no{})) : (a.dropping ? pick(no{}, yes{}) : pick(no{}, no{}));
    PRIOR_LAUNCH(kernel, dim3((unsigned)blocks), dim3(DROP_THREADS), 0, s, a);
    return prof_mark(-1, s);
}

#if GLEAM_PRIOR_TYPE == 0
extern const Ops ops_f32;
const Ops ops_f32 = {forward, vjp, dropout};
#elif GLEAM_PRIOR_TYPE == 1
extern const Ops ops_f16;
const Ops ops_f16 = {forward, vjp, dropout};
#else
extern const Ops ops_bf16;
const Ops ops_bf16 = {forward, vjp, dropout};
#endif

}  // namespace prior
}  // namespace gleam
