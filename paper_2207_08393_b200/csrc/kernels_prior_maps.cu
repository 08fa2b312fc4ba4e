// Maps in tiles, for one element type (prior_unit.cuh); GLEAM_PRIOR_VJP is 0 for the forward kernels and 1 for the VJPs.
#include "prior_unit.cuh"
#include "prior_maps.cuh"

namespace gleam {
namespace prior {

// How maps are dealt to tiles (prior_maps.cuh); vp = 0 where the features of a tile do not fit.
struct MapPlan { int vp, items, warps; bool spread; size_t shared; };
static MapPlan map_plan(const Args& a, bool vjp, bool tail, std::initializer_list<std::pair<const void*, long long>> arrays) {
    MapPlan p{};
    if (a.features > MAP_FEATURES) return p;
    // a VJP has two sums more for each feature in registers: fewer threads, with 128 each
    p.items = !vjp && a.features <= 8 * MAP_TILE_WARPS ? 8 : a.features <= 16 * MAP_TILE_WARPS ? 16 : a.features <= 32 * MAP_TILE_WARPS ? 32 : MAP_ITEMS;
    p.warps = (int)((a.features + p.items - 1) / p.items);
    const int copies = (vjp ? 2 : 1) + tail;
    auto take = [&](int vp, bool spread) {
        bool ok = spread || a.inner % vp == 0;
        for (const auto& v : arrays) ok = ok && (spread || !v.first || ((uintptr_t)v.first % (vp * sizeof(T)) == 0 && (a.outer == 1 || v.second % vp == 0)));
        // two tiles on an SM with pieces of 16 bytes, else one with pieces of 8 (8 x 256 x 16384 in float32, VJP: one tile with 8
        // bytes 87 us, three with 4 bytes 123; tail of 8 x 160 x 16384 in bf16, VJP: 72 and 123)
        const size_t bytes = sizeof(float) * (map_exchange_floats(vp, p.warps) + 2 * (size_t)p.warps * p.items) + sizeof(T) * vp * 32 * (size_t)p.warps * p.items * copies;
        if (!ok || bytes > (vp * sizeof(T) > 8 ? 112 : 226) * 1024u) return false;
        p.vp = vp; p.spread = spread; p.shared = bytes;
        return true;
    };
    // pieces of 16 bytes, else of 8; where slices begin anywhere, four positions element by element; else smaller pieces, down to one
    // element, which still beat the kernels that read again (prior_norm.cuh; bf16, one element of 2 bytes: tail's VJP of 2 x 640 x 16384
    // 211 us and 323, of 300 x 65537 238 and 323; norm's VJP of 600 x 32769 97 and 188, tail's forward 140 and 190).  A VJP of a
    // float32 tail fits no tile from 561 features on (2 x 640 x 16384: 341 us)
    for (int vp = 16 / (int)sizeof(T); vp >= 4; vp /= 2) if (take(vp, false)) return p;
    if (a.inner >= 128 && take(4, true)) return p;
    for (int vp = 2; vp >= 1; --vp) if (take(vp, false)) return p;
    return p;
}
template <bool VJP, bool TAIL, int VP, bool SPREAD, int ITEMS>
static cudaError_t launch_maps(const Args& a, const MapPlan& p, int* blocks, cudaStream_t s) {
    constexpr auto KERNEL = [] { if constexpr (VJP) return map_tile_vjp<T, VP, ITEMS, TAIL, SPREAD>; else return map_tile_forward<T, VP, ITEMS, TAIL, SPREAD>; }();
    constexpr size_t SM_BYTES = 227 * 1024;
    cudaError_t e = ensure_smem(KERNEL, SM_BYTES, kernel_state<KERNEL>);
    if (e != cudaSuccess) return e;
    const long long tiles = SPREAD ? a.outer * ((a.inner + 32 * VP - 1) / (32 * VP)) : (a.outer * a.inner / VP + 31) / 32;
    int fit = (int)(SM_BYTES / (p.shared + 1024));
    const int threads = p.warps * 32, held = (!VJP && ITEMS <= 16 ? 2 : 1) * MAP_TILE_WARPS * 32 / threads;     // blocks that the registers of an SM hold
    if (fit > held) fit = held;
    const long long most = (long long)SMS * (fit < 1 ? 1 : fit);
    *blocks = (int)(tiles < most ? tiles : most);
    if (VJP && *blocks > MAP_PARTS_MOST) *blocks = MAP_PARTS_MOST;
    PRIOR_LAUNCH(KERNEL, dim3((unsigned)*blocks), dim3(threads), p.shared, s, a);
    return cudaSuccess;
}
template <bool VJP, bool TAIL, int VP, bool SPREAD>
static cudaError_t launch_maps(const Args& a, const MapPlan& p, int* blocks, cudaStream_t s) {
    if constexpr (!VJP) if (p.items == 8) return launch_maps<VJP, TAIL, VP, SPREAD, 8>(a, p, blocks, s);
    return p.items == 16 ? launch_maps<VJP, TAIL, VP, SPREAD, 16>(a, p, blocks, s) : p.items == 32 ? launch_maps<VJP, TAIL, VP, SPREAD, 32>(a, p, blocks, s)
                                                                                                  : launch_maps<VJP, TAIL, VP, SPREAD, MAP_ITEMS>(a, p, blocks, s);
}
template <bool VJP, bool TAIL>
static cudaError_t launch_maps(const Args& a, const MapPlan& p, int* blocks, cudaStream_t s) {
    if constexpr (sizeof(T) == 2) if (p.vp == 8) return launch_maps<VJP, TAIL, 8, false>(a, p, blocks, s);
    return p.spread ? launch_maps<VJP, TAIL, 4, true>(a, p, blocks, s) : p.vp == 4 ? launch_maps<VJP, TAIL, 4, false>(a, p, blocks, s)
         : p.vp == 2 ? launch_maps<VJP, TAIL, 2, false>(a, p, blocks, s) : launch_maps<VJP, TAIL, 1, false>(a, p, blocks, s);
}

#if GLEAM_PRIOR_VJP == 0
template <>
cudaError_t Maps<T>::forward(const Args& a, bool tail, bool* taken, cudaStream_t s) {
    const MapPlan p = map_plan(a, false, tail, {{a.x, a.px}, {a.res, a.pres}, {a.out, a.pout}, {a.out2, a.pout2}});
    *taken = p.vp != 0;
    int blocks = 0;
    return !p.vp ? cudaSuccess : tail ? launch_maps<false, true>(a, p, &blocks, s) : launch_maps<false, false>(a, p, &blocks, s);
}
#else
template <>
cudaError_t Maps<T>::vjp(const Args& a, bool tail, int* blocks, cudaStream_t s) {
    const MapPlan p = map_plan(a, true, tail, {{a.x, a.px}, {a.res, a.pres}, {a.gsum, a.pgsum}, {a.out, a.pout}, {a.out2, a.pout2}});
    *blocks = 0;
    return !p.vp ? cudaSuccess : tail ? launch_maps<true, true>(a, p, blocks, s) : launch_maps<true, false>(a, p, blocks, s);
}
#endif

}  // namespace prior
}  // namespace gleam
