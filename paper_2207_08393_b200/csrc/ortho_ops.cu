// Orthogonalised updates: entry points, argument checks, workspace, launches.
#include "../../include/gleam.h"
#include "dc_entry.h"
#include "launch_state.cuh"
#include "ortho_gemm.cuh"
#include "ortho_prepare.cuh"
#include "ortho_resident.cuh"

#include <algorithm>
#include <cmath>
#include <cstring>
#include <memory>
#include <new>

namespace gleam {
namespace ortho {

#define ORTHO_LAUNCH(...) do { cudaError_t e_ = prof_mark(GLEAM_K_ORTHO, s); if (e_ == cudaSuccess) e_ = (__VA_ARGS__); if (e_ != cudaSuccess) return e_; } while (0)

constexpr int SMS = 148;

// The tiled copies' map: the workspace's blocks as rows of cores, each eight parts of 512 bytes (32 columns, of hi and then of lo); a copy
// takes one part of 16 rows.  cuTensorMapEncodeTiled comes through the runtime's lookup: no link-time dependency on the driver.
static cudaError_t map_of(const Args& a, uint64_t bytes, CUtensorMap* map) {
    typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                               const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static std::atomic<Encode> kept{nullptr};
    Encode encode = kept.load(std::memory_order_acquire);
    if (!encode) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess || !p) {
            cudaGetLastError();
            return cudaErrorNotSupported;
        }
        encode = (Encode)p;
        kept.store(encode, std::memory_order_release);
    }
    const cuuint64_t dims[3] = {128, 8, bytes / ROW_BYTES}, strides[2] = {512, ROW_BYTES};
    const cuuint32_t box[3] = {128, 1, 16}, steps[3] = {1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, a.blocks, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

// More than eight blocks to a cluster have to be allowed kernel by kernel.
template <class K>
static cudaError_t allow_clusters(K kernel, int ranks) {
    return ranks > RESIDENT_PORTABLE ? cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) : cudaSuccess;
}

// Clusters of so many blocks, one block an SM, that a B200 runs at once: its SMs come in groups that clusters do not cross, so 16
// clusters of 7 are more than 148 SMs may hold.  Constants (what cudaOccupancyMaxActiveClusters gives on the GPUs it was asked on, the
// least of them): sums are split by the sizes alone, so that the replicas of a model on several GPUs compute the same bits.  A GPU whose
// groups hold fewer takes one round more.  Only whether it takes more than eight blocks at all is asked of the GPU itself.
static int clusters_at_once(int ranks) {
    static constexpr int at_once[RESIDENT_RANKS + 1] = {0, SMS, 74, 45, 33, 26, 22, 15, 15, 15, 11, 7, 7, 7, 7, 7, 7};
    if (ranks <= RESIDENT_PORTABLE) return at_once[ranks];
    static PerDevice cache[RESIDENT_RANKS + 1];                       // 1: no, 2: yes
    std::atomic<int>* slot = cache[ranks].slot();
    if (slot) { const int v = slot->load(std::memory_order_acquire); if (v > 0) return v == 2 ? at_once[ranks] : 0; }
    static PerDevice done;
    constexpr auto KERNEL = resident_kernel<float, false>;
    int n = 0;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute at[2];
    launch_config(cfg, at, false, dim3((unsigned)ranks), dim3(RESIDENT_THREADS), RESIDENT_MOST, nullptr, 2);
    at[0].val.clusterDim.x = (unsigned)ranks;
    if (ensure_smem(KERNEL, RESIDENT_MOST, done) != cudaSuccess || allow_clusters(KERNEL, ranks) != cudaSuccess ||
        cudaOccupancyMaxActiveClusters(&n, KERNEL, &cfg) != cudaSuccess) {
        cudaGetLastError();
        n = 0;
    }
    if (slot) slot->store(n > 0 ? 2 : 1, std::memory_order_release);
    return n > 0 ? at_once[ranks] : 0;
}

template <int KIND, int RANKS, bool LONG, class T>
static cudaError_t gemm_of(const Args& a, const CUtensorMap& map, int count, cudaStream_t s) {
    static PerDevice done;
    const cudaError_t e = ensure_smem(gemm_kernel<KIND, RANKS, LONG, T>, Form<KIND, LONG>::SMEM, done);
    if (e != cudaSuccess) return e;
    const dim3 grid((unsigned)RANKS, (unsigned)tiles_of<KIND>(a), (unsigned)count), block(GEMM_THREADS);
    ORTHO_LAUNCH(launch_overlapped_cluster((unsigned)RANKS, gemm_kernel<KIND, RANKS, LONG, T>, grid, block, Form<KIND, LONG>::SMEM, s, a, map));
    return cudaSuccess;
}
// GRAM and POLY: blocks that share a sum over K
template <int KIND, bool LONG>
static cudaError_t gemm_in(int ranks, const Args& a, const CUtensorMap& map, int count, cudaStream_t s) {
    switch (ranks) {
        case 2: return gemm_of<KIND, 2, LONG, float>(a, map, count, s);
        case 3: return gemm_of<KIND, 3, LONG, float>(a, map, count, s);
        case 4: return gemm_of<KIND, 4, LONG, float>(a, map, count, s);
        case 6: return gemm_of<KIND, 6, LONG, float>(a, map, count, s);
        case 8: return gemm_of<KIND, 8, LONG, float>(a, map, count, s);
    }
    return gemm_of<KIND, 1, LONG, float>(a, map, count, s);
}
template <int KIND, class T = float>
static cudaError_t gemm(const Args& a, const CUtensorMap& map, int count, cudaStream_t s) {
    if constexpr (KIND == GRAM || KIND == POLY) {
        // a step takes about 0.45 us, all else of a block 6, 8 with others; rounds of clusters
        const long long tiles = (long long)tiles_of<KIND>(a) * count, steps = steps_of<KIND, false>(a);
        int best = 1;
        long long least = 0;
        for (const int ranks : {1, 2, 3, 4, 6, 8}) {
            if (ranks > 1 && steps < 2 * ranks) break;
            const int at_once = ranks > 1 ? clusters_at_once(ranks) : SMS;
            const long long time = (tiles + at_once - 1) / at_once * ((steps + ranks - 1) / ranks * 45 + (ranks > 1 ? 800 : 600));
            if (ranks == 1 || time < least) { best = ranks; least = time; }
        }
        return (steps + best - 1) / best > LONG_FROM<KIND> ? gemm_in<KIND, true>(best, a, map, count, s) : gemm_in<KIND, false>(best, a, map, count, s);
    } else {
        return steps_of<KIND, true>(a) > LONG_FROM<KIND> ? gemm_of<KIND, 1, true, T>(a, map, count, s) : gemm_of<KIND, 1, false, T>(a, map, count, s);
    }
}

// Whether a matrix fits a cluster that every GPU of this kind takes (eight blocks).
static bool resident_fits(long long S, long long L) {
    if (S > BLOCK) return false;
    const long long all = (L + BLOCK - 1) / BLOCK;
    for (int tiles = 1; resident_bytes(resident_rows(S), tiles) <= RESIDENT_MOST; ++tiles)
        if ((all + tiles - 1) / tiles <= RESIDENT_PORTABLE) return true;
    return false;
}
// Such calls of up to so many matrices have no workspace for the general kernels, which would not be faster.
constexpr long long RESIDENT_COUNT = 8;

// Tiles of a block of the resident kernel for a launch, 0 where the general kernels (if there is a workspace for them) take less time.  In
// 0.1 us, from measured calls of five turns: a round of clusters 580 and 110 for each tile of a block (8 x 128 x 1152 70 us, 1 x 112 x 3500
// 82); the general kernels 850 and 2.3 for each tile of all matrices (8 x 128 x 1152 109 us, 32 x 128 x 2048 205).
static int resident_tiles(long long S, long long L, int count, bool general) {
    if (S > BLOCK) return 0;
    const long long all = (L + BLOCK - 1) / BLOCK;
    int best = 0;
    long long least = general ? 850 + 23 * all * count / 10 : 0;
    for (int tiles = 1; tiles <= all && resident_bytes(resident_rows(S), tiles) <= RESIDENT_MOST; ++tiles) {
        const int ranks = (int)((all + tiles - 1) / tiles), at_once = ranks <= RESIDENT_RANKS ? clusters_at_once(ranks) : 0;
        if (at_once == 0) continue;
        const long long time = (count + at_once - 1) / at_once * (580 + 110 * tiles);
        if (least == 0 || time < least) { best = tiles; least = time; }
    }
    return best;
}

template <class T, bool UPDATE>
static cudaError_t run(Args& a, int count, int turns, cudaStream_t s) {
    if (const int tiles = resident_tiles(a.S, a.L, count, a.x != nullptr)) {
        static PerDevice done;
        const cudaError_t e = ensure_smem(resident_kernel<T, UPDATE>, RESIDENT_MOST, done);
        if (e != cudaSuccess) return e;
        const unsigned ranks = (unsigned)((a.lblocks + tiles - 1) / tiles);
        const cudaError_t allowed = allow_clusters(resident_kernel<T, UPDATE>, (int)ranks);
        if (allowed != cudaSuccess) return allowed;
        ORTHO_LAUNCH(launch_overlapped_cluster(ranks, resident_kernel<T, UPDATE>, dim3(ranks, (unsigned)count), dim3(RESIDENT_THREADS),
                                               (size_t)resident_bytes(resident_rows(a.S), tiles), s, a, tiles, turns));
        return cudaSuccess;
    }
    ORTHO_LAUNCH(launch_overlapped(true, sums_kernel<T, UPDATE>, dim3((unsigned)a.parts, (unsigned)count), dim3(PREPARE_THREADS), 0, s, a));
    const size_t tile = sizeof(float) * BLOCK * BLOCK;
    static PerDevice done;
    cudaError_t e = ensure_smem(first_kernel<T, UPDATE>, tile, done);
    if (e != cudaSuccess) return e;
    CUtensorMap map;
    if ((e = map_of(a, (uint64_t)((unsigned char*)a.part - a.blocks), &map)) != cudaSuccess) return e;
    ORTHO_LAUNCH(launch_overlapped(true, first_kernel<T, UPDATE>, dim3((unsigned)(a.sblocks * a.lblocks), (unsigned)count), dim3(PREPARE_THREADS), tile, s, a));
    for (int k = 0; k < turns; ++k) {
        a.turn = k;
        if ((e = gemm<GRAM>(a, map, count, s)) != cudaSuccess || (e = gemm<POLY>(a, map, count, s)) != cudaSuccess) return e;
        if ((e = k + 1 < turns ? gemm<APPLY>(a, map, count, s) : gemm<LAST, T>(a, map, count, s)) != cudaSuccess) return e;
        std::swap(a.x, a.y);
    }
    return cudaSuccess;
}

template <class T>
static cudaError_t run_for(Args& a, bool update, int count, int turns, cudaStream_t s) {
    return update ? run<T, true>(a, count, turns, s) : run<T, false>(a, count, turns, s);
}

struct Layout { int sblocks, lblocks, group; uint64_t x, square, part, status, total; };

static int layout_of(const gleam_matrix_dims* d, Layout* l) {
    if (!d) return GLEAM_ERR_NULL_POINTER;
    if (d->struct_version != GLEAM_MATRIX_DIMS_VERSION || d->dtype < GLEAM_F32 || d->dtype > GLEAM_BF16) return GLEAM_ERR_BAD_DIMS;
    if (d->count < 0 || d->rows < 0 || d->cols < 0 || d->count > (1 << 20) || d->rows > (1 << 20) || d->cols > (1 << 20)) return GLEAM_ERR_BAD_DIMS;
    const long long S = std::min(d->rows, d->cols), L = std::max(d->rows, d->cols);
    if (S > 16384) return GLEAM_ERR_BAD_DIMS;
    if (d->turns < 1 || d->turns > 100) return GLEAM_ERR_BAD_DIMS;
    for (const float v : {d->a, d->b, d->c})
        if (!(std::fabs(v) <= 16.f)) return GLEAM_ERR_BAD_DIMS;
    if (!(d->eps > 0.f) || !std::isfinite(d->eps)) return GLEAM_ERR_BAD_DIMS;
    l->sblocks = (int)((S + BLOCK - 1) / BLOCK); l->lblocks = (int)((L + BLOCK - 1) / BLOCK);
    // tiles of a launch are numbered by the y axis of its grid
    if ((long long)l->sblocks * l->lblocks > 65535) return GLEAM_ERR_BAD_DIMS;
    l->group = (int)std::min<long long>(d->count, GROUP);
    l->x = l->square = l->part = 0;
    l->total = d->count && S ? 256 : 0;
    if (l->total == 0 || (d->count <= RESIDENT_COUNT && resident_fits(S, L))) return GLEAM_OK;
    l->x = (uint64_t)l->group * l->sblocks * l->lblocks * BLOCK_BYTES;
    l->square = (uint64_t)l->group * l->sblocks * l->sblocks * BLOCK_BYTES;
    l->part = (uint64_t)GROUP * (PARTS + 1) * sizeof(float);                     // and the norms of X_0
    l->total += 2 * l->x + 2 * l->square + l->part;
    return GLEAM_OK;
}

struct Span { uintptr_t at; uint64_t bytes; bool written; };

// Every matrix of the call: on a device, aligned, and nothing written shared with anything else.
static int check_memory(Span* spans, size_t count) {
    for (size_t i = 0; i < count; ++i) {
        const Span& u = spans[i];
        const int rc = check_device_ptr((const void*)u.at);
        if (rc != GLEAM_OK) return rc;
    }
    std::sort(spans, spans + count, [](const Span& x, const Span& y) { return x.at < y.at; });
    uintptr_t end = 0, written = 0;                 // first byte behind all spans so far, behind the written ones
    for (size_t i = 0; i < count; ++i) {
        const Span& u = spans[i];
        if (u.at < written || (u.written && u.at < end)) return GLEAM_ERR_ALIAS;
        end = std::max<uintptr_t>(end, u.at + u.bytes);
        if (u.written) written = std::max<uintptr_t>(written, u.at + u.bytes);
    }
    return GLEAM_OK;
}

static int orthogonal(const void* const* u, float* const* momenta, void* const* out, const gleam_muon_args* m, const gleam_matrix_dims* d) {
    Layout l;
    int rc = layout_of(d, &l);
    if (rc != GLEAM_OK) return rc;
    if (l.total == 0) return GLEAM_OK;
    if (!u || !out || (m && !momenta) || !d->workspace) return GLEAM_ERR_NULL_POINTER;
    if (d->workspace_bytes < l.total) return GLEAM_ERR_WORKSPACE_TOO_SMALL;
    if ((uintptr_t)d->workspace & 255) return GLEAM_ERR_BAD_DIMS;
    const uint64_t n = (uint64_t)d->rows * d->cols, esize = d->dtype == GLEAM_F32 ? 4 : 2;
    {
        const std::unique_ptr<Span[]> spans(new (std::nothrow) Span[(size_t)d->count * 3 + 1]);     // no exception leaves a C entry
        if (!spans) return GLEAM_ERR_CUDA;
        size_t n_spans = 0;
        spans[n_spans++] = Span{(uintptr_t)d->workspace, l.total, true};
        for (int64_t i = 0; i < d->count; ++i) {
            if (!u[i] || !out[i] || (m && !momenta[i])) return GLEAM_ERR_NULL_POINTER;
            if ((uintptr_t)u[i] % esize || (uintptr_t)out[i] % esize || (m && (uintptr_t)momenta[i] % 4)) return GLEAM_ERR_BAD_DIMS;
            spans[n_spans++] = Span{(uintptr_t)u[i], n * esize, false};
            spans[n_spans++] = Span{(uintptr_t)out[i], n * esize, true};
            if (m) spans[n_spans++] = Span{(uintptr_t)momenta[i], n * 4, true};
        }
        if ((rc = check_memory(spans.get(), n_spans)) != GLEAM_OK) return rc;
    }
    Args a;
    std::memset(&a, 0, sizeof a);
    a.rows = d->rows; a.cols = d->cols; a.S = std::min(d->rows, d->cols); a.L = std::max(d->rows, d->cols);
    a.tall = d->rows > d->cols; a.dtype = d->dtype;
    a.sblocks = l.sblocks; a.lblocks = l.lblocks;
    a.parts = (int)std::max<long long>(1, std::min<long long>(PARTS, (long long)(n / (4 * PREPARE_THREADS))));
    a.a = d->a; a.b = d->b; a.c = d->c; a.eps = d->eps;
    if (m) {
        a.update = 1; a.nesterov = m->nesterov; a.mu = m->momentum;
        a.keep = (float)(1.0 - (double)m->lr * m->weight_decay); a.move = (float)((double)m->lr * m->scale);
    }
    unsigned char* ws = (unsigned char*)d->workspace;
    a.blocks = ws; a.g = ws + 2 * l.x; a.p = a.g + l.square;
    a.part = (float*)(a.p + l.square); a.size = a.part + GROUP * PARTS;
    a.status = (int*)(ws + l.total - 256);
    for (int64_t i0 = 0; i0 < d->count; i0 += GROUP) {
        const int count = (int)std::min<int64_t>(GROUP, d->count - i0);
        a.fresh = i0 == 0;
        if (l.x) { a.x = ws; a.y = ws + l.x; }                          // null: no workspace for the general kernels
        for (int k = 0; k < count; ++k) {
            a.u[k] = u[i0 + k]; a.out[k] = out[i0 + k]; a.momentum[k] = m ? momenta[i0 + k] : nullptr;
        }
        const cudaStream_t s = (cudaStream_t)d->stream;
        const cudaError_t e = d->dtype == GLEAM_F32 ? run_for<float>(a, m != nullptr, count, d->turns, s)
                            : d->dtype == GLEAM_F16 ? run_for<__half>(a, m != nullptr, count, d->turns, s)
                                                    : run_for<__nv_bfloat16>(a, m != nullptr, count, d->turns, s);
        if (e != cudaSuccess) return GLEAM_ERR_CUDA;
    }
    return GLEAM_OK;
}

}  // namespace ortho
}  // namespace gleam

using namespace gleam::ortho;

extern "C" {

GLEAM_API int gleam_orthogonalise_workspace_size(const gleam_matrix_dims* dims, uint64_t* bytes) {
    if (!bytes) return GLEAM_ERR_NULL_POINTER;
    Layout l;
    const int rc = layout_of(dims, &l);
    if (rc != GLEAM_OK) return rc;
    *bytes = l.total;
    return GLEAM_OK;
}

GLEAM_API int gleam_orthogonalise_check_status(const gleam_matrix_dims* dims) {
    Layout l;
    const int rc = layout_of(dims, &l);
    if (rc != GLEAM_OK) return rc;
    if (l.total == 0) return GLEAM_OK;
    if (!dims->workspace) return GLEAM_ERR_NULL_POINTER;
    if (dims->workspace_bytes < l.total) return GLEAM_ERR_WORKSPACE_TOO_SMALL;
    int status = 0;
    const unsigned char* at = (const unsigned char*)dims->workspace + l.total - 256;
    if (cudaMemcpyAsync(&status, at, sizeof status, cudaMemcpyDeviceToHost, (cudaStream_t)dims->stream) != cudaSuccess ||
        cudaStreamSynchronize((cudaStream_t)dims->stream) != cudaSuccess) return GLEAM_ERR_CUDA;
    return status ? GLEAM_ERR_TIMEOUT : GLEAM_OK;
}

GLEAM_API int gleam_orthogonalise(const void* const* x, void* const* out, const gleam_matrix_dims* dims) {
    return orthogonal(x, nullptr, out, nullptr, dims);
}

GLEAM_API int gleam_muon_step(void* const* weights, const void* const* grads, float* const* momenta, const gleam_muon_args* args,
                              const gleam_matrix_dims* dims) {
    if (!args) return GLEAM_ERR_NULL_POINTER;
    for (const float v : {args->lr, args->momentum, args->weight_decay, args->scale})
        if (!std::isfinite(v)) return GLEAM_ERR_BAD_DIMS;
    if (args->lr < 0.f || !(args->momentum >= 0.f && args->momentum < 1.f) || args->weight_decay < 0.f || (args->nesterov != 0 && args->nesterov != 1)) return GLEAM_ERR_BAD_DIMS;
    return orthogonal(grads, momenta, weights, args, dims);
}

}  // extern "C"
