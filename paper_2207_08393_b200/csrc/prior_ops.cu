// Host side of the prior's operators (layer norm, dropout, residual tail): argument checks, workspace, choice of the type.
#include "../../include/gleam.h"
#include "dc_entry.h"
#include "prior_entry.h"

#include <cmath>
#include <cstring>

namespace gleam {
namespace prior {

static const Ops* find_ops(int dtype) {
    return dtype == GLEAM_F32 ? &ops_f32 : dtype == GLEAM_F16 ? &ops_f16 : dtype == GLEAM_BF16 ? &ops_bf16 : nullptr;
}

// An activation array of a call.
struct Array {
    const void* p;
    long long pitch;
    bool written, needed;
};

struct Call {
    const gleam_feature_dims* d;
    long long slice, esize;
    Array arrays[5];
    int count;

    // first byte behind the last slice
    uint64_t bytes(const Array& v) const { return (uint64_t)((d->outer - 1) * v.pitch + slice) * (uint64_t)esize; }

    bool meet(const Array& u, const Array& v) const {
        const uintptr_t u0 = (uintptr_t)u.p, v0 = (uintptr_t)v.p;
        if (u0 >= v0 + bytes(v) || v0 >= u0 + bytes(u)) return false;
        // slices of one wider array, side by side: apart if they are so modulo the pitch
        if (u.pitch == v.pitch && d->outer > 1) {
            const uint64_t pitch = (uint64_t)(u.pitch * esize), wide = (uint64_t)(slice * esize);
            const uint64_t gap = u0 > v0 ? (u0 - v0) % pitch : (pitch - (v0 - u0) % pitch) % pitch;     // from v's slice to u's
            return gap < wide || gap + wide > pitch;
        }
        return true;
    }
};

static bool span_meets(const Call& c, const Array& v, const void* p, uint64_t n) {
    const uintptr_t a0 = (uintptr_t)v.p, b0 = (uintptr_t)p;
    return v.p && p && n && a0 < b0 + n && b0 < a0 + c.bytes(v);
}

static int check_dims(const gleam_feature_dims* d) {
    if (!d) return GLEAM_ERR_NULL_POINTER;
    if (d->struct_version != GLEAM_FEATURE_DIMS_VERSION) return GLEAM_ERR_BAD_DIMS;
    if (!find_ops(d->dtype) || (d->weight_dtype != GLEAM_F32 && d->weight_dtype != d->dtype)) return GLEAM_ERR_BAD_DIMS;
    if (d->features < 1 || d->outer < 0 || d->inner < 0) return GLEAM_ERR_BAD_DIMS;
    const long long most = 1ll << 46;
    if (d->features > (1ll << 24) || d->inner > most / d->features || (d->inner && d->outer > most / (d->features * d->inner))) return GLEAM_ERR_BAD_DIMS;
    for (int i = 0; i < 5; ++i)
        if (d->pitch[i] != 0 && (d->pitch[i] < d->features * d->inner || d->pitch[i] > most || (d->outer && d->pitch[i] > most / d->outer))) return GLEAM_ERR_BAD_DIMS;
    return GLEAM_OK;
}

// Fills the parts of the arguments that every call has, and checks the activation arrays.
static int begin(const gleam_feature_dims* d, Call* c, Args* a) {
    const int rc = check_dims(d);
    if (rc != GLEAM_OK) return rc;
    c->d = d;
    c->slice = d->features * d->inner;
    c->esize = d->dtype == GLEAM_F32 ? 4 : 2;
    for (int i = 0; i < c->count; ++i) {
        Array& v = c->arrays[i];
        if (!v.p && v.needed && d->outer && d->inner) return GLEAM_ERR_NULL_POINTER;
        v.pitch = d->pitch[i] ? d->pitch[i] : c->slice;
        if ((uintptr_t)v.p % (uintptr_t)c->esize) return GLEAM_ERR_BAD_DIMS;
    }
    std::memset(a, 0, sizeof *a);
    a->outer = d->outer; a->features = d->features; a->inner = d->inner;
    a->eps = d->eps; a->scale = 1.f;
    a->weight_f32 = d->weight_dtype == GLEAM_F32;
    return GLEAM_OK;
}

static int take_dropout(const gleam_dropout_args* m, Args* a) {
    if (!m) return GLEAM_ERR_NULL_POINTER;
    if (!(m->p >= 0.0 && m->p <= 1.0)) return GLEAM_ERR_BAD_DIMS;
    if ((uintptr_t)m->step & 7) return GLEAM_ERR_BAD_DIMS;
    a->scale = m->p < 1.0 ? (float)(1.0 / (1.0 - m->p)) : 0.f;
    const uint64_t limit = (uint64_t)std::floor(m->p * 4294967296.0);
    a->dropping = limit > 0;
    a->last = limit > 0 ? (uint32_t)(limit - 1) : 0;
    a->offset = m->offset;
    uint32_t k0 = (uint32_t)m->seed, k1 = (uint32_t)(m->seed >> 32);
    for (int r = 0; r < 10; ++r, k0 += 0x9E3779B9u, k1 += 0xBB67AE85u) { a->keys[2 * r] = k0; a->keys[2 * r + 1] = k1; }
    a->step = (const unsigned long long*)m->step;
    return GLEAM_OK;
}

// A vector of features or positions next to the activation arrays.
struct Small { const void* p; uint64_t bytes; int align; bool written; };

static int check_memory(const Call& c, const Small* small, int count) {
    const bool nothing = c.d->outer == 0 || c.d->inner == 0;
    int rc;
    for (int i = 0; i < count; ++i) {
        if ((uintptr_t)small[i].p % (uintptr_t)small[i].align) return GLEAM_ERR_BAD_DIMS;
        if (small[i].p && (rc = check_device_ptr(small[i].p)) != GLEAM_OK) return rc;
        for (int k = 0; k < i; ++k) {
            if ((!small[i].written && !small[k].written) || !small[i].p || !small[k].p) continue;
            const uintptr_t u = (uintptr_t)small[i].p, v = (uintptr_t)small[k].p;
            if (u < v + small[k].bytes && v < u + small[i].bytes) return GLEAM_ERR_ALIAS;
        }
    }
    if (nothing) return GLEAM_OK;                        // the arrays have no elements
    for (int i = 0; i < c.count; ++i) {
        const Array& u = c.arrays[i];
        if (!u.p) continue;
        if ((rc = check_device_ptr(u.p)) != GLEAM_OK) return rc;
        for (int k = 0; k < i; ++k) {
            const Array& v = c.arrays[k];
            if (!v.p || (!u.written && !v.written)) continue;
            const bool same = u.p == v.p && u.pitch == v.pitch && u.written != v.written;
            if (!same && c.meet(u, v)) return GLEAM_ERR_ALIAS;
        }
        for (int k = 0; k < count; ++k)
            if ((u.written || small[k].written) && span_meets(c, u, small[k].p, small[k].bytes)) return GLEAM_ERR_ALIAS;
    }
    return GLEAM_OK;
}

static uint64_t part_bytes(const Args& a) { return (uint64_t)parts_most(a) * 2u * (uint64_t)a.features * sizeof(float); }

static int status_of(cudaError_t e) { return e == cudaSuccess ? GLEAM_OK : GLEAM_ERR_CUDA; }

static int norm_forward(Call& c, Args& a, const void* weight, const void* bias, float* mean, float* rstd, bool tail) {
    const gleam_feature_dims* d = c.d;
    if (!(d->eps >= 0.f) || !std::isfinite(d->eps)) return GLEAM_ERR_BAD_DIMS;
    const uint64_t positions = (uint64_t)(d->outer * d->inner) * sizeof(float);
    const int wsize = a.weight_f32 ? 4 : 2;
    const uint64_t wbytes = (uint64_t)d->features * wsize;
    const Small small[5] = {{weight, wbytes, wsize, false}, {bias, wbytes, wsize, false}, {mean, positions, 4, true}, {rstd, positions, 4, true},
                            {a.step, a.step ? 8u : 0u, 8, false}};
    const int rc = check_memory(c, small, 5);
    if (rc != GLEAM_OK || d->outer == 0 || d->inner == 0) return rc;
    a.weight = weight; a.bias = bias; a.mean = mean; a.rstd = rstd;
    return status_of(find_ops(d->dtype)->forward(a, tail, (cudaStream_t)d->stream));
}

static int norm_vjp(Call& c, Args& a, const void* weight, const float* mean, const float* rstd, void* gw, void* gb, bool tail) {
    const gleam_feature_dims* d = c.d;
    const bool nothing = d->outer == 0 || d->inner == 0, sums = (gw || gb) && !nothing;
    if (!nothing && (!mean || !rstd)) return GLEAM_ERR_NULL_POINTER;
    const uint64_t positions = (uint64_t)(d->outer * d->inner) * sizeof(float), need = sums ? part_bytes(a) : 0;
    if (sums) {
        if (!d->workspace) return GLEAM_ERR_NULL_POINTER;
        if (d->workspace_bytes < need) return GLEAM_ERR_WORKSPACE_TOO_SMALL;
        if ((uintptr_t)d->workspace & 255) return GLEAM_ERR_BAD_DIMS;
    }
    const int wsize = a.weight_f32 ? 4 : 2;
    const uint64_t wbytes = (uint64_t)d->features * wsize;
    const Small small[7] = {{weight, wbytes, wsize, false}, {mean, positions, 4, false}, {rstd, positions, 4, false}, {gw, wbytes, wsize, true},
                            {gb, wbytes, wsize, true}, {sums ? d->workspace : nullptr, need, 1, true}, {a.step, a.step ? 8u : 0u, 8, false}};
    const int rc = check_memory(c, small, 7);
    if (rc != GLEAM_OK) return rc;
    cudaStream_t s = (cudaStream_t)d->stream;
    if (nothing) {
        if (gw && cudaMemsetAsync(gw, 0, wbytes, s) != cudaSuccess) return GLEAM_ERR_CUDA;
        if (gb && cudaMemsetAsync(gb, 0, wbytes, s) != cudaSuccess) return GLEAM_ERR_CUDA;
        return GLEAM_OK;
    }
    a.weight = weight; a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
    a.gw = gw; a.gb = gb; a.part = sums ? (float*)d->workspace : nullptr;
    return status_of(find_ops(d->dtype)->vjp(a, tail, s));
}

static int drop(Call& c, Args& a) {
    const gleam_feature_dims* d = c.d;
    const Small small[1] = {{a.step, a.step ? 8u : 0u, 8, false}};
    const int rc = check_memory(c, small, 1);
    if (rc != GLEAM_OK || d->outer == 0 || d->inner == 0) return rc;
    return status_of(find_ops(d->dtype)->dropout(a, (cudaStream_t)d->stream));
}

}  // namespace prior
}  // namespace gleam

using namespace gleam::prior;

extern "C" {

GLEAM_API int gleam_layer_norm_workspace_size(const gleam_feature_dims* dims, uint64_t* bytes) {
    if (!bytes) return GLEAM_ERR_NULL_POINTER;
    Call c{}; Args a;
    const int rc = begin(dims, &c, &a);
    if (rc != GLEAM_OK) return rc;
    *bytes = dims->outer && dims->inner ? part_bytes(a) : 0;
    return GLEAM_OK;
}

GLEAM_API int gleam_layer_norm_forward(const void* x, const void* weight, const void* bias, void* y, float* mean, float* rstd,
                                       const gleam_feature_dims* dims) {
    Call c{nullptr, 0, 0, {{x, 0, false, true}, {y, 0, true, true}}, 2}; Args a;
    const int rc = begin(dims, &c, &a);
    if (rc != GLEAM_OK) return rc;
    a.x = x; a.px = c.arrays[0].pitch; a.out = y; a.pout = c.arrays[1].pitch;
    return norm_forward(c, a, weight, bias, mean, rstd, false);
}

GLEAM_API int gleam_layer_norm_vjp(const void* grad_y, const void* x, const void* weight, const float* mean, const float* rstd,
                                   void* grad_x, void* grad_weight, void* grad_bias, const gleam_feature_dims* dims) {
    Call c{nullptr, 0, 0, {{grad_y, 0, false, true}, {x, 0, false, true}, {grad_x, 0, true, true}}, 3}; Args a;
    const int rc = begin(dims, &c, &a);
    if (rc != GLEAM_OK) return rc;
    a.x = grad_y; a.px = c.arrays[0].pitch; a.res = x; a.pres = c.arrays[1].pitch; a.out = grad_x; a.pout = c.arrays[2].pitch;
    return norm_vjp(c, a, weight, mean, rstd, grad_weight, grad_bias, false);
}

GLEAM_API int gleam_dropout_forward(const void* x, const void* residual, void* out, const gleam_dropout_args* dropout,
                                    const gleam_feature_dims* dims) {
    Call c{nullptr, 0, 0, {{x, 0, false, true}, {residual, 0, false, false}, {out, 0, true, true}}, 3}; Args a;
    int rc = begin(dims, &c, &a);
    if (rc != GLEAM_OK || (rc = take_dropout(dropout, &a)) != GLEAM_OK) return rc;
    a.x = x; a.px = c.arrays[0].pitch; a.res = residual; a.pres = c.arrays[1].pitch; a.out = out; a.pout = c.arrays[2].pitch;
    return drop(c, a);
}

GLEAM_API int gleam_dropout_vjp(const void* grad_out, void* grad_x, const gleam_dropout_args* dropout,
                                const gleam_feature_dims* dims) {
    Call c{nullptr, 0, 0, {{grad_out, 0, false, true}, {grad_x, 0, true, true}}, 2}; Args a;
    int rc = begin(dims, &c, &a);
    if (rc != GLEAM_OK || (rc = take_dropout(dropout, &a)) != GLEAM_OK) return rc;
    a.x = grad_out; a.px = c.arrays[0].pitch; a.out = grad_x; a.pout = c.arrays[1].pitch;
    return drop(c, a);
}

GLEAM_API int gleam_dropout_add_layer_norm_forward(const void* x, const void* residual, const void* weight, const void* bias,
                                                   void* sum, void* y, float* mean, float* rstd,
                                                   const gleam_dropout_args* dropout, const gleam_feature_dims* dims) {
    Call c{nullptr, 0, 0, {{x, 0, false, true}, {residual, 0, false, true}, {sum, 0, true, true}, {y, 0, true, true}}, 4}; Args a;
    int rc = begin(dims, &c, &a);
    if (rc != GLEAM_OK || (rc = take_dropout(dropout, &a)) != GLEAM_OK) return rc;
    a.x = x; a.px = c.arrays[0].pitch; a.res = residual; a.pres = c.arrays[1].pitch;
    a.out2 = sum; a.pout2 = c.arrays[2].pitch; a.out = y; a.pout = c.arrays[3].pitch;
    return norm_forward(c, a, weight, bias, mean, rstd, true);
}

GLEAM_API int gleam_dropout_add_layer_norm_vjp(const void* grad_y, const void* grad_sum, const void* sum, const void* weight,
                                               const float* mean, const float* rstd, void* grad_x, void* grad_residual,
                                               void* grad_weight, void* grad_bias, const gleam_dropout_args* dropout,
                                               const gleam_feature_dims* dims) {
    Call c{nullptr, 0, 0, {{grad_y, 0, false, true}, {grad_sum, 0, false, false}, {sum, 0, false, true}, {grad_x, 0, true, true},
                           {grad_residual, 0, true, true}}, 5}; Args a;
    int rc = begin(dims, &c, &a);
    if (rc != GLEAM_OK || (rc = take_dropout(dropout, &a)) != GLEAM_OK) return rc;
    a.x = grad_y; a.px = c.arrays[0].pitch; a.gsum = grad_sum; a.pgsum = c.arrays[1].pitch; a.res = sum; a.pres = c.arrays[2].pitch;
    a.out = grad_x; a.pout = c.arrays[3].pitch; a.out2 = grad_residual; a.pout2 = c.arrays[4].pitch;
    return norm_vjp(c, a, weight, mean, rstd, grad_weight, grad_bias, true);
}

}  // extern "C"
