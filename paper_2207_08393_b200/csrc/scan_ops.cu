// Host side of the gated recurrence: argument checks, workspace, choice of the type.
#include "../../include/gleam.h"
#include "dc_entry.h"
#include "scan_entry.h"

#include <algorithm>
#include <cstring>

namespace gleam {
namespace scan {

static const Ops* find_ops(int dtype) {
    return dtype == GLEAM_F32 ? &ops_f32 : dtype == GLEAM_F16 ? &ops_f16 : dtype == GLEAM_BF16 ? &ops_bf16 : nullptr;
}

// Memory that a call reads or writes.
struct Span { const void* p; uint64_t bytes; bool written; };

struct Call {
    const gleam_scan_dims* d;
    const Ops* ops;
    Args a;
    long long saved, scratch;
    Span spans[11];                    // the VJP: five arrays, three of states, saved, workspace, lengths
    int count;

    void add(const void* p, uint64_t bytes, bool written) {
        if (p && bytes) spans[count++] = Span{p, bytes, written};
    }
};

static int check_dims(const gleam_scan_dims* d) {
    if (!d) return GLEAM_ERR_NULL_POINTER;
    if (d->struct_version != GLEAM_SCAN_DIMS_VERSION || !find_ops(d->dtype) || (d->reverse != 0 && d->reverse != 1) || d->reserved != 0) return GLEAM_ERR_BAD_DIMS;
    const long long most = 1ll << 37;
    long long n = 1;
    for (long long v : {(long long)d->batch, (long long)d->channels, (long long)d->inner, (long long)d->steps}) {
        if (v < 0 || v > (1ll << 31)) return GLEAM_ERR_BAD_DIMS;
        if (n && v > most / n) return GLEAM_ERR_BAD_DIMS;
        n *= v;
    }
    if (d->steps > (1ll << 31) - (1 << 16)) return GLEAM_ERR_BAD_DIMS;             // counted in 32 bits, tiles beyond the end included
    if ((uintptr_t)d->lengths % 4) return GLEAM_ERR_BAD_DIMS;
    return GLEAM_OK;
}

static int begin(const gleam_scan_dims* d, Call* c) {
    const int rc = check_dims(d);
    if (rc != GLEAM_OK) return rc;
    std::memset(c, 0, sizeof *c);
    c->d = d;
    c->ops = find_ops(d->dtype);
    c->a.batch = d->batch; c->a.channels = d->channels; c->a.steps = d->steps; c->a.inner = d->inner;
    c->a.lengths = d->lengths;
    c->ops->plan(c->a, &c->saved, &c->scratch);
    return GLEAM_OK;
}

// Strides of activation array number i.  No two elements of an array share memory.
static int take_array(Call* c, int i, const void* p, bool written, Strides* s) {
    const gleam_scan_dims* d = c->d;
    const int64_t* v = d->stride[i];
    const long long esize = d->dtype == GLEAM_F32 ? 4 : 2;
    *s = Strides{d->channels * d->steps * d->inner, d->steps * d->inner, d->inner};
    if (v[0] || v[1] || v[2]) *s = Strides{v[0], v[1], v[2]};
    if (c->a.rows == 0 || d->steps == 0) return GLEAM_OK;                // no elements
    if (!p) return GLEAM_ERR_NULL_POINTER;
    if ((uintptr_t)p % (uintptr_t)esize) return GLEAM_ERR_BAD_DIMS;
    struct Axis { long long stride, count; } axes[3] = {{s->batch, d->batch}, {s->channel, d->channels}, {s->step, d->steps}};
    std::sort(axes, axes + 3, [](const Axis& x, const Axis& y) { return x.stride < y.stride; });
    long long wide = d->inner;
    for (const Axis& x : axes) {
        if (x.count <= 1) continue;
        if (x.stride < wide || x.stride > (1ll << 46) / x.count) return GLEAM_ERR_BAD_DIMS;
        wide += x.stride * (x.count - 1);
    }
    c->add(p, (uint64_t)wide * (uint64_t)esize, written);
    return GLEAM_OK;
}

static int take_states(Call* c, const void* p, bool written) {
    if ((uintptr_t)p % 4) return GLEAM_ERR_BAD_DIMS;
    c->add(p, (uint64_t)c->a.rows * sizeof(float), written);
    return GLEAM_OK;
}

// Workspace and saved states; then all memory of the call: on a device, and nothing that is written shared with anything else.
static int check_memory(Call* c, const void* saved, bool saves, bool parts) {
    const gleam_scan_dims* d = c->d;
    if (saved) {
        if ((uintptr_t)saved & 15) return GLEAM_ERR_BAD_DIMS;
        c->add(saved, (uint64_t)c->saved * sizeof(float), saves);
    }
    if (parts && c->scratch) {
        const uint64_t need = (uint64_t)c->scratch * sizeof(float);
        if (!d->workspace) return GLEAM_ERR_NULL_POINTER;
        if (d->workspace_bytes < need) return GLEAM_ERR_WORKSPACE_TOO_SMALL;
        if ((uintptr_t)d->workspace & 255) return GLEAM_ERR_BAD_DIMS;
        c->add(d->workspace, need, true);
        c->a.maps_a = (float*)d->workspace;
        c->a.maps_b = c->a.maps_a + c->scratch / 2;
    }
    c->add(d->lengths, (uint64_t)d->batch * sizeof(int32_t), false);
    for (int i = 0; i < c->count; ++i) {
        const Span& u = c->spans[i];
        const int rc = check_device_ptr(u.p);
        if (rc != GLEAM_OK) return rc;
        for (int k = 0; k < i; ++k) {
            const Span& v = c->spans[k];
            if ((u.written || v.written) && (uintptr_t)u.p < (uintptr_t)v.p + v.bytes && (uintptr_t)v.p < (uintptr_t)u.p + u.bytes) return GLEAM_ERR_ALIAS;
        }
    }
    return GLEAM_OK;
}

// Chains without steps: the state at the end is the one at the start.
static int pass_on(const float* from, float* to, long long rows, cudaStream_t s) {
    if (!to) return GLEAM_OK;
    const size_t n = (size_t)rows * sizeof(float);
    const cudaError_t e = from ? cudaMemcpyAsync(to, from, n, cudaMemcpyDeviceToDevice, s) : cudaMemsetAsync(to, 0, n, s);
    return e == cudaSuccess ? GLEAM_OK : GLEAM_ERR_CUDA;
}

static int status_of(cudaError_t e) { return e == cudaSuccess ? GLEAM_OK : GLEAM_ERR_CUDA; }

}  // namespace scan
}  // namespace gleam

using namespace gleam::scan;

#define TRY(call) do { const int rc_ = (call); if (rc_ != GLEAM_OK) return rc_; } while (0)

extern "C" {

GLEAM_API int gleam_gated_scan_workspace_size(const gleam_scan_dims* dims, uint64_t* bytes) {
    if (!bytes) return GLEAM_ERR_NULL_POINTER;
    Call c;
    TRY(begin(dims, &c));
    *bytes = (uint64_t)c.scratch * sizeof(float);
    return GLEAM_OK;
}

GLEAM_API int gleam_gated_scan_saved_size(const gleam_scan_dims* dims, uint64_t* bytes) {
    if (!bytes) return GLEAM_ERR_NULL_POINTER;
    Call c;
    TRY(begin(dims, &c));
    *bytes = (uint64_t)c.saved * sizeof(float);
    return GLEAM_OK;
}

GLEAM_API int gleam_gated_scan_forward(const void* x, const void* gate, const float* state, void* y, float* last, float* saved,
                                       const gleam_scan_dims* dims) {
    Call c;
    TRY(begin(dims, &c));
    Args& a = c.a;
    a.x = x; a.gate = gate; a.y = y; a.state = state; a.last = last; a.saved = saved;
    TRY(take_array(&c, 0, x, false, &a.sx));
    TRY(take_array(&c, 1, gate, false, &a.sgate));
    TRY(take_array(&c, 2, y, true, &a.sy));
    TRY(take_states(&c, state, false));
    TRY(take_states(&c, last, true));
    TRY(check_memory(&c, saved, true, true));
    if (a.rows == 0) return GLEAM_OK;
    if (a.steps == 0) return pass_on(state, last, a.rows, (cudaStream_t)dims->stream);
    return status_of(c.ops->forward(a, dims->reverse != 0, (cudaStream_t)dims->stream));
}

GLEAM_API int gleam_gated_scan_vjp(const void* grad_y, const float* grad_last, const void* x, const void* gate, const float* state,
                                   const float* saved, void* grad_x, void* grad_gate, float* grad_state, const gleam_scan_dims* dims) {
    Call c;
    TRY(begin(dims, &c));
    Args& a = c.a;
    a.dy = grad_y; a.x = x; a.gate = gate; a.dx = grad_x; a.dg = grad_gate;
    a.state = state; a.dlast = grad_last; a.dstate = grad_state; a.saved = const_cast<float*>(saved);
    TRY(take_array(&c, 0, grad_y, false, &a.sdy));
    TRY(take_array(&c, 1, x, false, &a.sx));
    TRY(take_array(&c, 2, gate, false, &a.sgate));
    TRY(take_array(&c, 3, grad_x, true, &a.sdx));
    TRY(take_array(&c, 4, grad_gate, true, &a.sdg));
    TRY(take_states(&c, state, false));
    TRY(take_states(&c, grad_last, false));
    TRY(take_states(&c, grad_state, true));
    if (!saved && c.saved) return GLEAM_ERR_NULL_POINTER;
    TRY(check_memory(&c, saved, false, true));
    if (a.rows == 0) return GLEAM_OK;
    if (a.steps == 0) return pass_on(grad_last, grad_state, a.rows, (cudaStream_t)dims->stream);
    return status_of(c.ops->vjp(a, dims->reverse != 0, (cudaStream_t)dims->stream));
}

GLEAM_API int gleam_gated_step(const void* x, const void* gate, float* state, void* y, const gleam_scan_dims* dims) {
    Call c;
    TRY(begin(dims, &c));
    if (dims->steps != 1 || dims->lengths) return GLEAM_ERR_BAD_DIMS;
    Args& a = c.a;
    a.x = x; a.gate = gate; a.y = y; a.last = state;
    TRY(take_array(&c, 0, x, false, &a.sx));
    TRY(take_array(&c, 1, gate, false, &a.sgate));
    TRY(take_array(&c, 2, y, true, &a.sy));
    if (!state && a.rows) return GLEAM_ERR_NULL_POINTER;
    TRY(take_states(&c, state, true));
    TRY(check_memory(&c, nullptr, false, false));
    if (a.rows == 0) return GLEAM_OK;
    return status_of(c.ops->step(a, (cudaStream_t)dims->stream));
}

}  // extern "C"
