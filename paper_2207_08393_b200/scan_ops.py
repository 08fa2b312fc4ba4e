"""The gated recurrence on torch tensors: h_t = f_t h_(t-1) + (1 - f_t) x_t with f_t = 1 / (1 + exp(-gate_t)) along one axis.

A prior looks along the frames of a cine, the sections of a volume or a row of tokens with it (include/gleam.h states the formulas).
Three layers, as for the other operators of the prior:

* ``gated_scan_forward`` / ``gated_scan_vjp``: the C calls on plain tensors; outputs are allocated, the workspace comes from
  torch's allocator for the current stream, nothing is kept between calls;
* ``gated_scan``: the same as an autograd node, which can be differentiated once;
* ``gated_step``: one new step with the state updated in place, for frames that arrive one at a time.

x, gate and their cotangents are CUDA tensors of one shape and type (float32, float16 or bfloat16); states are float32, contiguous, of that
shape without axis ``dim``.  The axes behind ``dim`` are contiguous and those before it step evenly, apart from axis 0, which
may step on its own: halves of a wider array along an axis before ``dim`` are fine.  ``lengths`` (int32, one for each index of
axis 0) ends each example's chain early: behind its length y and the gradients are 0, what stands there is not used and the state stays.
"""
from __future__ import annotations

import torch

from . import binding as _b
from .prior_ops import _DTYPES, _HERE, _On, _check_kind, _check_sign, _numel, _plain, _steps, _stream


def _check_lengths(x, dim, lengths):
    if lengths is None:
        return
    if dim == 0:
        raise ValueError("lengths: there is no axis of examples before axis 0")
    if lengths.dtype != torch.int32 or lengths.dim() != 1 or lengths.shape[0] != x.shape[0] or lengths.device != x.device or not lengths.is_contiguous():
        raise ValueError("lengths: a contiguous int32 vector of %d values on %s is wanted" % (x.shape[0], x.device))


class _Chains:
    """(batch, channels, steps, inner) of a call, and its structure with the strides of the arrays."""
    __slots__ = ("dim", "sizes", "shape", "device", "dims", "sizes_of_scratch")

    def __init__(self, x, dim, reverse, lengths, *others):
        _check_kind(x)
        shape = x.shape
        if x.dim() == 0 or not -x.dim() <= dim < x.dim():
            raise ValueError("no axis %d in shape %s" % (dim, tuple(shape)))
        self.dim = dim = dim % x.dim()
        self.sizes = (shape[0] if dim else 1, _numel(shape[1:dim]), shape[dim], _numel(shape[dim + 1:]))
        self.shape = shape[:dim] + shape[dim + 1:]
        self.device = _On(x)
        strides = self._strides(x, "x")
        for t, what in others:
            if t is None:                                # an output: contiguous
                strides += (0, 0, 0)
                continue
            if t.shape != shape or t.dtype != x.dtype or t.device != x.device:
                raise ValueError("%s: %s %s on %s where %s %s on %s is wanted" % (what, tuple(t.shape), t.dtype, t.device, tuple(shape),
                                                                                 x.dtype, x.device))
            _check_sign(t)
            strides += self._strides(t, what)
        _check_lengths(x, dim, lengths)
        self.dims = _b.gleam_scan_dims(1, _DTYPES[x.dtype], bool(reverse), 0, *self.sizes, strides, _b._at(lengths), _stream(x) or None,
                                       None, 0)
        self.sizes_of_scratch = None

    def _strides(self, t, what):
        """(batch, channel, step) in elements; all 0 for a contiguous array."""
        if t.is_contiguous() or t.numel() == 0:
            return (0, 0, 0)
        shape, strides, dim = t.shape, t.stride(), self.dim
        want, ok = 1, True
        for k in range(len(shape) - 1, dim, -1):
            ok = ok and (shape[k] == 1 or strides[k] == want)
            want *= shape[k]
        channel, count = 1, 1
        for k in range(dim - 1, 0, -1):
            if shape[k] != 1:
                if count == 1:
                    channel = strides[k]
                ok = ok and strides[k] == channel * count
                count *= shape[k]
        # an axis of length one steps anywhere: by 1, so that not all three are 0
        got = (strides[0] if dim and shape[0] != 1 else 1, channel, strides[dim] if shape[dim] != 1 else 1)
        reach = sorted((s, n) for s, n in zip(got, self.sizes) if n > 1)
        for s, n in reach:
            ok = ok and s >= want
            want = want + s * (n - 1)
        if not ok:
            raise ValueError("%s: memory order not supported (shape %s, strides %s, steps at axis %d): call .contiguous()"
                             % (what, tuple(shape), tuple(strides), dim))
        return got

    def check_state(self, x, t, what):
        if t is not None and (t.shape != self.shape or t.dtype is not torch.float32 or t.device != x.device or not t.is_contiguous()
                              or t.is_neg()):
            raise ValueError("%s: contiguous float32 of shape %s on %s is wanted (.contiguous(), .resolve_neg())"
                             % (what, tuple(self.shape), x.device))

    def state(self, x):
        return torch.empty_strided(self.shape, _steps(self.shape) if self.shape else (), dtype=torch.float32, device=x.device)

    def scratch(self, x, size):
        """Device memory of so many bytes, or None."""
        return torch.empty_strided((size,), (1,), dtype=torch.uint8, device=x.device) if size else None

    def _sizes_of_scratch(self):
        """Bytes of the saved states and of the workspace."""
        if self.sizes_of_scratch is None:
            self.sizes_of_scratch = _b.gleam_gated_scan_saved_size(self.dims), _b.gleam_gated_scan_workspace_size(self.dims)
        return self.sizes_of_scratch

    def saved(self, x):
        return self.scratch(x, self._sizes_of_scratch()[0])

    def workspace(self, x):
        ws = self.scratch(x, self._sizes_of_scratch()[1])
        if ws is not None:
            self.dims.workspace, self.dims.workspace_bytes = ws.data_ptr(), ws.numel()
        return ws


_CALLS = {}                                      # structures of calls on contiguous tensors, by shape, type, axis and direction
_CALLS_MOST = 256                                # beyond that the table starts over
_new_dims = _b.gleam_scan_dims.from_buffer_copy


def _chains(x, dim, reverse, lengths, *others):
    """``_Chains`` of a call; where all tensors are contiguous its structure is copied from a kept one (filling one takes longer than a small
    kernel: forward and VJP of 3 x 5 x 20 x 33 55 -> 43 us a pair)."""
    if not _plain(x, *[t for t, _ in others]):
        return _Chains(x, dim, reverse, lengths, *others)
    key = x.shape, x.dtype, dim, bool(reverse)
    kept = _CALLS.get(key)
    if kept is None:
        c = _Chains(x, dim, reverse, None)
        c.dims.stream = None
        kept = c.dim, c.sizes, c.shape, c._sizes_of_scratch(), bytes(c.dims)
        if len(_CALLS) >= _CALLS_MOST:
            _CALLS.clear()
        _CALLS[key] = kept
    c = _Chains.__new__(_Chains)
    c.dim, c.sizes, c.shape, c.sizes_of_scratch, template = kept
    c.device = _HERE
    c.dims = _new_dims(template)
    c.dims.stream = _b._current_stream_handle() or None
    if lengths is not None:
        _check_lengths(x, c.dim, lengths)
        c.dims.lengths = lengths.data_ptr()
    return c


def _new(x):
    return torch.empty_like(x) if x.is_contiguous() else torch.empty(x.shape, dtype=x.dtype, device=x.device)


def gated_scan_forward(x, gate, state=None, lengths=None, dim=-2, reverse=False, save=True):
    """(y, last, saved): y_t = h_t in x's type, last = the state behind the last step, saved = what ``gated_scan_vjp`` needs besides
    x and gate (None with ``save=False``).  ``state`` (None: zeros) is the state before the first step."""
    c = _chains(x, dim, reverse, lengths, (gate, "gate"), (None, "y"))
    c.check_state(x, state, "state")
    y, last = _new(x), c.state(x)
    with c.device:
        starts = c.saved(x) if save else None
        ws = c.workspace(x)
        _b.gleam_gated_scan_forward(x, gate, state, y, last, starts, c.dims)
    del ws
    return y, last, (starts, state) if save else None


def gated_scan_vjp(grad_y, grad_last, x, gate, saved, lengths=None, dim=-2, reverse=False, state_grad=True):
    """(grad_x, grad_gate, grad_state) of ``gated_scan_forward`` for the cotangents of y and last (``grad_last`` None: zero); the last
    one is None where it is not wanted.  x, gate, lengths and the state given there are what they were."""
    c = _chains(x, dim, reverse, lengths, (gate, "gate"), (grad_y, "grad_y"))
    c.check_state(x, grad_last, "grad_last")
    if saved is None:
        raise ValueError("saved: the forward call was made with save=False")
    starts, state = saved
    c.check_state(x, state, "state")
    if c.device is not _HERE:
        s = tuple(c.dims.stride)
        c.dims.stride = s[6:9] + s[:6] + (0,) * 6            # in the order of the call: grad_y, x, gate, then the outputs
    gx, gg = _new(x), _new(x)
    gs = c.state(x) if state_grad else None
    with c.device:
        need = c._sizes_of_scratch()[0]
        if need and (starts is None or starts.numel() != need or starts.device != x.device):
            raise ValueError("saved: the forward call on these sizes saves %d bytes on %s" % (need, x.device))
        ws = c.workspace(x)
        _b.gleam_gated_scan_vjp(grad_y, grad_last, x, gate, state, starts, gx, gg, gs, c.dims)
    del ws
    return gx, gg, gs


_AXIS_MOST = 1 << 31                             # elements of an axis of a call


def _step_sizes(shape):
    """(batch, inner) of a step on contiguous tensors: all in one run, or two factors where that is more than an axis of the call holds."""
    batch, inner = 1, _numel(shape)
    for s in shape:
        if inner <= _AXIS_MOST:
            break
        batch, inner = batch * s, inner // s
    if max(batch, inner) > _AXIS_MOST:
        raise ValueError("an axis of more than 2^31 elements (shape %s)" % (tuple(shape),))
    return batch, inner


_STEPS = {}                                      # structures of steps on contiguous tensors, by shape and type
_STEPS_MOST = 256                                # beyond that the table starts over


def _changed(t):
    """Tells autograd that a tensor was written in place, as torch's own operators do."""
    if not t.is_inference():
        torch.autograd.graph.increment_version(t)


def gated_step(x, gate, state):
    """One step: state <- f state + (1 - f) x in place; returns the new state in x's type.  x, gate and state have one shape.  Not
    differentiable: gradients go through ``gated_scan``."""
    if torch.is_grad_enabled() and any(isinstance(t, torch.Tensor) and t.requires_grad for t in (x, gate, state)):
        raise ValueError("single steps are not differentiable: use gated_scan, or torch.no_grad()")
    if _plain(x, gate) and isinstance(state, torch.Tensor) and state.shape == x.shape and state.dtype is torch.float32 and \
            state.is_contiguous() and state.get_device() == x.get_device() and not state.is_neg():
        key = x.shape, x.dtype                   # filling a structure takes longer than the kernel (18.7 -> 11 us a call)
        kept = _STEPS.get(key)
        if kept is None:
            batch, inner = _step_sizes(x.shape)
            kept = bytes(_b.gleam_scan_dims(1, _DTYPES[x.dtype], 0, 0, batch, 1, 1, inner))
            if len(_STEPS) >= _STEPS_MOST:
                _STEPS.clear()
            _STEPS[key] = kept
        dims = _new_dims(kept)
        dims.stream = _b._current_stream_handle() or None
        y = torch.empty_like(x)
        _b.gleam_gated_step(x, gate, state, y, dims)
        _changed(state)
        return y
    _check_kind(x)
    at = 1 if x.dim() > 1 else 0
    c = _Chains(x.unsqueeze(at), at, False, None, (gate.unsqueeze(at) if gate.dim() >= at else gate, "gate"), (None, "y"))
    if state is None:
        raise ValueError("state: there is none to update")
    c.check_state(x, state, "state")
    y = _new(x)
    with c.device:
        _b.gleam_gated_step(x, gate, state, y, c.dims)
    _changed(state)
    return y


# ---- autograd ------------------------------------------------------------------------------------------------------------

def _viewable(t, x, dim):
    """``t`` itself if the calls take it or refuse it, else a contiguous copy (cotangents come in any order)."""
    t = t.resolve_neg()
    if t.shape != x.shape or t.is_contiguous():
        return t
    try:
        _Chains(t, dim, False, None)
        return t
    except ValueError:
        return t.contiguous()


class _GatedScan(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gate, state, lengths, dim, reverse):
        y, last, (starts, _) = gated_scan_forward(x, gate, state, lengths, dim, reverse)
        ctx.save_for_backward(x, gate, state, lengths, starts)
        ctx.args = dim, reverse
        ctx.set_materialize_grads(False)
        return y, last

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_y, grad_last):
        x, gate, state, lengths, starts = ctx.saved_tensors
        dim, reverse = ctx.args
        if grad_y is None and grad_last is None:
            return (None,) * 6
        grad_y = torch.zeros_like(x, memory_format=torch.contiguous_format) if grad_y is None else _viewable(grad_y, x, dim)
        grad_last = None if grad_last is None else grad_last.resolve_neg().contiguous()
        gx, gg, gs = gated_scan_vjp(grad_y, grad_last, x, gate, (starts, state), lengths, dim, reverse, ctx.needs_input_grad[2])
        return gx, gg, gs, None, None, None


def gated_scan(x, gate, state=None, lengths=None, dim=-2, reverse=False):
    """(y, last) of the recurrence, with gradients for x, gate and state."""
    if state is not None:
        state = state.resolve_neg().contiguous()
    return _GatedScan.apply(_viewable(x, x, dim), _viewable(gate, x, dim), state, lengths, dim, reverse)
