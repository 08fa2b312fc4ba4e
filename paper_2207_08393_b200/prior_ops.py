"""Operators of the learned prior on torch tensors: layer norm, dropout, and the residual tail that joins them.

Two layers over the C calls (include/gleam.h states the formulas and the definition of the dropout mask):

* ``*_forward`` / ``*_vjp``: one C call each on plain tensors; outputs are allocated, the workspace comes from torch's
  allocator for the current stream, nothing is kept between calls;
* ``layer_norm``, ``dropout``, ``dropout_add_layer_norm``: the same as autograd nodes, which can be differentiated once.

Tensors are CUDA tensors of float32, float16 or bfloat16, all of one type and shape; weights are float32 or of that type.
``dim`` is the axis of the features.  A tensor may be a slice of a wider one along an axis before ``dim`` or along ``dim`` itself,
or hold the features last in memory (``torch.channels_last``); any other order is refused.  No result depends on the layout
but the dropout mask, which numbers the elements in memory order.
"""
from __future__ import annotations

import threading

import torch

from . import binding as _b

_DTYPES = {torch.float32: _b.GLEAM_F32, torch.float16: _b.GLEAM_F16, torch.bfloat16: _b.GLEAM_BF16}


class _View:
    """(outer, features, inner) view of a tensor's memory; ``last`` where the features are last in memory but not in the shape."""
    __slots__ = ("outer", "features", "inner", "pitch", "last")

    def __init__(self, outer, features, inner, pitch, last):
        self.outer, self.features, self.inner, self.pitch, self.last = outer, features, inner, pitch, last


def _numel(sizes):
    n = 1
    for s in sizes:
        n *= s
    return n


def _steps(shape):
    """Strides of a contiguous tensor."""
    if len(shape) == 1:
        return (1,)
    steps, n = [], 1
    for s in reversed(shape):
        steps.append(n)
        n *= s
    return steps[::-1]


def _slices(shape, strides, dim):
    """(outer, inner, pitch) if the axes from ``dim`` on are contiguous and those before step evenly, else None.  An axis of
    length one steps anywhere."""
    want = 1
    for k in range(len(shape) - 1, dim - 1, -1):
        if shape[k] != 1:
            if strides[k] != want:
                return None
            want *= shape[k]
    outer, pitch = 1, 0
    for k in range(dim - 1, -1, -1):
        if shape[k] == 1:
            continue
        if outer == 1:
            pitch = strides[k]
            if pitch < want:
                return None
        elif strides[k] != pitch * outer:
            return None
        outer *= shape[k]
    return outer, _numel(shape[dim + 1:]), 0 if pitch == want else pitch


def _view(t, dim):
    shape = t.shape
    if t.is_contiguous() or t.numel() == 0:
        return _View(_numel(shape[:dim]), shape[dim], _numel(shape[dim + 1:]), 0, False)
    got = _slices(shape, t.stride(), dim)
    if got is not None:
        return _View(got[0], shape[dim], got[1], got[2], False)
    m = t.movedim(dim, -1)
    got = _slices(m.shape, m.stride(), len(shape) - 1)
    if got is not None:
        return _View(got[0], shape[dim], 1, got[2], True)
    raise ValueError("memory order not supported (shape %s, strides %s, features at axis %d): call .contiguous()"
                     % (tuple(shape), tuple(t.stride()), dim))


def _like(t, dim, view):
    """A dense tensor of the same shape, type and order."""
    if not view.last:
        return torch.empty(t.shape, dtype=t.dtype, device=t.device)
    shape = list(t.shape)
    shape.append(shape.pop(dim))
    return torch.empty(shape, dtype=t.dtype, device=t.device).movedim(-1, dim)


def _check_kind(x):
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise ValueError("expected CUDA tensors: there is no CPU fallback")
    if x.dtype not in _DTYPES:
        raise ValueError("type %s is not supported" % x.dtype)
    _check_sign(x)


def _check_sign(t):
    if t.is_neg():                                   # a view that torch negates when it reads it
        raise ValueError("memory holds the negated values: call .resolve_neg()")


def _features_axis(x, dim):
    _check_kind(x)
    if x.dim() == 0 or not -x.dim() <= dim < x.dim():
        raise ValueError("no axis %d in shape %s" % (dim, tuple(x.shape)))
    dim %= x.dim()
    if x.shape[dim] == 0:
        raise ValueError("no features (shape %s)" % (tuple(x.shape),))
    return dim


def _same_kind(x, t, what):
    if t.shape != x.shape or t.dtype != x.dtype or t.device != x.device:
        raise ValueError("%s: %s %s on %s where %s %s on %s is wanted" % (what, tuple(t.shape), t.dtype, t.device,
                                                                         tuple(x.shape), x.dtype, x.device))
    _check_sign(t)


def _same(x, t, view, dim, what):
    """The view of another activation tensor of the same call."""
    _same_kind(x, t, what)
    v = _view(t, dim)
    if (v.outer, v.inner) != (view.outer, view.inner):
        raise ValueError("%s has its elements in another order than the first tensor" % what)
    return v


def _match(x, t, dim):
    """``t`` itself if the calls take it next to ``x`` or refuse it, else a copy in x's order (cotangents come in any order)."""
    t = t.resolve_neg()
    if t.shape != x.shape or t.dtype != x.dtype or t.device != x.device or (t.is_contiguous() and x.is_contiguous()):
        return t
    view = _view(x, dim)
    try:
        v = _view(t, dim)
        if (v.outer, v.inner) == (view.outer, view.inner):
            return t
    except ValueError:
        pass
    return _like(x, dim, view).copy_(t)


def _weight_type(x, features, weight, bias=None):
    """The type of the weights.  None stands for ones or zeros."""
    kind, device = None, x.get_device()
    for w in (weight, bias):
        if w is None:
            continue
        if w.dim() != 1 or w.numel() != features or w.get_device() != device or not w.is_contiguous() or w.is_neg():
            raise ValueError("weights: a contiguous vector of %d features on %s is wanted (.contiguous(), .resolve_neg())"
                             % (features, x.device))
        if w.dtype not in (torch.float32, x.dtype) or kind not in (None, w.dtype):
            raise ValueError("weights: %s where float32 or %s is wanted, the same for all" % (w.dtype, x.dtype))
        kind = w.dtype
    return torch.float32 if kind is None else kind


def _check_statistics(x, shape, mean, rstd):
    device = x.get_device()
    for t in (mean, rstd):
        if t.shape != shape or t.dtype is not torch.float32 or t.get_device() != device or not t.is_contiguous() or t.is_neg():
            raise ValueError("statistics: contiguous float32 of shape %s is wanted (.contiguous(), .resolve_neg())" % (tuple(shape),))


class _On:
    """The tensor's device as the current one, for a call's duration (None: it is)."""
    __slots__ = ("other",)

    def __init__(self, x):
        self.other = None if x is None or x.get_device() == _current_device() else torch.cuda.device(x.device)

    def __enter__(self):
        if self.other is not None:
            self.other.__enter__()

    def __exit__(self, *a):
        if self.other is not None:
            self.other.__exit__(*a)


_HERE = _On(None)


def _current_device():
    """torch.cuda.current_device() without its checks where torch offers that (not part of its documented interface)."""
    try:
        return torch._C._cuda_getDevice()
    except AttributeError:
        return torch.cuda.current_device()


class _Call:
    """What a call on contiguous tensors of one shape and type takes, apart from addresses: the structure to copy, the shape of
    the statistics, the bytes of a VJP's scratch.  Kept by shape and type: filling these takes longer than the kernels of a small
    call (tail of 20 x 160, forward and VJP: 64 us)."""
    __slots__ = ("dim", "features", "stats", "template", "scratch")

    def __init__(self, x, dim, wtype, eps):
        self.dim = _features_axis(x, dim)
        v = _View(_numel(x.shape[:self.dim]), x.shape[self.dim], _numel(x.shape[self.dim + 1:]), 0, False)
        self.features = v.features
        self.stats = torch.Size(x.shape[:self.dim] + x.shape[self.dim + 1:])
        d = _dims(x, wtype, v, eps, ())
        d.stream = None
        self.scratch = max(_b.gleam_layer_norm_workspace_size(d), 256)
        self.template = bytes(d)


_CALLS = {}
_CALLS_MOST = 256                                # beyond that the table starts over
_new_dims = _b.gleam_feature_dims.from_buffer_copy


def _call(x, dim, wtype, eps):
    key = (x.shape, x.dtype, dim, wtype, float(eps))
    c = _CALLS.get(key)
    if c is None:
        c = _Call(x, dim, wtype, eps)
        if len(_CALLS) >= _CALLS_MOST:
            _CALLS.clear()
        _CALLS[key] = c
    return c


def _plain(x, *others):
    """Whether all tensors are contiguous CUDA tensors of x's shape and type on the current device (None: not there), with the
    values that their memory holds."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda or not x.is_contiguous() or x.numel() == 0 or x.is_neg():
        return False
    device, shape, dtype = x.get_device(), x.shape, x.dtype
    if device != _current_device() or dtype not in _DTYPES:
        return False
    for t in others:
        if t is not None and not (t.is_contiguous() and t.shape == shape and t.dtype is dtype and t.get_device() == device and not t.is_neg()):
            return False
    return True


def _dims(x, wtype, view, eps, pitches):
    return _b.gleam_feature_dims(1, _DTYPES[x.dtype], _DTYPES[wtype], eps, view.outer, view.features, view.inner, pitches,
                                 _stream(x) or None, None, 0)


def _stream(x):
    """Handle of the current stream of the tensor's device."""
    if x.get_device() != _current_device():
        return torch.cuda.current_stream(x.device).cuda_stream
    return _b._current_stream_handle()


def _drop_args(x, p, seed, offset, step):
    if not 0.0 <= p <= 1.0:
        raise ValueError("p = %r is not a probability" % (p,))
    if step is not None and (step.dtype != torch.int64 or step.numel() != 1 or step.device != x.device):
        raise ValueError("step: one int64 value on %s is wanted" % x.device)
    return _b.make_dropout_args(p, seed, offset, step)


def _workspace(x, dims, wanted):
    """Scratch of a VJP from torch's allocator, put into ``dims``; the caller holds it until the call is made."""
    if not wanted:
        return None
    ws = torch.empty(max(_b.gleam_layer_norm_workspace_size(dims), 256), dtype=torch.uint8, device=x.device)
    dims.workspace, dims.workspace_bytes = ws.data_ptr(), ws.numel()
    return ws


class _Prepared:
    """Views, outputs' layout and structure of one norm call on the tensors x, *others: the general way, or from the kept
    table where all are plain."""
    __slots__ = ("dim", "features", "wtype", "stats", "view", "dims", "scratch", "device")

    def __init__(self, x, dim, eps, weight, bias, *others):
        if _plain(x, *[t for t, _ in others]):
            self.wtype = _weight_type(x, weight.numel() if weight is not None else bias.numel() if bias is not None else 0, weight, bias)
            c = _call(x, dim, self.wtype, eps)
            if (weight is not None and weight.numel() != c.features) or (bias is not None and bias.numel() != c.features):
                _weight_type(x, c.features, weight, bias)                # raises
            self.dim, self.features, self.stats, self.view, self.scratch = c.dim, c.features, c.stats, None, c.scratch
            self.dims = _new_dims(c.template)
            self.dims.stream = _b._current_stream_handle() or None
            self.device = _HERE
            return
        self.dim = dim = _features_axis(x, dim)
        self.view = v = _view(x, dim)
        views = [v if t is None else _same(x, t, v, dim, what) for t, what in others]
        self.features = v.features
        self.wtype = _weight_type(x, v.features, weight, bias)
        self.stats = x.shape[:dim] + x.shape[dim + 1:]
        self.scratch = None
        self.dims = _dims(x, self.wtype, v, eps, tuple([u.pitch for u in views]))
        self.device = _On(x)

    def like(self, x):
        return torch.empty_like(x) if self.view is None else _like(x, self.dim, self.view)

    def vectors(self, x, weight, *wanted):
        out = [None, None]
        for k, w in enumerate(wanted):
            if w:
                out[k] = torch.empty_like(weight) if weight is not None else x.new_empty(self.features, dtype=self.wtype)
        return out

    def statistics(self, x):
        # the cheapest of torch's ways to new memory (1.4 us; torch.empty with a device takes 3.0, new_empty 2.3)
        mean = torch.empty_strided(self.stats, _steps(self.stats), dtype=torch.float32, device=x.device)
        return mean, torch.empty_like(mean)

    def workspace(self, x, wanted):
        if not wanted:
            return None
        if self.scratch is None:
            return _workspace(x, self.dims, True)
        ws = torch.empty_strided((self.scratch,), (1,), dtype=torch.uint8, device=x.device)
        self.dims.workspace, self.dims.workspace_bytes = ws.data_ptr(), self.scratch
        return ws


# A contiguous array's pitch is 0 in the structure, so that the order of the arguments does not matter to the kept one.

def layer_norm_forward(x, weight=None, bias=None, eps=1e-5, dim=-1):
    """(y, mean, rstd): y = (x - mean) rstd weight + bias over axis ``dim``; mean and rstd are float32 without that axis."""
    c = _Prepared(x, dim, eps, weight, bias, (None, "x"))
    y = c.like(x)
    mean, rstd = c.statistics(x)
    with c.device:
        _b.gleam_layer_norm_forward(x, weight, bias, y, mean, rstd, c.dims)
    return y, mean, rstd


def layer_norm_vjp(grad_y, x, weight, mean, rstd, dim=-1, weight_grad=True, bias_grad=True):
    """(grad_x, grad_weight, grad_bias) of ``layer_norm_forward``; the last two are None where they are not wanted."""
    c = _Prepared(x, dim, 0.0, weight, None, (grad_y, "grad_y"), (None, "x"))
    _check_statistics(x, c.stats, mean, rstd)
    gx = c.like(x)
    gw, gb = c.vectors(x, weight, weight_grad, bias_grad)
    with c.device:
        ws = c.workspace(x, weight_grad or bias_grad)
        _b.gleam_layer_norm_vjp(grad_y, x, weight, mean, rstd, gx, gw, gb, c.dims)
    del ws
    return gx, gw, gb


def _memory_order(x):
    """The axes from the slowest to the fastest in memory."""
    strides = x.stride()
    return sorted(range(x.dim()), key=lambda k: -strides[k])


def _flat(first, *others):
    """(outer, elements of a slice, pitches) for a call that knows no features; the tensors have one memory order."""
    if all(t.is_contiguous() for t in (first,) + others):
        return 1, first.numel(), [0] * (1 + len(others))
    axes = _memory_order(first)
    tensors = [t.permute(axes) for t in (first,) + others]
    for dim in range(first.dim()):
        got = [_slices(t.shape, t.stride(), dim) for t in tensors]
        if None not in got:
            return got[0][0], _numel(tensors[0].shape[dim:]), [g[2] for g in got]
    raise ValueError("memory order not supported (shape %s, strides %s): call .contiguous()"
                     % (tuple(first.shape), " and ".join(str(tuple(t.stride())) for t in (first,) + others)))


def _dense(x):
    """A tensor like x whose elements have x's order in memory, without gaps."""
    if x.is_contiguous():
        return torch.empty(x.shape, dtype=x.dtype, device=x.device)
    axes = _memory_order(x)
    t = torch.empty([x.shape[k] for k in axes], dtype=x.dtype, device=x.device)
    return t.permute([axes.index(k) for k in range(x.dim())])


def _residual_beside(x, t):
    """``t`` itself if dropout takes it next to ``x`` or refuses it, else a copy in x's order."""
    if t is None or (t.is_contiguous() and x.is_contiguous() and not t.is_neg()):
        return t
    if t.shape != x.shape or t.dtype != x.dtype or t.device != x.device:
        return t
    t = t.resolve_neg()
    try:
        _flat(x, t)
    except ValueError:
        return _dense(x).copy_(t)
    return t


def dropout_forward(x, p, seed, offset, residual=None, step=None):
    """[residual +] dropout(x).  The call takes ceil(x.numel() / 4) counters from ``offset``."""
    if _plain(x, residual):
        outer, slice_, pitch, device = 1, x.numel(), (), _HERE
        out = torch.empty_like(x)
    else:
        _check_kind(x)
        others = ()
        if residual is not None:
            _same_kind(x, residual, "residual")
            others = (residual,)
        outer, slice_, pitch = (1, 0, ()) if x.numel() == 0 else _flat(x, *others)
        out, device = _dense(x), _On(x)
    args = _drop_args(x, p, seed, offset, step)
    with device:
        dims = _b.gleam_feature_dims(1, _DTYPES[x.dtype], _b.GLEAM_F32, 0.0, outer, 1, slice_, tuple(pitch),
                                     _stream(x) or None, None, 0)
        _b.gleam_dropout_forward(x, residual, out, args, dims)
    return out


def dropout_vjp(grad_out, p, seed, offset, step=None):
    """Gradient with respect to x of ``dropout_forward`` with the same arguments (that of residual is grad_out itself);
    grad_out has x's memory order."""
    return dropout_forward(grad_out, p, seed, offset, None, step)


def dropout_add_layer_norm_forward(x, residual, weight, bias, p, seed, offset, eps=1e-5, dim=-1, step=None):
    """(y, total, mean, rstd): total = residual + dropout(x), y = layer norm of total over axis ``dim``."""
    c = _Prepared(x, dim, eps, weight, bias, (None, "x"), (residual, "residual"))
    args = _drop_args(x, p, seed, offset, step)
    y, total = c.like(x), c.like(x)
    mean, rstd = c.statistics(x)
    with c.device:
        _b.gleam_dropout_add_layer_norm_forward(x, residual, weight, bias, total, y, mean, rstd, args, c.dims)
    return y, total, mean, rstd


def dropout_add_layer_norm_vjp(grad_y, grad_total, total, weight, mean, rstd, p, seed, offset, dim=-1, step=None,
                               weight_grad=True, bias_grad=True):
    """(grad_x, grad_residual, grad_weight, grad_bias); ``grad_total`` (None: zero) is the cotangent of total."""
    c = _Prepared(total, dim, 0.0, weight, None, (grad_y, "grad_y"), (grad_total, "grad_total"), (None, "total"))
    _check_statistics(total, c.stats, mean, rstd)
    args = _drop_args(total, p, seed, offset, step)
    gx, gr = c.like(total), c.like(total)
    gw, gb = c.vectors(total, weight, weight_grad, bias_grad)
    with c.device:
        ws = c.workspace(total, weight_grad or bias_grad)
        _b.gleam_dropout_add_layer_norm_vjp(grad_y, grad_total, total, weight, mean, rstd, gx, gr, gw, gb, args, c.dims)
    del ws
    return gx, gr, gw, gb


# ---- autograd ------------------------------------------------------------------------------------------------------------

class DropoutGenerator:
    """Counter ranges for the dropout sites of a model: every call that drops takes the range behind the last one (a call that is
    then refused spends it), so no two share a mask, whichever threads they come from; p = 0, as in an evaluation, takes none.
    A copy (``copy.deepcopy``, pickling) stands where the first one stood and goes its own way.  A generator is no part of a
    module's state: a run that is resumed loads the ``state_dict()`` saved with the optimiser's, or it would draw its first
    masks again.

    ``capturable=True`` adds a counter on the device that the kernels read when they run: a captured training step ends with
    ``advance()`` inside the graph, and every replay draws new masks with the ranges it was captured with.  The counter must
    not move between a forward call and its backward pass (autograd and ``recompute`` raise if it has, but do not see what a
    replayed graph does to it), and the generator lives as long as a graph that reads it.

    A forward pass that is run again in the backward pass (activation checkpointing) has to take its first ranges again:
    ``torch.utils.checkpoint.checkpoint(f, x, use_reentrant=False, context_fn=generator.recompute)``.  Without that it would
    draw other masks than the outputs were made with.
    """

    def __init__(self, seed, device="cuda", capturable=False):
        self.seed, self.offset = int(seed), 0
        self.step = torch.zeros(1, dtype=torch.int64, device=device) if capturable else None
        self._unshared()

    def _unshared(self):
        self._lock = threading.Lock()
        self._here = threading.local()               # .passes: the passes that are under way in this thread, the outermost first

    def __getstate__(self):
        return {k: v for k, v in self.__dict__.items() if k not in ("_lock", "_here")}

    def __setstate__(self, state):
        self.__dict__.update(state)
        self._unshared()

    def _passes(self):
        try:
            return self._here.passes
        except AttributeError:
            self._here.passes = []
            return self._here.passes

    def take(self, numel):
        count = (int(numel) + 3) // 4
        told, offset = [], None
        for p in reversed(self._passes()):
            if isinstance(p, _Again):
                offset = p.next(count, self.step)    # passes around this one had nothing to do with its first run
                break
            told.append(p)
        if offset is None:
            with self._lock:
                offset = self.offset
                self.offset += count
        for p in told:
            p.taken.append((offset, count, None if self.step is None else self.step._version))
        return offset

    def recompute(self):
        """The contexts of a forward pass and of its recomputation, in which the ranges of the former are taken again."""
        first = _Ranges(self)
        return first, _RangesAgain(first)

    def state_dict(self):
        """Where the generator stands, in plain numbers (waits for the device's counter)."""
        with self._lock:
            return {"seed": self.seed, "offset": self.offset, "step": None if self.step is None else int(self.step)}

    def load_state_dict(self, state):
        seed, offset, step = int(state["seed"]), int(state["offset"]), state["step"]
        step = None if step is None else int(step)
        if (step is None) != (self.step is None):
            raise ValueError("a state with%s a counter for a generator with capturable=%s" % ("out" * (step is None), self.step is not None))
        with self._lock:
            self.seed, self.offset = seed, offset
            if step is not None:
                self.step.fill_(step)

    def advance(self):
        if self.step is None:
            raise RuntimeError("advance() needs capturable=True")
        self.step.add_(1)


class _Ranges:
    """Notes the ranges that a forward pass takes."""

    def __init__(self, generator):
        self.generator, self.taken, self.passes = generator, [], None

    def __enter__(self):
        self.passes = self.generator._passes()
        self.passes.append(self)

    def __exit__(self, *a):
        # not always the innermost one: a pass that raised ends when its frames are released
        self.passes.remove(self)


class _Again:
    """One recomputation of a pass: the ranges that it has not yet asked for."""

    def __init__(self, first):
        self.first, self.left = first, iter(first.taken)

    def next(self, count, step):
        offset, wanted, version = next(self.left, (None, None, None))
        if count != wanted:
            raise RuntimeError("the recomputed pass asks for other ranges than the forward pass did")
        # the check that autograd makes of a saved tensor: a recomputation saves the counter anew, so nobody else would see it
        if step is not None and step._version != version:
            raise RuntimeError("the generator's counter has moved since the forward pass that is recomputed: advance() belongs "
                               "behind the backward pass")
        return offset


class _RangesAgain:
    """The ranges of a noted pass once more; a graph that is kept may ask for this more than once."""

    def __init__(self, first):
        self.first = first

    def __enter__(self):
        self.first.generator._passes().append(_Again(self.first))

    def __exit__(self, *a):
        passes = self.first.generator._passes()
        passes.remove(next(p for p in reversed(passes) if isinstance(p, _Again) and p.first is self.first))


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, dim):
        y, mean, rstd = layer_norm_forward(x, weight, bias, eps, dim)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.dim = dim
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        x, weight, mean, rstd = ctx.saved_tensors
        dim = ctx.dim % x.dim()
        gx, gw, gb = layer_norm_vjp(_match(x, grad, dim), x, weight, mean, rstd, dim, ctx.needs_input_grad[1],
                                    ctx.needs_input_grad[2])
        return gx, gw, gb, None, None


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, seed, offset, step):
        out = dropout_forward(x, p, seed, offset, _residual_beside(x, residual), step)
        ctx.save_for_backward(step)
        ctx.args = p, seed, offset
        ctx.axes = _memory_order(x)
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        (step,) = ctx.saved_tensors
        gx = None
        if ctx.needs_input_grad[0]:
            axes = ctx.axes                              # the mask numbers elements in x's memory order
            gx = dropout_vjp(grad.permute(axes).contiguous().resolve_neg(), *ctx.args, step=step)
            gx = gx.permute([axes.index(k) for k in range(len(axes))])
        return gx, grad if ctx.needs_input_grad[1] else None, None, None, None, None


class _Tail(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, weight, bias, p, seed, offset, eps, dim, step):
        residual = _match(x, residual, _features_axis(x, dim))
        y, total, mean, rstd = dropout_add_layer_norm_forward(x, residual, weight, bias, p, seed, offset, eps, dim, step)
        ctx.save_for_backward(total, weight, mean, rstd, step)
        ctx.args, ctx.dim = (p, seed, offset), dim
        ctx.set_materialize_grads(False)
        return y, total

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_y, grad_total):
        total, weight, mean, rstd, step = ctx.saved_tensors
        dim = ctx.dim % total.dim()
        none = (None,) * 6
        if grad_y is None and grad_total is None:
            return (None,) * 4 + none
        grad_y = torch.zeros_like(total) if grad_y is None else _match(total, grad_y, dim)
        if grad_total is not None:
            grad_total = _match(total, grad_total, dim)
        gx, gr, gw, gb = dropout_add_layer_norm_vjp(grad_y, grad_total, total, weight, mean, rstd, *ctx.args, dim, step,
                                                    ctx.needs_input_grad[2], ctx.needs_input_grad[3])
        return (gx, gr, gw, gb) + none


def layer_norm(x, weight=None, bias=None, eps=1e-5, dim=-1):
    """Layer norm over axis ``dim`` with gradients for x, weight and bias."""
    return _LayerNorm.apply(x, weight, bias, eps, dim)


def _site(x, p, generator):
    """(seed, offset, step) of a call.  Where nothing is dropped there is no mask: no range is taken and no counter read."""
    if p == 0:
        return 0, 0, None
    if generator is None:
        raise ValueError("dropout needs a generator")
    return generator.seed, generator.take(x.numel()), generator.step


def dropout(x, p, generator=None, residual=None):
    """[residual +] dropout(x) with the next range of the generator, which may be None where p is 0; the backward pass draws the
    mask again."""
    return _Dropout.apply(x, residual, p, *_site(x, p, generator))


def dropout_add_layer_norm(x, residual, weight, bias, p, generator=None, eps=1e-5, dim=-1):
    """(y, total) of the residual tail, with gradients; ``generator`` may be None where p is 0."""
    seed, offset, step = _site(x, p, generator)
    return _Tail.apply(x, residual, weight, bias, p, seed, offset, eps, dim, step)
