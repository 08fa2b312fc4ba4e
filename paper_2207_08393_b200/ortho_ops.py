"""Orthogonalised updates of a prior's matrices (include/gleam.h states the formulas).

``orthogonalise`` takes matrices towards U V^T of their singular value decomposition by products alone; ``muon_step`` updates weights with
the orthogonalised momentum of their gradients; ``Muon`` is the optimiser around it (K. Jordan et al., "Muon: an optimizer for hidden
layers in neural networks", 2024).  Weights with more than two axes count as matrices (axis 0, all others), as those of convolutions do.

Tensors are CUDA tensors of float32, float16 or bfloat16; the arithmetic is near that of 32-bit products whatever the type (include/gleam.h
says how near).  Should a kernel give up waiting for its own copies (after two seconds, which no working launch needs), what it was to compute is
NaN, updated weights included.
"""
from __future__ import annotations

import torch

from . import binding as _b
from .prior_ops import _DTYPES, _On, _check_kind, _numel, _stream

COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def _dims(x, count, rows, cols, steps, coefficients, eps):
    a, b, c = coefficients
    return _b.gleam_matrix_dims(1, _DTYPES[x.dtype], count, rows, cols, steps, a, b, c, eps, _stream(x) or None, None, 0)


def _workspace(x, dims):
    size = _b.gleam_orthogonalise_workspace_size(dims)
    if not size:
        return None
    ws = torch.empty_strided((size,), (1,), dtype=torch.uint8, device=x.device)
    dims.workspace, dims.workspace_bytes = ws.data_ptr(), size
    return ws


def _check_grad(*tensors):
    if torch.is_grad_enabled() and any(t.requires_grad for t in tensors):
        raise ValueError("not differentiable: call it under torch.no_grad()")


def orthogonalise(x, steps=5, coefficients=COEFFICIENTS, eps=1e-7):
    """X_0 = x / (|x| + eps), then ``steps`` times X <- a X + (b A + c A A) X with A = X X^T over the shorter side, for every matrix in the
    last two axes of ``x``; the result has x's type.  Not differentiable: an x that requires gradients is taken under ``torch.no_grad()``."""
    _check_kind(x)
    _check_grad(x)
    if x.dim() < 2:
        raise ValueError("a matrix is wanted, or several (shape %s)" % (tuple(x.shape),))
    if not x.is_contiguous():
        raise ValueError("memory order not supported (shape %s, strides %s): call .contiguous()" % (tuple(x.shape), tuple(x.stride())))
    rows, cols = x.shape[-2:]
    count = _numel(x.shape[:-2])
    out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    with _On(x):
        dims = _dims(x, count, rows, cols, steps, coefficients, eps)
        ws = _workspace(x, dims)
        size = rows * cols * x.element_size()
        first, to = x.data_ptr(), out.data_ptr()
        _b.gleam_orthogonalise(range(first, first + count * size, size) if ws is not None else [],
                               range(to, to + count * size, size) if ws is not None else [], dims)
    del ws
    return out


def muon_step(weights, grads, momenta, lr, momentum=0.95, nesterov=True, weight_decay=0.0, scale=1.0, steps=5,
              coefficients=COEFFICIENTS, eps=1e-7):
    """For every matrix of the lists, all of one shape, in place:

        momentum <- mu momentum + grad,   u = grad + mu momentum (nesterov) or momentum,
        weight <- (1 - lr weight_decay) weight - lr scale orthogonalise(u)

    Weights and gradients have one type, momenta are float32; all are contiguous.  Weights that require gradients are taken under
    ``torch.no_grad()``.  A captured call keeps the lr that it was given."""
    if not len(weights) == len(grads) == len(momenta):
        raise ValueError("%d weights, %d gradients, %d momenta" % (len(weights), len(grads), len(momenta)))
    if not weights:
        return
    w0 = weights[0]
    _check_kind(w0)
    shape, dtype, device = w0.shape, w0.dtype, w0.device
    if len(shape) < 2:
        raise ValueError("weights: matrices are wanted (shape %s)" % (tuple(shape),))
    for what, tensors, kind in (("weights", weights, dtype), ("gradients", grads, dtype), ("momenta", momenta, torch.float32)):
        for t in tensors:
            if t.shape != shape or t.dtype is not kind or t.device != device or not t.is_contiguous() or t.is_neg():
                raise ValueError("%s: %s %s on %s where contiguous %s %s on %s is wanted" % (what, tuple(t.shape), t.dtype, t.device,
                                                                                            tuple(shape), kind, device))
        _check_grad(*tensors)
    with _On(w0):
        dims = _dims(w0, len(weights), shape[0], _numel(shape[1:]), steps, coefficients, eps)
        ws = _workspace(w0, dims)
        if ws is not None:
            _b.gleam_muon_step(weights, grads, momenta, _b.gleam_muon_args(lr, momentum, weight_decay, scale, bool(nesterov)), dims)
            for tensors in (weights, momenta):
                torch.autograd.graph.increment_version([t for t in tensors if not t.is_inference()])
    del ws


class Muon(torch.optim.Optimizer):
    """Updates matrices (weights with two axes or more) by ``muon_step``; those of one shape and type go together.  ``scale`` is a number
    or "rms" for 0.2 sqrt(max(rows, columns)), with which updates are as large as Adam's (J. Liu et al., "Muon is scalable for LLM training",
    2025).  Vectors (biases, norms) belong to another optimiser.  Take a first step before one is captured: it makes the momenta."""

    def __init__(self, params, lr=0.02, momentum=0.95, nesterov=True, weight_decay=0.0, scale="rms", steps=5, coefficients=COEFFICIENTS,
                 eps=1e-7):
        if not lr >= 0.0 or not 0.0 <= momentum < 1.0 or not weight_decay >= 0.0:
            raise ValueError("lr = %r, momentum = %r, weight_decay = %r" % (lr, momentum, weight_decay))
        if scale != "rms" and not isinstance(scale, (int, float)):
            raise ValueError("scale = %r is neither a number nor \"rms\"" % (scale,))
        super().__init__(params, dict(lr=lr, momentum=momentum, nesterov=nesterov, weight_decay=weight_decay, scale=scale, steps=steps,
                                      coefficients=tuple(coefficients), eps=eps))

    def add_param_group(self, group):
        super().add_param_group(group)
        for p in self.param_groups[-1]["params"]:
            if p.dim() < 2:
                self.param_groups.pop()
                raise ValueError("a parameter of shape %s is no matrix: give it to another optimiser" % (tuple(p.shape),))

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for group in self.param_groups:
            alike = {}
            for p in group["params"]:
                if p.grad is None or p.numel() == 0:
                    continue
                if p.grad.is_sparse:
                    raise ValueError("sparse gradients are not supported")
                state = self.state[p]
                if "momentum" not in state:
                    if group["momentum"] and p.is_cuda and torch.cuda.is_current_stream_capturing():
                        raise RuntimeError("the first step makes the momenta: take it before a capture, whose every replay would empty them")
                    state["momentum"] = torch.zeros(p.shape, dtype=torch.float32, device=p.device)
                alike.setdefault((p.shape, p.dtype, p.device), []).append(p)
            for params in alike.values():
                shape = params[0].shape
                scale = 0.2 * max(shape[0], _numel(shape[1:])) ** 0.5 if group["scale"] == "rms" else float(group["scale"])
                # a weight in another memory order (channels_last) is updated in a copy
                weights = [p if p.is_contiguous() else p.contiguous() for p in params]
                muon_step(weights, [p.grad.contiguous().resolve_neg() for p in params], [self.state[p]["momentum"] for p in params], float(group["lr"]),
                          group["momentum"], group["nesterov"], group["weight_decay"], scale, group["steps"], group["coefficients"],
                          group["eps"])
                for p, w in zip(params, weights):
                    if w is not p:
                        p.copy_(w)
        return loss

    def load_state_dict(self, state):
        names = [i for group in state["param_groups"] for i in group["params"]]
        momenta = {i: s["momentum"] for i, s in state["state"].items() if "momentum" in s}
        params = [p for group in self.param_groups for p in group["params"]]
        for i, p in zip(names, params):
            if i in momenta and momenta[i].shape != p.shape:
                raise ValueError("momentum of shape %s for a parameter of shape %s" % (tuple(momenta[i].shape), tuple(p.shape)))
        super().load_state_dict(state)
        for i, p in zip(names, params):                    # the base class rounds a state to its parameter's type, and may share it
            if i in momenta:
                self.state[p]["momentum"] = torch.empty(p.shape, dtype=torch.float32, device=p.device).copy_(momenta[i])
